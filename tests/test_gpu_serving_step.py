"""GPU tests of a serving step as a loop keeps it: page tables with room to grow, and the step captured in a CUDA graph and
replayed on new inputs."""
import numpy as np
import pytest
import torch

import kv_ref as R
from test_gpu_attend_cache import cache, dev, make, reference

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g
    g.build()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("lens,n_q,C,H,G,D,dtype,stride", [
    ([40, 17, 0], 1, 16, 2, 4, 128, "bf16", 400),
    ([333, 80], 4, 16, 1, 4, 128, "fp16", 4096),
    ([1000, 1], 1, 48, 1, 3, 64, "bf16", 1000),
    ([2500], 2, 256, 1, 2, 128, "bf16", 512),
])
def test_tables_wider_than_the_requests(lens, n_q, C, H, G, D, dtype, stride):
    narrow = max(1, max(-(-n // C) for n in lens))
    pool, pages, rng = make(lens, C, H, D, 71, stride=narrow)
    wide = np.full((len(lens), stride), -1, np.int32)  # no slot: never looked at
    wide[:, :narrow] = pages
    kv = cache(pool, C, H, D)
    q = torch.from_numpy(rng.standard_normal((len(lens), n_q, H * G, D))).to(DT[dtype])
    w0 = rng.uniform(0, 2, wide.shape).astype(np.float32)
    weight = dev(w0)
    out, lse = kv.attend(q.cuda(), dev(np.array(lens, np.int32)), dev(wide), 0.125, weight)
    kv.check()
    ref, rl, rw, mag, err = reference(pool, pages, lens, q.double().numpy(), C, H, D, 0.125)
    n = max(lens)
    assert np.all(np.abs(out.double().cpu().numpy() - ref) <= R.out_bound(ref, mag, R.U["fp16"], R.U[dtype], err, n))
    gl, none = lse.double().cpu().numpy(), np.isneginf(rl)
    assert np.array_equal(none, np.isneginf(gl))
    assert np.all(np.abs(gl[~none] - rl[~none]) <= R.lse_bound(rl, err, n)[~none])
    got = weight.double().cpu().numpy()
    full = np.zeros(wide.shape)
    full[:, :narrow] = rw
    used = np.arange(stride) < np.array([-(-x // C) for x in lens])[:, None]
    assert np.array_equal(got[~used], w0.astype(np.float64)[~used])
    bound = (2 * np.expm1(err) + (n + 128) * 2.0 ** -24) * full + 2.0 ** -23 * (w0 + full)
    assert np.all(np.abs(got - w0 - full) <= bound + 1e-9)


@pytest.mark.parametrize("steps,C,H,G,D", [(3, 16, 2, 4, 128), (2, 48, 1, 3, 64)])
def test_a_captured_decode_step(steps, C, H, G, D):
    """Append, attend with page weights, cut to a budget, read back: each replay gives a plain step's bits."""
    from paper_2609_38706_gb300.service import KVPages
    lens, room = [70, 200, 15], 100
    pool, pages, rng = make(lens, C, H, D, 72, stride=-(-(max(lens) + room) // C))
    n, budget = len(lens), pages.shape[1] - 2
    new = [[torch.from_numpy(rng.standard_normal((n, h, D))).to(torch.bfloat16).cuda() for h in (H * G, H, H)] for _ in range(steps)]
    tok_off = torch.arange(n + 1, device="cuda")

    def state():
        kv = cache(pool, C, H, D)
        return kv, [x.clone() for x in new[0]], dev(np.array(lens, np.int32)), torch.zeros(pages.shape, device="cuda")

    def step(kv, x, kv_len, weight, table):
        q, k, v = x
        kv.write(k, v, tok_off, kv_len, table)
        kv_len += 1
        out, lse = kv.attend(q.unsqueeze(1), kv_len, table, weight=weight)
        cut = kv.evict(table, weight, kv_len, budget, sinks=1, recent=1)
        rows = kv.read(tok_off, kv_len - 1, table, n)
        return [out, lse, *cut, *rows]

    table = dev(pages)
    kv, x, kv_len, weight = state()
    want = []
    for s in range(steps):
        for a, b in zip(x, new[s]):
            a.copy_(b)
        want.append([t.clone() for t in step(kv, x, kv_len, weight, table)] + [weight.clone(), kv.pool.clone()])
    kv.check()

    kv, x, kv_len, weight = state()
    kept = kv.pool.clone(), kv_len.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(kv, x, kv_len, weight, table)  # loads the kernels
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(kv, x, kv_len, weight, table)
    kv.pool.copy_(kept[0]), kv_len.copy_(kept[1]), weight.zero_()
    for s in range(steps):
        for a, b in zip(x, new[s]):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got + [weight, kv.pool], want[s]):
            assert torch.equal(a, b)
    kv.check()
