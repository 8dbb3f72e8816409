"""GPU tests of attention over the 4-bit page cache with a sliding window and first tokens that stay visible, against a plain
64-bit implementation, with the pages' accumulated weights."""
import numpy as np
import pytest
import torch

import kv_ref as R
import window_ref as W
from test_gpu_attend_cache import DT, cache, dev, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g
    g.build()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def reference(pool, pages, lens, q, C, H, D, scale, window, sinks):
    """out, lse, per-page weights, mag, the scores' error bound, and which pages are seen."""
    n_q, G = q.shape[1], q.shape[2] // H
    out, mag = np.zeros(q.shape), np.zeros(q.shape)
    lse, weight, err = np.zeros(q.shape[:3]), np.zeros(pages.shape), 0.0
    used = np.zeros(pages.shape, bool)
    for r, n in enumerate(lens):
        ok = W.seen(n - n_q, n_q, n, window, sinks)
        full = np.zeros((n_q, pages.shape[1] * C), bool)
        full[:, :n] = ok
        used[r] = full.reshape(n_q, -1, C).any((0, 2))
        k = v = np.zeros((0, H, D))
        if n:
            slots = np.where(used[r], pages[r], 0)[: -(-n // C)]  # the others may be anything
            k, v = R.get_tokens(pool, slots, n, C, H, D)
        for h in range(H * G):
            o, l, p, m = W.attend(q[r, :, h], k[:, h // G], v[:, h // G], ok, scale)
            out[r, :, h], lse[r, :, h], mag[r, :, h] = o, l, m
            if n:
                err = max(err, R.score_error(q[r, :, h], k[:, h // G], scale))
                at = np.zeros(pages.shape[1] * C)
                at[:n] = p.sum(0)
                weight[r] += at.reshape(-1, C).sum(1)
    return out, lse, weight, mag, err, used


CASES = [
    # lens, n_q, C, H, G, D, dtype, window, sinks
    ([1, 2, 0, 3], 1, 16, 1, 1, 64, "bf16", 1, 0),
    ([1, 2, 0, 30], 1, 16, 2, 1, 64, "fp16", 1, 1),
    ([5, 16, 17, 33, 100], 1, 16, 2, 4, 128, "bf16", 16, 0),
    ([5, 16, 17, 33, 500], 1, 16, 2, 4, 128, "bf16", 17, 4),
    ([300, 47, 48, 49, 600], 1, 48, 2, 3, 64, "fp16", 40, 17),
    ([1000, 129], 2, 256, 1, 8, 128, "fp16", 100, 0),
    ([5, 3, 70, 200], 4, 32, 2, 3, 64, "bf16", 2, 1),       # 12 rows; queries before position 0; window below the queries
    ([2500, 700, 40], 1, 16, 1, 16, 128, "bf16", 1000, 4),  # two column tiles
    ([333, 2000], 5, 16, 1, 7, 128, "fp16", 300, 100),      # 35 rows: row tiles
    ([9000], 1, 64, 3, 5, 64, "fp16", 4096, 64),            # splits
    ([5000], 3, 16, 2, 2, 128, "bf16", 4995, 3),            # the hole is a few tokens
    ([700, 90], 2, 16, 1, 2, 64, "bf16", 5000, 4),          # wider than any request
    ([700, 90], 2, 16, 1, 2, 64, "bf16", 60, 100000),       # everything is a first token
]


@pytest.mark.parametrize("weigh", [False, True])
@pytest.mark.parametrize("lens,n_q,C,H,G,D,dtype,window,sinks", CASES)
def test_matches_reference(lens, n_q, C, H, G, D, dtype, window, sinks, weigh):
    pool, pages, rng = make(lens, C, H, D, 21)
    q = torch.from_numpy(rng.standard_normal((len(lens), n_q, H * G, D)) * 2).to(DT[dtype])
    scale = D ** -0.5
    ref, rl, rw, mag, err, used = reference(pool, pages, lens, q.double().numpy(), C, H, D, scale, window, sinks)
    kv = cache(pool, C, H, D)
    pages = np.where(used, pages, -1)  # what nobody sees may have been given back
    w0 = rng.uniform(0, 2, pages.shape).astype(np.float32)
    weight = dev(w0) if weigh else None
    out, lse = kv.attend(q.cuda(), dev(np.array(lens, np.int32)), dev(pages), scale, weight, window=window, sinks=sinks)
    kv.check()
    n = max(lens)
    assert np.all(np.abs(out.double().cpu().numpy() - ref) <= R.out_bound(ref, mag, R.U["fp16"], R.U[dtype], err, n))
    gl = lse.double().cpu().numpy()
    none = np.isneginf(rl)
    assert np.array_equal(none, np.isneginf(gl))
    assert np.all(np.abs(gl[~none] - rl[~none]) <= R.lse_bound(rl, err, n)[~none])
    if weigh:
        got = weight.double().cpu().numpy()
        assert np.array_equal(got[~used], w0.astype(np.float64)[~used])
        bound = (2 * np.expm1(err) + (n + 128) * 2.0 ** -24) * rw + 2.0 ** -23 * (w0 + rw)
        assert np.all(np.abs(got - w0 - rw) <= bound + 1e-9)


def test_wide_window_is_no_window():
    """The same bits as without one, where it holds all that a request can."""
    lens, C, H, D = [300, 47, 0, 333], 16, 2, 64
    pool, pages, rng = make(lens, C, H, D, 3)
    kv = cache(pool, C, H, D)
    q = torch.from_numpy(rng.standard_normal((4, 2, 6, D))).to(torch.bfloat16).cuda()
    n, p = dev(np.array(lens, np.int32)), dev(pages)
    w = [torch.zeros(pages.shape, device="cuda") for _ in range(3)]
    want = kv.attend(q, n, p, weight=w[0])
    for i, window in ((1, pages.shape[1] * C), (2, 2 ** 31 - 1)):
        got = kv.attend(q, n, p, weight=w[i], window=window, sinks=3)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(w[i], w[0])
    kv.check()


@pytest.mark.parametrize("D,G", [(64, 2), (128, 16)])
def test_marked_blocks_reach_only_queries_that_see_them(D, G):
    """NaN blocks in V and K, at the window's ends, among the first tokens and in the hole between."""
    n, C, H, n_q, window, sinks = 150, 16, 1, 4, 20, 5
    pool, pages, rng = make([n], C, H, D, 8)
    gb = 16 * (D + D // 8)
    bad = [2, 5, 50, 126, 127, 128, 129, 130, 146, 147, 148, 149]
    for which in (0, 1):  # K, V
        for j in bad:
            marked = pool.copy()
            tok = j % C
            marked[pages[0, j // C], 16 * D + which * D + tok * (D // 16) + 1] = 0x7F  # the second block of 16 dimensions
            kv = cache(marked, C, H, D)
            q = torch.from_numpy(rng.standard_normal((1, n_q, G, D))).to(torch.float16).cuda()
            args = (q, dev(np.array([n], np.int32)), dev(pages))
            out, lse = kv.attend(*args, window=window, sinks=sinks)
            clean, clean_lse = cache(pool, C, H, D).attend(*args, window=window, sinks=sinks)
            ok = W.seen(n - n_q, n_q, n, window, sinks)[:, j]
            for i in range(n_q):
                if not ok[i]:
                    assert torch.equal(out[0, i], clean[0, i]) and torch.equal(lse[0, i], clean_lse[0, i]), (which, j, i)
                elif which:
                    assert bool(out[0, i, :, 16:32].isnan().all()) and bool(out[0, i, :, :16].isfinite().all())
                else:
                    assert bool(out[0, i].isnan().all()) and bool(lse[0, i].isnan().all())
    assert gb == pool.shape[1] // (C // 16)


def test_slots_in_sight_out_of_range():
    from paper_2609_38706_gb300 import pk
    lens, C, H, D = [200, 200], 16, 2, 64
    pool, pages, rng = make(lens, C, H, D, 3)
    kv = cache(pool, C, H, D)
    q = torch.from_numpy(rng.standard_normal((2, 1, 4, D))).to(torch.bfloat16).cuda()
    n = dev(np.array(lens, np.int32))
    w0 = torch.ones(pages.shape, device="cuda")
    weight = w0.clone()
    want, _ = kv.attend(q, n, dev(pages), weight=weight, window=50, sinks=1)
    pages[0, 11] = 1 << 20
    weight = w0.clone()
    out, lse = kv.attend(q, n, dev(pages), weight=weight, window=50, sinks=1)
    assert kv.take_status() == pk.PK_ERR_ARG
    assert bool(out[0].isnan().all()) and bool(lse[0].isnan().all()) and torch.equal(out[1], want[1])
    assert torch.equal(weight[0], w0[0]) and not torch.equal(weight[1], w0[1])


def test_wide_queries():
    """A row whose values lie far apart: what halves lose of the small one goes through its own product, under a window too."""
    n, C, H, D = 100, 16, 1, 64
    pool, pages, rng = make([n], C, H, D, 5)
    pool.reshape(-1, C // 16, 16 * (D + D // 8))[:, :, 0: 8 * D: D // 2] &= 0xF0  # K: dimension 0 holds nothing
    q = torch.from_numpy(rng.standard_normal((1, 1, 2, D))).to(torch.bfloat16)
    q[..., 0] = 2.0 ** 27
    kv = cache(pool, C, H, D)
    out, lse = kv.attend(q.cuda(), dev(np.array([n], np.int32)), dev(pages), window=30, sinks=2)
    kv.check()
    ref, rl, _, mag, err, _ = reference(pool, pages, [n], np.where(np.arange(D) == 0, 0, q.double().numpy()), C, H, D, D ** -0.5, 30, 2)
    assert np.all(np.abs(out.double().cpu().numpy() - ref) <= R.out_bound(ref, mag, R.U["fp16"], R.U["bf16"], err, n))
    assert np.all(np.abs(lse.double().cpu().numpy() - rl) <= R.lse_bound(rl, err, n))


def test_captured_with_growing_lengths():
    lens, C, H, D = [500, 61], 16, 2, 128
    pool, pages, rng = make([700, 300], C, H, D, 4)
    kv = cache(pool, C, H, D)
    q = torch.from_numpy(rng.standard_normal((2, 1, 8, D))).to(torch.float16).cuda()
    n, p = dev(np.array(lens, np.int32)), dev(pages)
    weight = torch.zeros(pages.shape, device="cuda")
    kv.attend(q, n, p, weight=weight, window=64, sinks=4)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, lse = kv.attend(q, n, p, weight=weight, window=64, sinks=4)
    for step in range(3):
        n += 50
        weight.zero_()
        g.replay()
        w2 = torch.zeros_like(weight)
        want = kv.attend(q, n, p, weight=w2, window=64, sinks=4)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and torch.equal(weight, w2)
    kv.check()


def test_refusals():
    from paper_2609_38706_gb300 import pk
    pool, pages, rng = make([40], 16, 1, 64, 4)
    kv = cache(pool, 16, 1, 64)
    q = torch.zeros((1, 1, 1, 64), dtype=torch.float16, device="cuda")
    args = (q, dev(np.array([40], np.int32)), dev(pages))
    for kw in (dict(window=0), dict(window=-1), dict(window=1 << 31), dict(window=4, sinks=-1), dict(window=4, sinks=1 << 31),
               dict(window=1 << 32)):
        with pytest.raises(pk.PKError):
            kv.attend(*args, **kw)
