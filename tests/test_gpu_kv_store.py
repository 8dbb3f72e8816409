"""GPU tests of the 4-bit page store: written bytes equal the format's definition bit for bit, bytes of other positions
stay, reading gives the stored values, non-finite blocks, strided inputs, refusals."""
import numpy as np
import pytest
import torch

import kv_ref as R

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g
    g.build()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def make(lens, starts, C, H, D, dtype, seed, k_scale=1.0, v_scale=1.0, spare=2):
    from paper_2609_38706_gb300.service import KVPages
    rng = np.random.default_rng(seed)
    n = len(lens)
    stride = max(-(-(a + b) // C) for a, b in zip(starts, lens)) if n else 1
    slots = n * stride + spare
    pages = rng.permutation(slots)[: n * stride].reshape(n, stride).astype(np.int32)
    kv = KVPages(slots, C, H, D, k_scale, v_scale)
    kv.pool.fill_(0xA5)
    off = np.concatenate(([0], np.cumsum(lens))).astype(np.int64)
    t = int(off[-1])
    x = rng.standard_normal((2, t, H, D)).astype(np.float32) * np.exp(rng.uniform(-3, 2, (2, t, H, 1))).astype(np.float32)
    x = torch.from_numpy(x).to(DT[dtype])
    return kv, pages, off, x


def expected_pool(pool, pages, off, starts, x, C, H, D, k_scale, v_scale):
    want = pool.copy()
    ref = [R.quantise(x[j].float().numpy(), g) for j, g in ((0, k_scale), (1, v_scale))]
    for r in range(len(starts)):
        for i in range(off[r], off[r + 1]):
            pos = starts[r] + i - off[r]
            for h in range(H):
                R.put_token(want, pages[r, pos // C], pos % C, h, C, H, D, ref[0][0][i, h], ref[0][1][i, h],
                            ref[1][0][i, h], ref[1][1][i, h])
    return want


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


@pytest.mark.parametrize("lens,starts,C,H,D,dtype,k_scale,v_scale", [
    ([1], [0], 16, 1, 128, "bf16", 1.0, 1.0),
    ([1, 1, 1], [15, 16, 47], 16, 3, 64, "fp16", 1.0, 1.0),
    ([37, 0, 1, 130], [5, 9, 0, 31], 48, 2, 128, "bf16", 0.0173, 0.5),
    ([300, 17], [0, 255], 256, 5, 64, "bf16", 1.0, 3.7e-3),
    ([64] * 40, list(range(40)), 32, 8, 128, "fp16", 1.0, 1.0),
])
def test_written_bytes_and_read_back(lens, starts, C, H, D, dtype, k_scale, v_scale):
    kv, pages, off, x = make(lens, starts, C, H, D, dtype, 3, k_scale, v_scale)
    before = kv.pool.cpu().numpy()
    d_off, d_start, d_pages = dev(off), dev(np.array(starts, np.int32)), dev(pages)
    kv.write(x[0].cuda(), x[1].cuda(), d_off, d_start, d_pages)
    kv.check()
    got = kv.pool.cpu().numpy()
    assert np.array_equal(got, expected_pool(before, pages, off, starts, x, C, H, D, k_scale, v_scale))
    k, v = kv.read(d_off, d_start, d_pages, x.shape[1], x.dtype)
    kv.check()
    for y, j, g in ((k, 0, k_scale), (v, 1, v_scale)):
        want = torch.from_numpy(R.dequantise(*R.quantise(x[j].float().numpy(), g), g)).to(torch.float32).to(x.dtype)
        assert torch.equal(y.cpu(), want)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_ties_extremes_and_non_finite_blocks(dtype):
    C, H, D = 16, 1, 64
    kv, pages, off, x = make([16], [0], C, H, D, dtype, 4)
    k = x[0].clone()
    # every multiple of 1/8 between two codes, so every tie; one block's scale is exactly 1, another's 1.25
    k[0, 0, :16] = torch.tensor([6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -.75, -1.25, -1.75, -2.5, -3.5, -5, -0.])
    k[0, 0, 16:32] = k[0, 0, :16] * 1.25
    k[0, 0, 32:48] = 0
    k[0, 0, 48:] = -0.0
    k[1, 0, 3], k[1, 0, 17], k[1, 0, 40] = float("nan"), float("inf"), float("-inf")
    k[2] = torch.finfo(k.dtype).max
    k[3] = torch.finfo(k.dtype).tiny
    k[4] = k[4] * 1e-3
    x = torch.stack((k, x[1]))
    before = kv.pool.cpu().numpy()
    args = dev(off), dev(np.zeros(1, np.int32)), dev(pages)
    kv.write(x[0].cuda(), x[1].cuda(), *args)
    kv.check()
    assert np.array_equal(kv.pool.cpu().numpy(), expected_pool(before, pages, off, [0], x, C, H, D, 1.0, 1.0))
    got = kv.read(*args, 16, x.dtype)[0].cpu()
    bad = torch.isnan(got[1, 0]).reshape(4, 16).all(1)
    assert bad.tolist() == [True, True, True, False] and not torch.isnan(got[0]).any() and not torch.isnan(got[2:]).any()


def test_strided_inputs_and_another_stream():
    """K and V as slices of one fused projection, and head-major; written and read on a side stream."""
    from paper_2609_38706_gb300.service import KVPages
    C, H, D, lens = 16, 4, 128, [33, 20]
    kv, pages, off, x = make(lens, [0, 3], C, H, D, "bf16", 5)
    t = x.shape[1]
    fused = torch.zeros((t, 3 * H + 1, D), dtype=x.dtype, device="cuda")
    fused[:, H:2 * H], fused[:, 2 * H:3 * H] = x[0].cuda(), x[1].cuda()
    args = dev(off), dev(np.array([0, 3], np.int32)), dev(pages)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = KVPages(kv.pool.shape[0], C, H, D, stream=side, pool=kv.pool.clone())
    side.wait_stream(torch.cuda.current_stream())
    kv.write(x[0].cuda(), x[1].cuda(), *args)
    other.write(fused[:, H:2 * H], fused[:, 2 * H:3 * H], *args)
    k, v = other.read(*args, t)
    side.synchronize()
    assert torch.equal(kv.pool, other.pool)
    head_major = x[0].cuda().transpose(0, 1).contiguous().transpose(0, 1)
    again = KVPages(kv.pool.shape[0], C, H, D, pool=torch.full_like(kv.pool, 0xA5))
    again.write(head_major, x[1].cuda(), *args)
    assert torch.equal(kv.pool, again.pool)
    assert torch.equal(k, kv.read(*args, t)[0])
    # rows that start on 16 bytes but not on 32
    odd = torch.zeros(t * H * D + 16, dtype=x.dtype, device="cuda")[8:-8].view(t, H, D)
    odd.copy_(x[0])
    third = KVPages(kv.pool.shape[0], C, H, D, pool=torch.full_like(kv.pool, 0xA5))
    third.write(odd, x[1].cuda(), *args)
    assert torch.equal(kv.pool, third.pool)
    from paper_2609_38706_gb300 import pk
    v2 = torch.empty_like(k)
    odd.zero_()
    pk.pk_kv_read(kv.kv, odd, v2, *args, kv.status)
    assert torch.equal(odd, k) and torch.equal(v2, v)
    kv.check(), other.check(), again.check()


def test_empty_calls():
    from paper_2609_38706_gb300.service import KVPages
    kv = KVPages(1, 16, 2, 64)
    e = torch.empty((0, 2, 64), dtype=torch.float16, device="cuda")
    kv.write(e, e, dev(np.zeros(1, np.int64)), dev(np.zeros(0, np.int32)), torch.empty((0, 0), dtype=torch.int32, device="cuda"))
    kv.write(e, e, dev(np.zeros(3, np.int64)), dev(np.zeros(2, np.int32)), torch.empty((2, 0), dtype=torch.int32, device="cuda"))
    kv.check()


@pytest.mark.parametrize("what", ["slot", "start", "negative start", "order", "range"])
def test_device_errors_are_reported_and_write_nothing_else(what):
    from paper_2609_38706_gb300 import pk
    kv, pages, off, x = make([20, 20], [0, 0], 16, 2, 64, "bf16", 6)
    start = np.zeros(2, np.int32)
    off = off.copy()
    if what == "slot":
        pages[1] = kv.pool.shape[0]
    elif what == "start":
        start[1] = 32 - 19
    elif what == "negative start":
        start[1] = -3
    elif what == "order":
        off[1] = 45
    else:
        off[2] = 1 << 40
    before = kv.pool.cpu().numpy()
    kv.write(x[0].cuda(), x[1].cuda(), dev(off), dev(start), dev(pages))
    assert kv.take_status() == pk.PK_ERR_ARG
    spare = sorted(set(range(kv.pool.shape[0])) - set(pages.reshape(-1).tolist()))
    assert np.array_equal(kv.pool.cpu().numpy()[spare], before[spare])


def test_argument_refusals():
    from paper_2609_38706_gb300 import pk
    from paper_2609_38706_gb300.service import KVPages
    for bad in (dict(page_tokens=24), dict(page_tokens=0), dict(head_dim=96), dict(kv_heads=0), dict(n_slots=0)):
        with pytest.raises(pk.PKError):
            KVPages(**(dict(n_slots=2, page_tokens=16, kv_heads=2, head_dim=64) | bad))
    kv = KVPages(4, 16, 2, 64)
    k = torch.zeros((16, 2, 64), dtype=torch.bfloat16, device="cuda")
    off, start, pages = dev(np.array([0, 16])), dev(np.zeros(1, np.int32)), dev(np.zeros((1, 1), np.int32))
    for args in ((k.float(), k.float()), (k, k.half()), (k[:, :1], k[:, :1]), (k, k[:8]),
                 (torch.zeros(16 * 128 + 1, dtype=k.dtype, device="cuda")[1:].view(16, 2, 64), k)):
        with pytest.raises(pk.PKError):
            kv.write(*args, off, start, pages)
    with pytest.raises(pk.PKError):
        kv.write(k, k, off.int(), start, pages)
    with pytest.raises(pk.PKError):
        kv.write(k, k, off, start, pages.long())
    for s in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(pk.PKError):
            KVPages(4, 16, 2, 64, k_scale=s).write(k, k, off, start, pages)
