"""GPU tests of attention over pages whose scores' factor, times a row's own power of two, leaves 32 bits, while the scores are 0:
all keys that a query sees weigh alike."""
import numpy as np
import pytest
import torch

import kv_ref as R
from test_gpu_attend_cache import DT, cache, dev, make
from test_gpu_attend_chunk import check, offsets, reference, roomy

pytestmark = pytest.mark.gpu

# |q| up to, scale: q's power of two times scale * log2 e passes 2^128 by far, or by the powers that a kernel brings a row to
TOPS = [("bf16", 2.0 ** 60, 1e30), ("bf16", 2.0 ** 127, 65536.0), ("bf16", 2.0 ** 60, -1e30), ("bf16", 2.0 ** 17, 2.2e38),
        ("fp16", 1000.0, 2.2e38), ("fp16", 60000.0, -1e36)]


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g
    g.build()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def flat(lens, C, H, D, seed):
    """Pages whose K is 0."""
    pool, pages, rng = make(lens, C, H, D, seed)
    pool.reshape(-1, C // 16, 16 * (D + D // 8))[:, :, : 8 * D] = 0
    return pool, pages, rng


def large(rng, shape, top, dtype):
    return torch.from_numpy(rng.uniform(0.5, 0.99, shape) * rng.choice((-1.0, 1.0), shape) * top).to(DT[dtype])


@pytest.mark.parametrize("room", [False, True])
@pytest.mark.parametrize("D,window", [(64, None), (128, None), (128, 70)])
@pytest.mark.parametrize("dtype,top,scale", TOPS)
def test_chunks(dtype, top, scale, D, window, room):
    new, lens, C, H, G = [5, 40], [300, 40], 16, 1, 2
    pool, pages, rng = flat(lens, C, H, D, 4)
    q = large(rng, (sum(new), G, D), top, dtype)
    q[3] *= 2.0 ** -20 if dtype == "bf16" else 0.0  # a row whose own factor is in range
    kv = cache(pool, C, H, D)
    out, lse = kv.attend_chunk(q.cuda(), offsets(new), dev(np.array(lens, np.int32)), dev(roomy(pages) if room else pages), scale,
                               window=window, sinks=3)
    kv.check()
    check(out, lse, *reference(pool, pages, new, lens, np.zeros(q.shape), C, H, D, 1.0, window, 3)[:4], dtype, max(lens))


@pytest.mark.parametrize("weigh", [False, True])
@pytest.mark.parametrize("D,G,n_q,window", [(64, 1, 1, None), (128, 3, 1, 70), (128, 4, 5, None), (64, 2, 3, 70)])
@pytest.mark.parametrize("dtype,top,scale", TOPS)
def test_steps(dtype, top, scale, D, G, n_q, window, weigh):
    """The same of a decode step's queries, whose page weights add up to one for each query that sees a key."""
    lens, C, H = [300, 2], 16, 2
    pool, pages, rng = flat(lens, C, H, D, 6)
    q = large(rng, (len(lens), n_q, H * G, D), top, dtype)
    q[0, 0, 0] *= 2.0 ** -20 if dtype == "bf16" else 0.0
    kv = cache(pool, C, H, D)
    weight = torch.zeros(pages.shape, dtype=torch.float32, device="cuda") if weigh else None
    out, lse = kv.attend(q.cuda(), dev(np.array(lens, np.int32)), dev(pages), scale, weight, window=window, sinks=3)
    kv.check()
    shape = (len(lens) * n_q, H * G, D)
    check(out.view(shape), lse.view(shape[:2]),
          *reference(pool, pages, [n_q] * len(lens), lens, np.zeros(shape), C, H, D, 1.0, window, 3)[:4], dtype, max(lens))
    if weigh:
        total = sum(min(n, n_q) for n in lens) * H * G
        assert abs(float(weight.sum()) - total) <= total * (max(lens) + 64) * 2.0 ** -23  # sums of 32 bits
