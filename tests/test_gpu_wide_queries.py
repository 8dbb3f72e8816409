"""GPU tests of attention over the page cache by queries whose dimensions lie far apart in size, with nothing behind the
large one in K: the small dimensions alone decide the scores."""
import numpy as np
import pytest
import torch

import kv_ref as R
from test_gpu_attend_cache import cache, dev, make

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g
    g.build()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def score_error(q, k, scale):
    """As kv_ref.score_error, but from the products themselves: those with a K of 0 are 0 and carry no rounding."""
    return (q.shape[-1] + 8) * 2.0 ** -23 * float((np.abs(q) @ np.abs(k).T).max()) * abs(scale) + 2.0 ** -20


@pytest.mark.parametrize("dtype,top,small", [
    ("fp16", 32768.0, 0.0009995), ("fp16", 65504.0, 2.0 ** -14 * 1.37), ("fp16", 60000.0, 3e-7), ("fp16", 3.0, 1.1),
    ("bf16", 2.0 ** 27, 1.0078125), ("bf16", 2.0 ** 40, 0.7), ("bf16", 1e30, 1e15), ("bf16", 1.5, 2.0 ** -50),
])
@pytest.mark.parametrize("D,H,G,n_q,lens,weigh", [
    (64, 2, 3, 1, [500, 77], True), (128, 1, 4, 1, [333], False), (128, 2, 8, 2, [900, 40], True),
    (64, 1, 5, 3, [3000], False),
])
def test_small_dimensions_beside_a_large_one(dtype, top, small, D, H, G, n_q, lens, weigh):
    C = 16
    pool, pages, rng = make(lens, C, H, D, 61)
    # K of dimension 5 is 0 everywhere (the low or high half of a code byte)
    g = 16 * (D + D // 8)
    codes = pool.reshape(pool.shape[0], H, C // 16, g)[..., : 8 * D].reshape(pool.shape[0], H, C // 16, 16, D // 2)
    codes[..., 2] &= 0x0F
    grans = pool.reshape(pool.shape[0], H, C // 16, g)
    grans[..., : 8 * D] = codes.reshape(*codes.shape[:3], -1)
    pool = grans.reshape(pool.shape[0], -1)
    kv = cache(pool, C, H, D)
    q = rng.choice((small, -small, small / 2, 0.0), (len(lens), n_q, H * G, D)) * rng.uniform(0.6, 1, (len(lens), n_q, H * G, D))
    q[..., 5] = top
    q[..., 0, 5] = small  # a row without a large dimension among them
    q = torch.from_numpy(q).to(DT[dtype])
    scale = float(np.float32(0.3 / max(small, 1e-37)))
    weight = torch.zeros(pages.shape, dtype=torch.float32, device="cuda") if weigh else None
    out, lse = kv.attend(q.cuda(), dev(np.array(lens, np.int32)), dev(pages), scale, weight)
    kv.check()
    qd = q.double().numpy()
    total_w = 0.0
    for r, n in enumerate(lens):
        k, v = R.get_tokens(pool, pages[r, : -(-n // C)], n, C, H, D)
        assert not k[..., 5].any()
        for h in range(H * G):
            ref, rl, p, mag = R.attend(qd[r, :, h], k[:, h // G], v[:, h // G], n - n_q + np.arange(n_q), scale)
            err = score_error(qd[r, :, h], k[:, h // G], scale)
            assert err < 0.02  # the bound says something
            got, gl = out[r, :, h].double().cpu().numpy(), lse[r, :, h].double().cpu().numpy()
            assert np.all(np.abs(got - ref) <= R.out_bound(ref, mag, R.U["fp16"], R.U[dtype], err, n)), (r, h)
            assert np.all(np.abs(gl - rl) <= R.lse_bound(rl, err, n)), (r, h)
            total_w += n_q
    if weigh:
        assert abs(float(weight.sum()) - total_w) <= total_w * 1e-3
