"""GPU test of the page store where a value divided by its block's scale passes the top of 32 bits: the code saturates on
the value's own side.  Only a block whose scale saturates (448) gets there: large values under a small tensor scale."""
import numpy as np
import pytest
import torch

import kv_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g
    g.build()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("k_scale,v_scale", [(1e-3, 2.0 ** -12), (1.9e-3, 3e-7), (2.0 ** -60, 1e-18), (1e-20, 1.0), (1e-25, 3.0)])
def test_quotients_past_the_top_keep_their_sign(D, k_scale, v_scale):
    from paper_2609_38706_gb300.service import KVPages
    C, H, n = 16, 2, 32
    rng = np.random.default_rng(41)
    # magnitudes over the type's whole range, both signs, in one block and alone; whole blocks alike as well
    x = rng.standard_normal((2, n, H, D)) * 2.0 ** rng.uniform(-126, 126, (2, n, H, D))
    x[:, :8] = rng.choice((1.6e38, -1.6e38, 3.38e38, -3.38e38, 1e30, -1e30, 1.0, -0.0), (2, 8, H, D))
    x[:, 8:12] = rng.standard_normal((2, 4, H, D)) * 2.0 ** rng.integers(100, 126, (2, 4, H, 1))
    x = torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16)
    assert torch.isfinite(x).all()
    kv = KVPages(2, C, H, D, k_scale, v_scale)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    kv.write(x[0].cuda(), x[1].cuda(), dev(np.array([0, n])), dev(np.zeros(1, np.int32)),
             dev(np.array([[1, 0]], np.int32)))
    kv.check()
    want = np.zeros((2, R.page_bytes(C, H, D)), np.uint8)
    (kc, ks), (vc, vs) = (R.quantise(x[j].float().numpy(), g) for j, g in ((0, k_scale), (1, v_scale)))
    for i in range(n):
        for h in range(H):
            R.put_token(want, 1 - i // C, i % C, h, C, H, D, kc[i, h], ks[i, h], vc[i, h], vs[i, h])
    assert np.array_equal(kv.pool.cpu().numpy(), want)
