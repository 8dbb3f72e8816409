"""GPU tests of attention over pages whose table names a slot that the pool does not have: the request gets NaN, never
another request's state, its pages' weights stay, and the other requests are answered."""
import numpy as np
import pytest
import torch

from test_gpu_attend_cache import cache, dev, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g
    g.build()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("slot", [-1, 0x7FFFFFFF, "count"])
@pytest.mark.parametrize("lens,n_q,C,H,G,D,at", [
    ([40, 40, 33], 1, 16, 2, 4, 128, 1),        # one CTA a request and head
    ([70, 70, 70], 4, 16, 1, 3, 64, 4),         # the last page: only the last queries attend its tokens
    ([3000, 2900, 10], 1, 16, 1, 2, 128, 150),  # splits
    ([900, 5000, 64], 2, 256, 2, 8, 64, 0),     # splits, two column tiles
])
@pytest.mark.parametrize("weigh", [False, True])
def test_a_slot_out_of_range_gives_nan_and_nothing_else(slot, lens, n_q, C, H, G, D, at, weigh):
    from paper_2609_38706_gb300 import pk
    pool, pages, rng = make(lens, C, H, D, 51)
    kv = cache(pool, C, H, D)
    q = torch.from_numpy(rng.standard_normal((len(lens), n_q, H * G, D))).to(torch.bfloat16).cuda()
    n = dev(np.array(lens, np.int32))
    w0 = torch.from_numpy(rng.uniform(0, 2, pages.shape).astype(np.float32)).cuda()
    w = w0.clone() if weigh else None
    want, want_lse = kv.attend(q, n, dev(pages), weight=w)
    kv.check()
    bad = pages.copy()
    bad[1, at] = pool.shape[0] if slot == "count" else slot
    got_w = w0.clone() if weigh else None
    out, lse = kv.attend(q, n, dev(bad), weight=got_w)
    assert kv.take_status() == pk.PK_ERR_ARG
    others = [0, 2]
    assert torch.equal(out[others], want[others]) and torch.equal(lse[others], want_lse[others])
    assert torch.isnan(out[1]).all() and torch.isnan(lse[1]).all()
    if weigh:
        assert torch.equal(got_w[others], w[others]) and torch.equal(got_w[1], w0[1])


def test_a_slot_out_of_range_past_the_length_does_not_matter():
    pool, pages, rng = make([40, 20], 16, 2, 64, 52, stride=9)
    kv = cache(pool, 16, 2, 64)
    q = torch.from_numpy(rng.standard_normal((2, 1, 4, 64))).to(torch.float16).cuda()
    n = dev(np.array([40, 20], np.int32))
    want = kv.attend(q, n, dev(pages))
    pages[0, 3:], pages[1, 2:] = -1, 0x7FFFFFFF
    got = kv.attend(q, n, dev(pages))
    kv.check()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
