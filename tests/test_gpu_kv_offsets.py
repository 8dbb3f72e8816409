"""GPU test of the page store with offsets at the ends of their type and out of order: reported, and no token of theirs is
written or read."""
import numpy as np
import pytest
import torch

from test_gpu_kv_store import dev, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g
    g.build()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("R", [1, 2, 33, 70])
@pytest.mark.parametrize("value", [-(1 << 63), -(1 << 63) + 1, -1, (1 << 63) - 1])
@pytest.mark.parametrize("where", ["last", "all", "first"])
def test_offsets_at_the_ends_of_their_type(R, value, where):
    from paper_2609_38706_gb300 import pk
    kv, pages, off, x = make([3] * R, [0] * R, 16, 2, 64, "bf16", 8)
    off = off.copy()
    off[{"last": slice(R, None), "all": slice(None), "first": slice(0, 1)}[where]] = value
    before = kv.pool.cpu().numpy()
    args = dev(off), dev(np.zeros(R, np.int32)), dev(pages)
    kv.write(x[0].cuda(), x[1].cuda(), *args)
    assert kv.take_status() == pk.PK_ERR_ARG
    # requests whose own offsets are in order may have been written, nobody else's page was
    bad = [r for r in range(R) if not 0 <= off[r] <= off[r + 1] <= x.shape[1]]
    assert bad
    keep = sorted(set(range(kv.pool.shape[0])) - set(pages[[r for r in range(R) if r not in bad]].reshape(-1).tolist()))
    assert np.array_equal(kv.pool.cpu().numpy()[keep], before[keep])
    k, v = torch.full_like(x[0], 7.0).cuda(), torch.full_like(x[1], 7.0).cuda()
    pk.pk_kv_read(kv.kv, k, v, *args, kv.status)
    assert kv.take_status() == pk.PK_ERR_ARG
    if where == "all":
        assert torch.all(k == 7.0) and torch.all(v == 7.0)
