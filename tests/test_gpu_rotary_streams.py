"""GPU test of a rotation's table that is dropped while a call of another stream may still read it."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g
    g.build()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("given", [False, True])
def test_a_dropped_table_is_not_given_out_again_too_early(given):
    from paper_2609_38706_gb300 import service
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    q, k = (torch.randn((50, h, 64), device="cuda").to(torch.bfloat16) for h in (4, 2))
    args = dev(np.array([0, 50])), dev(np.array([7], np.int32))
    want = service.rotate(q, k, *args, service.Rotary(64))
    side = torch.cuda.Stream()
    work = torch.ones(1 << 28, device="cuda")
    torch.cuda.synchronize()
    rotary = service.Rotary(64)
    table = rotary.turns.data_ptr()
    with torch.cuda.stream(side):
        for _ in range(40):  # some milliseconds, behind which the call waits
            work.mul_(1.0000001)
        if not given:
            got = service.rotate(q, k, *args, rotary)
    if given:
        got = service.rotate(q, k, *args, rotary, stream=side)
    del rotary
    others = [torch.full((32,), -1, dtype=torch.int64, device="cuda") for _ in range(64)]
    assert table not in [t.data_ptr() for t in others]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
