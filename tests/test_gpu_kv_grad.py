"""GPU test that a tensor whose gradient is asked for is refused by the KV-page calls, which have no backward pass, instead of
answered without a graph."""
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


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def test_tensors_that_ask_for_a_gradient():
    from paper_2609_38706_gb300 import pk, service
    kv = service.KVPages(4, 16, 2, 64)
    x = torch.randn((16, 2, 64), device="cuda").to(torch.bfloat16)
    g = x.clone().requires_grad_()
    off, start, pages, n = dev(np.array([0, 16])), dev(np.zeros(1, np.int32)), dev(np.zeros((1, 1), np.int32)), dev(np.array([16], np.int32))
    calls = [lambda a, b, c: kv.write(a, b, off, start, pages), lambda a, b, c: kv.attend(a.view(1, 16, 2, 64), n, pages),
             lambda a, b, c: kv.attend_prompt(a, b, c, off, off)]
    for call, takes in zip(calls, (2, 1, 3)):
        for i in range(takes):
            args = [g if j == i else x for j in range(3)]
            with pytest.raises(pk.PKError, match="gradient"):
                call(*args)
            with torch.no_grad():
                call(*args)
            call(*(a.detach() for a in args))
    kv.check()
