"""GPU tests of a pool and a key table that belong to a side stream: what they fill and clear at construction, and their
status word, are ordered with their own calls, without a wait by the caller."""
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


def busy():
    """Some milliseconds of work on the current stream."""
    x = torch.ones(1 << 28, device="cuda")
    for _ in range(40):
        x.mul_(1.0000001)
    return x


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def test_pages_written_at_once_survive_the_zero_fill():
    """The current stream is busy when the pool is made: its zero fill must not come behind the first write."""
    from paper_2609_38706_gb300.service import KVPages
    C, H, D, n = 16, 8, 128, 4096
    k = torch.randn((n, H, D), device="cuda").to(torch.bfloat16)
    args = dev(np.array([0, n])), dev(np.zeros(1, np.int32)), dev(np.arange(n // C, dtype=np.int32)[None])
    plain = KVPages(n // C, C, H, D)
    plain.write(k, k, *args)
    plain.check()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    keep = busy()
    kv = KVPages(n // C, C, H, D, stream=side)
    kv.write(k, k, *args)
    torch.cuda.synchronize()
    assert torch.equal(kv.pool, plain.pool)
    kv.check()
    del keep


def test_an_error_on_the_side_stream_is_seen_at_once():
    from paper_2609_38706_gb300 import pk
    from paper_2609_38706_gb300.service import KVPages
    C, H, D = 16, 8, 128
    side = torch.cuda.Stream()
    kv = KVPages(4, C, H, D, stream=side)
    k = torch.randn((16, H, D), device="cuda").to(torch.bfloat16)
    args = dev(np.array([0, 16])), dev(np.zeros(1, np.int32)), dev(np.array([[99]], np.int32))
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        keep = busy()  # the failing call starts only behind this
    kv.write(k, k, *args)
    with pytest.raises(pk.PKError):
        kv.check()
    kv.check()  # and it was cleared
    torch.cuda.synchronize()
    assert kv.take_status() == 0
    del keep


def test_a_key_tables_error_on_its_stream_is_seen_at_once():
    from paper_2609_38706_gb300 import pk
    from paper_2609_38706_gb300.service import KeyTable
    side = torch.cuda.Stream()
    kt = KeyTable(16, 10, stream=side)
    tokens, off = dev(np.arange(64, dtype=np.int32)), dev(np.array([0, 64]))
    desc = dev(np.array([7], np.int32))  # there is one descriptor: out of range
    digests = torch.zeros((1, 32), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    kt.derive(tokens, off, torch.zeros_like(desc), digests)  # loads the kernels
    torch.cuda.synchronize()
    kt.check()
    with torch.cuda.stream(side):
        keep = busy()
    kt.derive(tokens, off, desc, digests)
    with pytest.raises(pk.PKError):
        kt.check()
    torch.cuda.synchronize()
    assert kt.take_status() == 0
    kt.close()
    del keep
