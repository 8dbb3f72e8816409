"""GPU tests of a key table on a side stream while either stream is busy: buffers that a call fills or uploads are ordered
with its kernels and are not given out again before these have run."""
import numpy as np
import pytest
import torch

from test_gpu_kv_streams import busy

pytestmark = pytest.mark.gpu
C, R = 16, 64
DESCRIPTORS = [{"model_id": f"m{i}", "weight_precision": "bf16", "weight_version": "1", "kv_format": "fp16"} for i in range(3)]


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g
    g.build()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def batch(seed):
    rng = np.random.default_rng(seed)
    off = np.arange(R + 1, dtype=np.int64) * 8 * C
    return rng.integers(0, 1000, off[-1]).astype(np.int32), off, np.zeros(R, np.uint32)


@pytest.fixture
def tables():
    from paper_2609_38706_gb300.service import KeyTable
    side = torch.cuda.Stream()
    plain, other = KeyTable(C, 14), KeyTable(C, 14, stream=side)
    d = plain.digests(DESCRIPTORS)
    for kt in (plain, other):  # loads the kernels
        kt.derive_enc(*batch(0), DESCRIPTORS)
        kt.derive(*batch(0), kt.digests(DESCRIPTORS))
    torch.cuda.synchronize()
    yield plain, other, side, d
    torch.cuda.synchronize()
    plain.close(), other.close()


def test_digests_survive_their_zero_fill(tables):
    """The current stream is busy when the digests' buffer is made."""
    plain, other, side, want = tables
    torch.cuda.synchronize()
    keep = busy()
    got = other.digests(DESCRIPTORS)
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    other.check()
    del keep


@pytest.mark.parametrize("enc", [False, True])
def test_uploads_are_kept_until_their_kernels_have_run(tables, enc):
    """Three calls with host arrays while the side stream is busy: each gets the keys of its own tokens."""
    plain, other, side, d = tables
    batches = [batch(s) for s in (1, 2, 3)]
    want = [plain.derive(*b, d)[1].clone() for b in batches]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        keep = busy()
    got = [other.derive_enc(*b, DESCRIPTORS)[2] if enc else other.derive(*b, d)[1] for b in batches]
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    other.check(), plain.check()
    del keep


def test_lookup_and_store_with_host_slots(tables):
    """Slots uploaded for two stores in a row while the side stream is busy."""
    plain, other, side, d = tables
    off, keys = plain.derive(*batch(5), d)
    torch.cuda.synchronize()
    n = keys.shape[0]
    with torch.cuda.stream(side):
        keep = busy()
    first = other.lookup_store(keys, off, np.arange(n, dtype=np.uint32))
    again = other.lookup_store(keys, off, np.arange(n, dtype=np.uint32) + 7)
    torch.cuda.synchronize()
    assert torch.equal(first[3].cpu(), torch.arange(n, dtype=torch.int32)) and int(first[0].sum()) == 0
    assert torch.equal(again[1].cpu(), torch.arange(n, dtype=torch.int32))
    other.check()
    del keep
