"""GPU tests of eviction by accumulated attention weight: every output equals the plain rule's."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
NO = -1


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g
    g.build()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def plain(pages, w, kv_len, C, budget, sinks, recent):
    R, stride = pages.shape
    po, wo = np.full((R, budget), NO, np.int32), np.zeros((R, budget), np.float32)
    ev, lo = np.full((R, stride), NO, np.int32), np.zeros(R, np.int32)
    for r in range(R):
        n = -(-int(kv_len[r]) // C)
        if n <= budget:
            keep = list(range(n))
        else:
            mid = range(sinks, n - recent)
            key = lambda j: (-np.inf if np.isnan(w[r, j]) else w[r, j])
            # NaN below every weight, -inf included
            best = sorted(mid, key=lambda j: (np.isnan(w[r, j]), -key(j), j))[: budget - sinks - recent]
            keep = sorted([*range(sinks), *best, *range(n - recent, n)])
        gone = sorted(set(range(n)) - set(keep))
        po[r, : len(keep)], wo[r, : len(keep)], ev[r, : len(gone)] = pages[r, keep], w[r, keep], pages[r, gone]
        lo[r] = kv_len[r] - len(gone) * C
    return po, wo, lo, ev


def run(pages, w, kv_len, C, budget, sinks, recent, status=None):
    from paper_2609_38706_gb300 import service
    d = [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (pages, w, kv_len)]
    out = service.evict_pages(*d, C, budget, sinks, recent, status)
    return [x.cpu().numpy() for x in out]


def weights(kind, shape, rng):
    if kind == "spread":
        return np.exp(4 * rng.standard_normal(shape)).astype(np.float32)
    if kind == "equal":
        return np.full(shape, 0.25, np.float32)
    if kind == "few values":
        return rng.choice(np.array([0.0, -0.0, 1.0, 1.0000001, -2.0], np.float32), shape)
    w = rng.standard_normal(shape).astype(np.float32)
    w[rng.random(shape) < 0.2] = np.nan
    w[rng.random(shape) < 0.1] = np.inf
    w[rng.random(shape) < 0.1] = -np.inf
    return w


@pytest.mark.parametrize("kind", ["spread", "equal", "few values", "odd"])
@pytest.mark.parametrize("R,stride,C,budget,sinks,recent", [
    (1, 1, 16, 1, 0, 1), (3, 5, 16, 3, 1, 1), (7, 33, 48, 8, 0, 8), (5, 300, 16, 100, 4, 17), (4, 1024, 16, 1023, 1, 1),
    (6, 1025, 256, 512, 4, 32), (3, 5000, 16, 700, 0, 1), (2, 9001, 16, 9000, 3, 5), (3, 70, 16, 90, 2, 3),
    (2, 40000, 16, 20001, 4, 64), (3, 4096, 16, 1000, 1, 7), (3, 4097, 16, 4000, 0, 1), (2, 8192, 32, 4, 2, 2),
    (2, 8193, 16, 77, 1, 1), (5, 1024, 16, 6, 3, 3),
])
def test_matches_the_rule(kind, R, stride, C, budget, sinks, recent):
    rng = np.random.default_rng(31)
    w = weights(kind, (R, stride), rng)
    pages = rng.integers(0, 1 << 31, (R, stride)).astype(np.int32)
    kv_len = rng.integers(0, stride * C + 1, R).astype(np.int32)
    kv_len[0] = stride * C
    for a, b in zip(run(pages, w, kv_len, C, budget, sinks, recent), plain(pages, w, kv_len, C, budget, sinks, recent)):
        assert np.array_equal(a, b, equal_nan=a.dtype.kind == "f")


def test_empty_and_short_requests():
    rng = np.random.default_rng(32)
    pages, w = rng.integers(0, 99, (4, 6)).astype(np.int32), rng.random((4, 6)).astype(np.float32)
    kv_len = np.array([0, 1, 16, 96], np.int32)
    for a, b in zip(run(pages, w, kv_len, 16, 4, 1, 1), plain(pages, w, kv_len, 16, 4, 1, 1)):
        assert np.array_equal(a, b)


def test_bad_length_is_reported():
    from paper_2609_38706_gb300 import pk
    rng = np.random.default_rng(33)
    pages, w = rng.integers(0, 99, (3, 6)).astype(np.int32), rng.random((3, 6)).astype(np.float32)
    for n in (-1, 97):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        po, wo, lo, ev = run(pages, w, np.array([96, n, 96], np.int32), 16, 4, 1, 1, status)
        assert int(status.item()) == pk.PK_ERR_ARG
        assert np.all(po[1] == NO) and lo[1] == 0 and np.all(ev[1] == NO)
        want = plain(pages[[0, 2]], w[[0, 2]], np.array([96, 96], np.int32), 16, 4, 1, 1)
        assert np.array_equal(po[[0, 2]], want[0]) and np.array_equal(ev[[0, 2]], want[3])


def test_refusals():
    from paper_2609_38706_gb300 import pk, service
    p = torch.zeros((2, 8), dtype=torch.int32, device="cuda")
    w, n = torch.zeros((2, 8), device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    for C, budget, sinks, recent in ((0, 4, 1, 1), (16, 4, 1, 0), (16, 4, 2, 3), (16, 0, 0, 1), (16, 4, -1, 1), (16, -4, 0, 1)):
        with pytest.raises(pk.PKError):
            service.evict_pages(p, w, n, C, budget, sinks, recent)
    for a in ((p.long(), w, n), (p, w.double(), n), (p, w[:, :4], n), (p, w, n.long()), (p[0], w, n)):
        with pytest.raises(pk.PKError):
            service.evict_pages(*a, 16, 4, 1, 1)
