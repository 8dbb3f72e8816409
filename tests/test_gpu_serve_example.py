"""GPU test of the example that runs keys, pages, attention and eviction together: what it hits, what it keeps, and that
a prompt served from a hit answers as it did when it was computed."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g
    g.build()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def test_example_serves_hits_and_keeps_its_budget():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import serve_from_pages as ex
    steps, budget = 24, 8
    report = ex.main(steps, budget, quiet=True)
    assert report["first"]["hit"] == [0, 0]
    # the second batch: the shared document's full chunks, all full chunks of a prompt seen before, nothing
    assert report["second"]["hit"] == [100 // ex.CHUNK, 140 // ex.CHUNK, 0]
    lens = {"first": [140, 107], "second": [160, 140, 5]}
    for name, r in report.items():
        for n, held in zip(lens[name], r["kv_len"]):
            before = n + steps
            pages = -(-before // ex.CHUNK)
            assert held == before - max(0, pages - budget) * ex.CHUNK + steps
        # a step's weights of a request sum to its query heads; evicted pages take theirs with them
        assert all(steps * ex.Q_HEADS * 0.999 < w <= 2 * steps * ex.Q_HEADS * 1.001 for w in r["weight"])
        assert all(0 <= t < ex.VOCAB for a in r["answers"] for t in a)
