"""GPU test that the serving example gives its pages back: over many batches every slot is free, private to a running request,
or led to by a key, and a slot is handed out once."""
import os
import sys

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g
    g.build()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def test_a_long_run_does_not_leak_pages():
    import serve_from_pages as ex
    rng = np.random.default_rng(5)
    slots = 90
    server = ex.Server(ex.Layer(1), slots)
    document = rng.integers(0, ex.VOCAB, 70).tolist()
    batch = [document + [3] * 20, document, document + [9] * 3, [1, 2, 3]]
    first = None
    for _ in range(6):
        report = server.serve(batch, steps=20, budget=4)
        assert not server.private
        keyed = slots - len(server.free)
        assert len(set(server.free)) == len(server.free)
        assert keyed == server.kt.entries()  # a chunk's page and no more
        if first is None:
            first = report
        else:  # served from the same pages each time
            assert report["hit"] == [90 // ex.CHUNK, 70 // ex.CHUNK, 73 // ex.CHUNK, 0]
            assert report["kv_len"] == first["kv_len"]
    # while requests run, no page is two requests' but the keyed ones
    logits, table, kv_len, hit = server.prefill(batch, room=40)
    own = [s for s in table.flatten().tolist() if s in server.private]
    assert len(own) == len(set(own)) == len(server.private) and not server.private & set(server.free)
    table, weight, kv_len = server.evict(table, torch.rand(table.shape, device="cuda"), kv_len, 3)
    rows = [[s for s in row if s >= 0] for row in table.tolist()]
    assert [len(r) for r in rows] == [3 + -(-(n + 40) // ex.CHUNK) - max(3, -(-n // ex.CHUNK)) if n > 48 else -(-(n + 40) // ex.CHUNK)
                                      for n in (90, 70, 73, 3)]
    assert server.private <= {s for r in rows for s in r} and not server.private & set(server.free)
    server.release(table)
    assert not server.private
    server.kv.check()
    server.kt.close()
