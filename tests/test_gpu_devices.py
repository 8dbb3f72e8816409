"""GPU tests of calls whose tensors are not on the current device, where their kernels would be launched: refused before any
launch.  One GPU is enough: the current device is said to be another one."""
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


@pytest.fixture
def elsewhere(monkeypatch):
    """Calls made behind this see device 1 as the current one."""
    from paper_2609_38706_gb300 import pk

    def go():
        monkeypatch.setattr(pk, "_current_device", lambda: 1, raising=False)
    return go


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def test_page_calls(elsewhere):
    from paper_2609_38706_gb300 import pk, service
    kv = service.KVPages(4, 16, 2, 64)
    k = torch.zeros((16, 2, 64), dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((1, 1, 4, 64), dtype=torch.bfloat16, device="cuda")
    off, start, pages, n = dev(np.array([0, 16])), dev(np.zeros(1, np.int32)), dev(np.zeros((1, 1), np.int32)), dev(np.array([16], np.int32))
    weight = torch.zeros((1, 1), device="cuda")
    calls = [lambda: kv.write(k, k, off, start, pages), lambda: kv.read(off, start, pages, 16),
             lambda: kv.attend(q, n, pages, weight=weight), lambda: service.attend_prompt(k, k, k, off, off),
             lambda: service.evict_pages(pages, weight, n, 16, 2, 0, 1)]
    for call in calls:
        call()
    kv.check()
    elsewhere()
    for call in calls:
        with pytest.raises(pk.PKError):
            call()


def test_a_pool_on_another_device():
    """The tensors are on the current device, the pool is not."""
    from paper_2609_38706_gb300 import pk, service
    kv = service.KVPages(4, 16, 2, 64)
    assert kv.kv.device == kv.device.index
    kv.kv.device = 1
    k = torch.zeros((16, 2, 64), dtype=torch.bfloat16, device="cuda")
    off, start, pages = dev(np.array([0, 16])), dev(np.zeros(1, np.int32)), dev(np.zeros((1, 1), np.int32))
    for call in (lambda: kv.write(k, k, off, start, pages), lambda: kv.read(off, start, pages, 16),
                 lambda: kv.attend(k.view(1, 16, 2, 64), start, pages)):
        with pytest.raises(pk.PKError):
            call()


def test_table_calls(elsewhere):
    from paper_2609_38706_gb300 import pk, service
    kt = service.KeyTable(16, 10)
    d = kt.digests([{"model_id": "m", "weight_precision": "bf16", "weight_version": "1", "kv_format": "fp16"}])
    tokens, off, idx = dev(np.arange(64, dtype=np.int32)), dev(np.array([0, 64])), dev(np.zeros(1, np.int32))
    key_off, keys = kt.derive(tokens, off, idx, d)
    slots = dev(np.arange(4, dtype=np.int32))
    saved = kt.save(torch.zeros(kt.table.numel() + 64, dtype=torch.uint8, device="cuda"))
    calls = [lambda: kt.derive(tokens, off, idx, d), lambda: kt.lookup(keys, key_off), lambda: kt.store(keys, slots),
             lambda: kt.lookup_store(keys, key_off, slots), lambda: kt.load(saved),
             lambda: pk.pk_init(kt.table, 16, 10)]
    for call in calls[:-1]:
        call()
    kt.check()
    on_host = torch.zeros(saved.numel(), dtype=torch.uint8)
    elsewhere()
    for call in calls:
        with pytest.raises(pk.PKError):
            call()
    kt.save(on_host)  # a copy may go anywhere
    torch.cuda.synchronize()
    assert torch.equal(on_host, saved.cpu())
    kt.close()
