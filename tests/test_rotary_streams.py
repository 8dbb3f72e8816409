"""Which stream a rotation's table is kept for (no GPU): one that is dropped right after its call must not be given out again
before the kernel has read it, whichever stream that runs on."""
import types

import pytest
import torch

from paper_2609_38706_gb300 import service


class Table:
    device = torch.device("cpu")
    is_cuda = True

    def __init__(self):
        self.kept = []

    def record_stream(self, stream):
        self.kept.append(stream)


@pytest.fixture
def run(monkeypatch):
    """Calls rotate as if on `current`, of a table made on `made`; returns the streams that the table was kept for."""
    def call(made, current, stream=None):
        monkeypatch.setattr(service.pk, "pk_rotate", lambda *a: None)
        monkeypatch.setattr(service.pk, "_stream_of", lambda s, t: current if s is None else s)
        monkeypatch.setattr(service, "_stream", lambda s: s)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current)
        rotary = types.SimpleNamespace(head_dim=64, turns=Table(), table=None, made_on=made)
        x = torch.zeros((1, 1, 64))
        service.rotate(x, x, None, None, rotary, out=(x, x), stream=stream)
        return rotary.turns.kept
    return call


def test_under_another_current_stream(run):
    assert run(made=0, current=7) == [7]


def test_on_a_stream_that_is_given(run):
    assert run(made=0, current=0, stream=7) == [7]
    assert run(made=7, current=0, stream=9) == [9]


def test_on_its_own_stream(run):
    """The allocator orders that by itself."""
    assert run(made=7, current=7) == []
