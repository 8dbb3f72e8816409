"""Host-side checks of the rotation (no GPU): its table, and refusals before any CUDA call."""
import ctypes
import math

import numpy as np
import pytest

from paper_2609_38706_gb300 import _build

FAKE = 1 << 40  # never dereferenced: every case fails its host check, or has nothing to do


@pytest.fixture(scope="module")
def pk():
    _build.build()
    from paper_2609_38706_gb300 import pk as m
    m.lib()
    return m


def frequency(i, rot, base, factor, context, low, high):
    f = base ** (-2 * i / rot)
    stays = 0.0
    if context:
        n = context * f / (2 * math.pi)
        stays = 0.0 if n <= low else 1.0 if n >= high else (n - low) / (high - low)
    return stays * f + (1 - stays) * f / factor


@pytest.mark.parametrize("rot,base,factor,context,low,high", [
    (128, 10000.0, 1.0, 0.0, 1.0, 32.0), (64, 500000.0, 8.0, 8192.0, 1.0, 4.0), (16, 1.5, 4.0, 0.0, 1.0, 32.0),
    (96, 10000.0, 40.0, 4096.0, 1.0, 32.0), (128, 1e7, 1.0, 100.0, 0.0, 1.0)])
def test_table(pk, rot, base, factor, context, low, high):
    got = pk.pk_rotary_turns(rot, base, factor, context, low, high)
    want = np.array([frequency(i, rot, base, factor, context, low, high) for i in range(rot // 2)]) / (2 * math.pi)
    # a power, three products and quotients and a sum, each off by a few units in the last place of 64 bits
    assert np.all(np.abs(got.astype(np.float64) * 2.0 ** -64 - want) <= want * 2.0 ** -48 + 2.0 ** -64)
    if context and factor > 1:  # parts: some as they were, some divided
        plain = pk.pk_rotary_turns(rot, base, 1.0, 0.0, 1.0, 32.0).astype(np.float64)
        ratio = plain / got.astype(np.float64)
        assert ratio.min() < 1 + 1e-9 and abs(ratio.max() - factor) < 1e-6 and np.all(np.diff(ratio) > -1e-9)


@pytest.mark.parametrize("args", [(0, 1e4, 1, 0, 1, 32), (24, 1e4, 1, 0, 1, 32), (144, 1e4, 1, 0, 1, 32), (64, 1.0, 1, 0, 1, 32),
                                  (64, 1e4, 0.5, 0, 1, 32), (64, 1e4, 1, -1, 1, 32), (64, 1e4, 1, 0, 32, 32),
                                  (64, 1e4, 1, 0, -1, 32), (64, float("nan"), 1, 0, 1, 32), (64, float("inf"), 1, 0, 1, 32),
                                  (64, 1e4, float("nan"), 0, 1, 32), (64, 1e4, 1, float("inf"), 1, 32),
                                  (64, 1e4, 1, 0, 1, float("inf"))])
def test_tables_refused(pk, args):
    with pytest.raises(pk.PKError):
        pk.pk_rotary_turns(*args)


def call(pk, dtype=0, q=None, k=None, qo=None, ko=None, n=4, qh=2, kh=1, D=64, rot=None, qw=None, kw=None, eps=1e-6, off=FAKE,
         start=FAKE, R=1):
    b = ctypes.byref
    h = lambda x, heads: b(pk.pk_heads(*(x or (FAKE, heads * 64, 64))))  # noqa: E731
    r = pk.pk_rotary(*(rot or (FAKE, 64, 0, 1.0)))
    return pk.lib().pk_rotate(dtype, h(q, qh), h(k, kh), h(qo, qh), h(ko, kh), n, qh, kh, D, b(r), qw, kw, eps, off, start, R,
                              None, None)


@pytest.mark.parametrize("change", [
    dict(dtype=2), dict(D=96), dict(n=1 << 32), dict(qh=65536), dict(rot=(0, 64, 0, 1.0)), dict(rot=(FAKE + 4, 64, 0, 1.0)),
    dict(rot=(FAKE, 128, 0, 1.0)), dict(rot=(FAKE, 8, 0, 1.0)), dict(rot=(FAKE, 24, 0, 1.0)), dict(rot=(FAKE, 64, 2, 1.0)),
    dict(rot=(FAKE, 64, 0, float("nan"))), dict(rot=(FAKE, 64, 0, float("inf"))), dict(qw=FAKE + 8), dict(kw=FAKE + 2),
    dict(eps=0.0), dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")), dict(eps=1e-40), dict(off=None),
    dict(start=None), dict(off=FAKE + 4), dict(start=FAKE + 2),
    dict(q=(FAKE + 2, 128, 64)), dict(k=(FAKE, 60, 64)), dict(q=(FAKE, -128, 64)), dict(qo=(FAKE, 64, 64)), dict(qo=(FAKE, 0, 64)),
    dict(ko=(0, 64, 64)), dict(ko=(FAKE, 56, 64))])
def test_refused(pk, change):
    assert call(pk, **change) == pk.PK_ERR_ARG


def test_nothing_to_do(pk):
    assert call(pk, R=0, off=None, start=None) == pk.PK_OK
    assert call(pk, n=0) == pk.PK_OK
    assert call(pk, qh=0, kh=0) == pk.PK_OK


def test_python_refusals(pk):
    from paper_2609_38706_gb300 import service
    for kw in (dict(rotary_dim=8), dict(rotary_dim=72), dict(rotary_dim=144), dict(amplitude=float("nan")),
               dict(turns=np.zeros(31, np.uint64)), dict(turns=np.zeros(64)), dict(factor=0.5), dict(base=1.0)):
        with pytest.raises(pk.PKError):
            service.Rotary(128, **{"device": "cpu", **kw})
