"""Host-side checks of the KV-page calls (no GPU): sizes, and refusals before any CUDA call."""
import ctypes

import numpy as np
import pytest

import kv_ref as R
from paper_2609_38706_gb300 import _build

FAKE = 1 << 40  # never dereferenced: every case fails its host check, or has nothing to do


@pytest.fixture(scope="module")
def pk():
    _build.build()
    from paper_2609_38706_gb300 import pk as m
    m.lib()
    return m


def test_page_bytes(pk):
    assert pk.pk_kv_page_bytes(16, 8, 128) == 8 * 2304 and pk.pk_kv_page_bytes(256, 1, 64) == 16 * 1152
    assert pk.pk_kv_page_bytes(48, 3, 128) == R.page_bytes(48, 3, 128)
    for bad in ((0, 8, 128), (8, 8, 128), (24, 8, 128), (32784, 1, 64), (16, 0, 128), (16, 1025, 128), (16, 8, 96)):
        assert pk.pk_kv_page_bytes(*bad) == 0


def test_reference_quantiser_ties_and_tables():
    """The tests' own reference: e4m3 and e2m1 values, ties to even."""
    assert R.E4M3[0x7E] == 448 and R.E4M3[1] == 2.0 ** -9 and np.isnan(R.E4M3[0x7F])
    y = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0])
    assert R.E2M1[R.nearest_even(y, R.E2M1[:8])].tolist() == [0, 1, 1, 2, 2, 4, 4, 6]


def good(pk):
    return pk.pk_kv_cache(FAKE, 4, 16, 2, 64, 1.0, 1.0), pk.pk_heads(FAKE, 128, 64)


@pytest.mark.parametrize("change", [dict(pool_dev=0), dict(pool_dev=FAKE + 8), dict(n_slots=0), dict(n_slots=1 << 32),
                                    dict(page_tokens=17), dict(kv_heads=0), dict(head_dim=80), dict(k_scale=0.0),
                                    dict(v_scale=float("nan")), dict(k_scale=float("inf")), dict(v_scale=-1.0)])
def test_bad_cache_refused_everywhere(pk, change):
    kv, h = good(pk)
    for k, v in change.items():
        setattr(kv, k, v)
    L, b = pk.lib(), ctypes.byref
    for fn in (L.pk_kv_write, L.pk_kv_read):
        assert fn(b(kv), 0, b(h), b(h), 4, FAKE, FAKE, 1, FAKE, 1, None, None) == pk.PK_ERR_ARG
    assert L.pk_attend_cache(b(kv), 0, b(h), b(h), None, 1, 1, 2, 1.0, FAKE, FAKE, 1, None, FAKE, 1 << 30, None,
                             None) == pk.PK_ERR_ARG


@pytest.mark.parametrize("h", [(0, 128, 64), (FAKE + 2, 128, 64), (FAKE, 127, 64), (FAKE, 128, 60), (FAKE, -128, 64),
                               (FAKE, 128, -64), (FAKE, 1 << 60, 64)])  # and, for prompts, what a tensor map does not take
def test_bad_strides_refused(pk, h):
    kv, ok = good(pk)
    bad = pk.pk_heads(*h)
    L, b = pk.lib(), ctypes.byref
    assert L.pk_kv_write(b(kv), 0, b(bad), b(ok), 4, FAKE, FAKE, 1, FAKE, 1, None, None) == pk.PK_ERR_ARG
    assert L.pk_kv_write(b(kv), 0, b(ok), b(bad), 4, FAKE, FAKE, 1, FAKE, 1, None, None) == pk.PK_ERR_ARG
    for i in range(4):
        hs = [b(bad) if j == i else b(ok) for j in range(4)]
        assert L.pk_attend_prompt(0, *hs, None, 4, 4, FAKE, FAKE, 1, 2, 2, 64, 1.0, FAKE, 1 << 20, None,
                                  None) == pk.PK_ERR_ARG


def test_outputs_that_overlap_themselves_refused(pk):
    kv, ok = good(pk)
    L, b = pk.lib(), ctypes.byref
    for h in ((FAKE, 0, 64), (FAKE, 128, 0), (FAKE, 56, 64)):
        bad = pk.pk_heads(*h)
        assert L.pk_kv_read(b(kv), 0, b(bad), b(ok), 4, FAKE, FAKE, 1, FAKE, 1, None, None) == pk.PK_ERR_ARG
        assert L.pk_attend_prompt(0, b(ok), b(ok), b(ok), b(bad), None, 4, 4, FAKE, FAKE, 1, 2, 2, 64, 1.0, FAKE,
                                  1 << 20, None, None) == pk.PK_ERR_ARG


def test_attention_arguments_refused(pk):
    kv, h = good(pk)
    L, b = pk.lib(), ctypes.byref

    def prompt(dtype=0, R=1, qh=2, kh=2, D=64, scale=1.0, scratch=FAKE, nbytes=1 << 20, off=FAKE, n_q=4):
        return L.pk_attend_prompt(dtype, b(h), b(h), b(h), b(h), None, n_q, 4, off, off, R, qh, kh, D, scale, scratch,
                                  nbytes, None, None)

    far = pk.pk_heads(FAKE, 1 << 39, 64)
    assert L.pk_attend_prompt(0, b(far), b(h), b(h), b(h), None, 4, 4, FAKE, FAKE, 1, 2, 2, 64, 1.0, FAKE, 1 << 20, None,
                              None) == pk.PK_ERR_ARG
    for kw in (dict(dtype=2), dict(qh=3), dict(kh=0), dict(qh=0), dict(D=96), dict(scale=float("nan")), dict(scratch=None),
               dict(scratch=FAKE + 8), dict(nbytes=8), dict(off=None), dict(off=FAKE + 4), dict(n_q=1 << 31)):
        assert prompt(**kw) == pk.PK_ERR_ARG, kw
    assert prompt(R=0, off=None, scratch=None, nbytes=0) == pk.PK_OK and prompt(n_q=0) == pk.PK_OK

    def cached(dtype=0, R=1, n_q=1, qh=2, scale=1.0, lens=FAKE, pages=FAKE, stride=4, scratch=FAKE, nbytes=1 << 30, w=None):
        return L.pk_attend_cache(b(kv), dtype, b(h), b(h), None, R, n_q, qh, scale, lens, pages, stride, w, scratch,
                                 nbytes, None, None)

    for kw in (dict(dtype=2), dict(n_q=0), dict(qh=3), dict(qh=0), dict(scale=float("inf")), dict(lens=None),
               dict(pages=None), dict(lens=FAKE + 2), dict(stride=1 << 31), dict(scratch=FAKE + 4), dict(w=FAKE + 1),
               dict(w=FAKE, nbytes=8), dict(w=FAKE, scratch=None)):
        assert cached(**kw) == pk.PK_ERR_ARG, kw
    assert cached(R=0, lens=None) == pk.PK_OK
    assert pk.pk_attend_cache_scratch_bytes(kv, 1, 1, 3, 4, False) == 0
    small = pk.pk_attend_cache_scratch_bytes(kv, 2, 1, 2, 4, False)
    assert pk.pk_attend_cache_scratch_bytes(kv, 2, 1, 2, 4, True) > small


def test_evict_arguments_refused(pk):
    L = pk.lib()

    def evict(R=1, stride=8, C=16, budget=4, sinks=1, recent=1, ptrs=(FAKE,) * 7):
        p = ptrs
        return L.pk_evict_pages(p[0], p[1], p[2], R, stride, C, budget, sinks, recent, p[3], p[4], p[5], p[6], None, None)

    for kw in (dict(C=0), dict(recent=0), dict(sinks=4), dict(budget=0), dict(budget=1 << 31), dict(stride=1 << 31),
               dict(sinks=0xFFFFFFFF)):
        assert evict(**kw) == pk.PK_ERR_ARG, kw
    for i in range(6):
        assert evict(ptrs=tuple(None if j == i else FAKE for j in range(7))) == pk.PK_ERR_ARG
        assert evict(ptrs=tuple(FAKE + 2 if j == i else FAKE for j in range(7))) == pk.PK_ERR_ARG
    assert evict(R=0, ptrs=(None,) * 7) == pk.PK_OK
