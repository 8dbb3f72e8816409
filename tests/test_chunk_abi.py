"""Host-side checks of attention of chunks and of windows over KV pages (no GPU): sizes, and refusals before any CUDA call."""
import ctypes

import pytest

from paper_2609_38706_gb300 import _build

FAKE = 1 << 40  # never dereferenced: every case fails its host check, or has nothing to do


@pytest.fixture(scope="module")
def pk():
    _build.build()
    from paper_2609_38706_gb300 import pk as m
    m.lib()
    return m


def chunk(pk, dtype=0, R=1, n=4, qh=2, scale=1.0, window=0, sinks=0, q=(FAKE, 128, 64), out=(FAKE, 128, 64), off=FAKE, lens=FAKE,
          pages=FAKE, stride=4, scratch=FAKE, nbytes=1 << 40, lse=None, **kv):
    b, c = ctypes.byref, pk.pk_kv_cache(FAKE, 4, 16, 2, 64, 1.0, 1.0)
    for k, v in kv.items():
        setattr(c, k, v)
    return pk.lib().pk_attend_chunk(b(c), dtype, b(pk.pk_heads(*q)), b(pk.pk_heads(*out)), lse, n, off, R, qh, scale, window, sinks,
                                    lens, pages, stride, scratch, nbytes, None, None)


@pytest.mark.parametrize("change", [
    dict(dtype=2), dict(n=0x7fff0001), dict(qh=3), dict(qh=0), dict(qh=65538), dict(R=1 << 31), dict(scale=float("nan")), dict(scale=float("inf")),
    dict(scale=3e38), dict(window=1 << 31), dict(sinks=1 << 31), dict(stride=1 << 31), dict(stride=0x7fff0000 // 16 + 1),
    dict(q=(0, 128, 64)), dict(q=(FAKE + 2, 128, 64)), dict(q=(FAKE, 127, 64)), dict(q=(FAKE, 128, -64)), dict(q=(FAKE, 1 << 39, 64)),
    dict(out=(FAKE, 64, 64)), dict(out=(FAKE, 0, 64)), dict(out=(FAKE, 128, 56)), dict(out=(0, 128, 64)),
    dict(off=None), dict(off=FAKE + 4), dict(lens=None), dict(lens=FAKE + 2), dict(pages=None), dict(pages=FAKE + 1),
    dict(scratch=None), dict(scratch=FAKE + 16), dict(nbytes=16), dict(lse=FAKE + 1),
    dict(pool_dev=0), dict(n_slots=0), dict(page_tokens=24), dict(head_dim=80), dict(k_scale=0.0), dict(v_scale=float("inf"))])
def test_chunk_refused(pk, change):
    assert chunk(pk, **change) == pk.PK_ERR_ARG


def test_nothing_to_do(pk):
    assert chunk(pk, R=0, off=None, lens=None, pages=None, scratch=None, nbytes=0) == pk.PK_OK
    assert chunk(pk, n=0, q=(0, 0, 0), out=(0, 0, 0)) == pk.PK_OK


def test_chunk_scratch(pk):
    import torch
    kv = pk.pk_kv_cache(FAKE, 1 << 20, 256, 8, 128, 1.0, 1.0)
    size = lambda n, R, stride, w=0, s=0: pk.pk_attend_chunk_scratch_bytes(kv, torch.float16, n, R, 32, stride, w, s)  # noqa: E731
    assert 0 < size(1, 1, 1) < size(16, 1, 512) < 1 << 27        # pieces of at most as many units as there are blocks
    assert size(1 << 20, 4, 512) == size(1 << 10, 4, 512)
    assert size(16, 1, 512, 128, 4) < size(16, 1, 512)           # a window is four tiles
    assert size(16, 1, 512, 512 * 256, 4) == size(16, 1, 512)    # one that no request outgrows is none
    one = pk.pk_kv_cache(FAKE, 4, 16, 1, 64, 1.0, 1.0)
    assert pk.pk_attend_chunk_scratch_bytes(one, torch.float16, 1, 1, 1, 1, 0, 0) < 4096  # one block: nothing is cut
    assert all(x % 16 == 0 for x in (size(16, 1, 512), size(16, 40, 512)))
    halves = [pk.pk_attend_chunk_scratch_bytes(kv, torch.bfloat16, 100, 1, 32, n, 0, 0) - size(100, 1, n) for n in (2, 512)]
    assert halves[0] == 0 and halves[1] >= 100 * 32 * (256 + 4)  # of queries in bfloat16, where the call is long enough
    assert pk.pk_attend_chunk_scratch_bytes(kv, torch.float32, 100, 1, 32, 2, 0, 0) == 0
    for bad in ((1 << 31, 1, 4, 0, 0), (4, 1, 4, 1 << 31, 0)):
        try:
            assert size(*bad) == 0
        except pk.PKError:
            pass


def windowed(pk, **kw):
    a = dict(dtype=0, R=1, n_q=1, qh=2, scale=1.0, window=5, sinks=1, lens=FAKE, pages=FAKE, stride=4, scratch=FAKE, nbytes=1 << 30, w=None)
    a.update(kw)
    b, c, h = ctypes.byref, pk.pk_kv_cache(FAKE, 4, 16, 2, 64, 1.0, 1.0), pk.pk_heads(FAKE, 128, 64)
    return pk.lib().pk_attend_cache_window(b(c), a["dtype"], b(h), b(h), None, a["R"], a["n_q"], a["qh"], a["scale"], a["window"],
                                           a["sinks"], a["lens"], a["pages"], a["stride"], a["w"], a["scratch"], a["nbytes"], None, None)


def test_window_refused(pk):
    for change in (dict(dtype=2), dict(n_q=0), dict(qh=3), dict(scale=float("inf")), dict(window=1 << 31), dict(sinks=1 << 31),
                   dict(lens=None), dict(pages=None), dict(lens=FAKE + 2), dict(stride=1 << 31), dict(scratch=FAKE + 4),
                   dict(w=FAKE + 1), dict(w=FAKE, nbytes=8), dict(w=FAKE, scratch=None)):
        assert windowed(pk, **change) == pk.PK_ERR_ARG, change
    assert windowed(pk, R=0, lens=None) == pk.PK_OK


def test_window_scratch(pk):
    kv = pk.pk_kv_cache(FAKE, 1 << 20, 16, 8, 128, 1.0, 1.0)
    size = lambda w, s: pk.pk_attend_cache_window_scratch_bytes(kv, 4, 1, 32, 8192, True, w, s)  # noqa: E731
    whole = pk.pk_attend_cache_scratch_bytes(kv, 4, 1, 32, 8192, True)
    assert size(0, 0) == whole == size(8192 * 16, 7) and 0 < size(100, 4) < size(10000, 4) < whole
    assert pk.pk_attend_cache_window_scratch_bytes(kv, 4, 1, 31, 8192, True, 5, 0) == 0
