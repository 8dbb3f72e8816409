"""Host-side checks (no GPU): calls that need more blocks than a launch takes are refused ahead of any launch."""
import ctypes

import pytest

from paper_2609_38706_gb300 import _build

FAKE = 1 << 40  # never dereferenced: refused before any CUDA call


@pytest.fixture(scope="module")
def pk():
    _build.build()
    from paper_2609_38706_gb300 import pk as m
    m.lib()
    return m


def test_prompts_of_more_items_than_a_launch_has_blocks(pk):
    h = pk.pk_heads(FAKE, 128, 64)
    L, b = pk.lib(), ctypes.byref
    call = lambda n_q, R, qh, kh: L.pk_attend_prompt(0, b(h), b(h), b(h), b(h), None, n_q, 4, FAKE, FAKE, R, qh, kh, 64, 1.0,
                                                     FAKE, 1 << 40, None, None)
    assert call(4, 1 << 30, 2, 2) == pk.PK_ERR_ARG          # requests times KV heads
    many = pk.pk_heads(FAKE, 65536 * 64, 64)
    h = many
    assert call(0x7fff0000, 40, 65536, 512) == pk.PK_ERR_ARG  # groups of 128: two tokens an item


def test_page_weights_of_more_blocks_than_a_launch_has(pk):
    kv, h = pk.pk_kv_cache(FAKE, 4, 16, 1, 64, 1.0, 1.0), pk.pk_heads(FAKE, 64, 64)
    L, b = pk.lib(), ctypes.byref
    stride = (1 << 27) - 1
    call = lambda R, w: L.pk_attend_cache(b(kv), 0, b(h), b(h), None, R, 1, 1, 1.0, FAKE, FAKE, stride, w, FAKE, 1 << 62, None,
                                          None)
    assert call(1 << 12, FAKE) == pk.PK_ERR_ARG


def test_rows_of_more_splits_than_a_launch_has_blocks(pk):
    kv, h = pk.pk_kv_cache(FAKE, 4, 16, 1, 64, 1.0, 1.0), pk.pk_heads(FAKE, 64, 64)
    L, b = pk.lib(), ctypes.byref
    assert L.pk_attend_cache(b(kv), 0, b(h), b(h), None, (1 << 31) - 1, 1, 1, 1.0, FAKE, FAKE, 1, None, FAKE, 1 << 62, None,
                             None) != pk.PK_ERR_ARG  # one block a request: as many as a launch takes
