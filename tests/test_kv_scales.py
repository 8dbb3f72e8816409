"""Host-side checks (no GPU): a score's factor that 32 bits do not hold is refused before any CUDA call, instead of answered
with NaN."""
import ctypes

import pytest

from paper_2609_38706_gb300 import _build

FAKE = 1 << 40  # never dereferenced


@pytest.fixture(scope="module")
def pk():
    _build.build()
    from paper_2609_38706_gb300 import pk as m
    m.lib()
    return m


@pytest.mark.parametrize("k_scale,scale,good", [(1e38, 10.0, False), (3e38, 0.7, True), (1.0, 3e38, False), (1e30, -1e9, False),
                                                (1.0, -2e38, True), (1e-30, 1e-30, True), (1.0, 0.0, True)])
def test_scale_of_a_cached_score(pk, k_scale, scale, good):
    L, b = pk.lib(), ctypes.byref
    kv, h = pk.pk_kv_cache(FAKE, 4, 16, 2, 64, k_scale, 1.0), pk.pk_heads(FAKE, 128, 64)
    rc = L.pk_attend_cache(b(kv), 0, b(h), b(h), None, 0, 1, 2, scale, None, None, 0, None, None, 0, None, None)
    assert rc == (pk.PK_OK if good else pk.PK_ERR_ARG)


@pytest.mark.parametrize("scale,good", [(3e38, False), (-2.5e38, False), (2e38, True), (1e-45, True)])
def test_scale_of_a_prompts_score(pk, scale, good):
    L, b = pk.lib(), ctypes.byref
    h = pk.pk_heads(FAKE, 128, 64)
    rc = L.pk_attend_prompt(0, b(h), b(h), b(h), b(h), None, 4, 4, None, None, 0, 2, 2, 64, scale, None, 0, None, None)
    assert rc == (pk.PK_OK if good else pk.PK_ERR_ARG)
