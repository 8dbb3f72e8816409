"""Host-side checks of strided outputs (no GPU): layouts in which two rows share bytes are refused before any CUDA call, and
the layouts that a serving program has are not."""
import ctypes

import pytest

from paper_2609_38706_gb300 import _build

FAKE = 1 << 40  # never dereferenced: refused, or there is no request to do anything for
ROWS, HEADS, D = 4, 3, 64


@pytest.fixture(scope="module")
def pk():
    _build.build()
    from paper_2609_38706_gb300 import pk as m
    m.lib()
    return m


def calls(pk, out, R):
    """The three calls with strided outputs, `R` requests."""
    L, b = pk.lib(), ctypes.byref
    kv, ok = pk.pk_kv_cache(FAKE, 4, 16, HEADS, D, 1.0, 1.0), pk.pk_heads(FAKE, HEADS * D, D)
    bad = pk.pk_heads(FAKE, *out)
    yield L.pk_kv_read(b(kv), 0, b(bad), b(ok), ROWS, FAKE, FAKE, R, FAKE, 1, None, None)
    yield L.pk_kv_read(b(kv), 0, b(ok), b(bad), ROWS, FAKE, FAKE, R, FAKE, 1, None, None)
    yield L.pk_attend_prompt(0, b(ok), b(ok), b(ok), b(bad), None, ROWS, 4, FAKE, FAKE, R, HEADS, HEADS, D, 1.0, FAKE, 1 << 20,
                             None, None)


def shares(ts, hs):
    used = set()
    for t in range(ROWS):
        for h in range(HEADS):
            row = range(t * ts + h * hs, t * ts + h * hs + D)
            if not used.isdisjoint(row):
                return True
            used.update(row)
    return False


# tokens' stride, heads' stride
SHARING = [(64, 64), (128, 64), (64, 128), (184, 64), (128, 72), (72, 136), (64, 248), (192, 96), (256, 256), (0, 64), (56, 64)]
APART = [(192, 64), (200, 64), (64, 256), (72, 280), (1024, 128), (256, 80)]


@pytest.mark.parametrize("out", SHARING)
def test_rows_that_share_bytes_are_refused(pk, out):
    assert shares(*out)
    assert all(rc == pk.PK_ERR_ARG for rc in calls(pk, out, 1))


@pytest.mark.parametrize("out", APART)
def test_rows_apart_are_not(pk, out):
    assert not shares(*out)
    assert all(rc == pk.PK_OK for rc in calls(pk, out, 0))


def test_the_cache_call(pk):
    L, b = pk.lib(), ctypes.byref
    kv, ok = pk.pk_kv_cache(FAKE, 4, 16, HEADS, D, 1.0, 1.0), pk.pk_heads(FAKE, HEADS * D, D)
    for out in SHARING:
        bad = pk.pk_heads(FAKE, *out)
        assert L.pk_attend_cache(b(kv), 0, b(ok), b(bad), None, ROWS, 1, HEADS, 1.0, FAKE, FAKE, 4, None, FAKE, 1 << 30, None,
                                 None) == pk.PK_ERR_ARG
