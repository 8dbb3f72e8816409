"""Tables of a rotation whose parts are ramped over the pair's index (no GPU)."""
import math

import numpy as np
import pytest

from paper_2609_38706_gb300 import _build


@pytest.fixture(scope="module")
def pk():
    _build.build()
    from paper_2609_38706_gb300 import pk as m
    m.lib()
    return m


# The ends are i(32) and i(1), by hand: 20.94 and 45.03; 23.60 and 39.65; 10.47 and 22.51; and with 1 and 4 turns of 8192,
# base 500000, 128 dimensions, i(4) = 64 ln(325.95) / ln(500000) = 28.22, i(1) = 34.98.
CASES = [(128, 1e4, 8.0, 4096.0, 1.0, 32.0, 20, 46), (128, 1e6, 4.0, 32768.0, 1.0, 32.0, 23, 40),
         (64, 1e4, 40.0, 4096.0, 1.0, 32.0, 10, 23), (128, 5e5, 8.0, 8192.0, 1.0, 4.0, 28, 35)]


@pytest.mark.parametrize("rot,base,factor,context,low,high,first,last", CASES)
def test_ramp_over_the_index(pk, rot, base, factor, context, low, high, first, last):
    got = pk.pk_rotary_turns_by_index(rot, base, factor, context, low, high).astype(np.float64) * 2.0 ** -64
    for i in range(rot // 2):
        f = math.exp(-2 * i / rot * math.log(base)) / (2 * math.pi)
        divided = min(max((i - first) / (last - first), 0.0), 1.0)
        want = f * (1 - divided) + f / factor * divided
        # an exponential of up to 13, whose argument is off by 2^-50, and a few products of 64 bits; cut at 2^-64
        assert abs(got[i] - want) <= want * 2.0 ** -46 + 2.0 ** -64, i


def test_the_two_ramps_differ(pk):
    """By 57%, 42% and 77% of a frequency: not a detail that a model gets over.  What turns often enough stays in both."""
    for case, most in zip(CASES, (0.57, 0.42, 0.77)):
        a = pk.pk_rotary_turns(*case[:6]).astype(np.float64)
        b = pk.pk_rotary_turns_by_index(*case[:6]).astype(np.float64)
        assert abs(np.abs(1 - a / b).max() - most) < 0.01 and np.array_equal(a[: case[6] + 1], b[: case[6] + 1])


def test_ends_outside_the_pairs(pk):
    # i(32) below 0: the ramp begins at the first pair; i(1) above the last pair: it ends behind them, at rotary_dim - 1
    plain = pk.pk_rotary_turns(16, 2.0, 1.0, 0.0, 1.0, 32.0).astype(np.float64)
    got = pk.pk_rotary_turns_by_index(16, 2.0, 4.0, 100.0, 1.0, 32.0).astype(np.float64)
    weigh = (15 - np.arange(8)) / 15  # i(1) = 8 ln(15.9) / ln 2 = 31.9
    assert np.allclose(got, plain * (weigh + (1 - weigh) / 4), rtol=1e-12, atol=0)


@pytest.mark.parametrize("args", [
    (128, 1e4, 8.0, 0.0, 1.0, 32.0), (128, 1e4, 8.0, 4096.0, 0.0, 32.0), (128, 1e4, 8.0, -1.0, 1.0, 32.0),
    (128, 1e4, 8.0, 4096.0, 32.0, 32.0), (24, 1e4, 8.0, 4096.0, 1.0, 32.0), (144, 1e4, 8.0, 4096.0, 1.0, 32.0),
    (128, 1.0, 8.0, 4096.0, 1.0, 32.0), (128, 1e4, float("nan"), 4096.0, 1.0, 32.0), (128, 1e4, 8.0, 4096.0, 1.0, float("inf")),
    (128, 1e4, 8.0, 0.5, 1.0, 32.0),      # no pair makes a turn: nothing stays, not even the first
    (16, 1.01, 8.0, 1e9, 1.0, 32.0)])     # all pairs make more than `high`: nothing is divided
def test_refused(pk, args):
    with pytest.raises(pk.PKError):
        pk.pk_rotary_turns_by_index(*args)


def test_rotary(pk):
    from paper_2609_38706_gb300 import service
    a = service.Rotary(128, factor=8.0, context=4096.0, ramp="index", device="cpu")
    assert np.array_equal(a.turns.numpy().view(np.uint64), pk.pk_rotary_turns_by_index(128, 10000.0, 8.0, 4096.0, 1.0, 32.0))
    for same in (dict(), dict(ramp="turns")):
        b = service.Rotary(128, factor=8.0, context=4096.0, device="cpu", **same)
        assert np.array_equal(b.turns.numpy().view(np.uint64), pk.pk_rotary_turns(128, 10000.0, 8.0, 4096.0, 1.0, 32.0))
    for kw in (dict(ramp="pairs"), dict(ramp="index"), dict(ramp="index", context=0.5)):
        with pytest.raises(pk.PKError):
            service.Rotary(128, factor=8.0, device="cpu", **kw)
