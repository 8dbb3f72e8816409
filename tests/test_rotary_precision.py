"""How far a rotation's angles may be off: its tables (no GPU) and the kernel's angle, against exact arithmetic."""
import math
import random
from decimal import Decimal, getcontext

import numpy as np
import pytest

from paper_2609_38706_gb300 import _build

PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459")


@pytest.fixture(scope="module")
def pk():
    _build.build()
    from paper_2609_38706_gb300 import pk as m
    m.lib()
    return m


@pytest.mark.parametrize("by", ["plain", "turns", "index"])
def test_entries(pk, by):
    """2^-51 of a turn, as documented.  With u = 2^-53 and f <= 1: f is off by |ln f| + 2 units, the part that stays by 2 |ln f| +
    13, and six operations follow: f / 2 pi (3 |ln f| + 22) u < 4 u.  The cut at 2^-64 comes on top."""
    getcontext().prec = 60
    rng = random.Random(1)
    worst = Decimal(0)
    for _ in range(60):
        rot, base, factor = 16 * rng.randint(1, 8), 10 ** rng.uniform(0.5, 7), 1 + 10 ** rng.uniform(-1, 2)
        context = 0.0 if by == "plain" else 10 ** rng.uniform(2.5, 6)
        low = 10 ** rng.uniform(-0.5, 0.5)
        high = low * rng.uniform(2, 40)
        b, ctx, lo, hi = (Decimal(x) for x in (base, context, low, high))

        def index(n):
            return rot * (ctx / (2 * PI * n)).ln() / (2 * b.ln())

        if by == "index":
            ends = index(hi), index(lo)
            if any(abs(x - x.to_integral_value()) < Decimal(1e-9) for x in ends):
                continue  # rounding decides which way the end goes
            first, last = max(math.floor(ends[0]), 0), min(math.ceil(ends[1]), rot - 1)
            if last < first:
                continue
        make = pk.pk_rotary_turns_by_index if by == "index" else pk.pk_rotary_turns
        got = make(rot, base, factor, context, low, high)
        for i in range(rot // 2):
            f = (-2 * i * b.ln() / rot).exp()
            stays = Decimal(0)
            if by == "turns":
                stays = min(max((ctx * f / (2 * PI) - lo) / (hi - lo), Decimal(0)), Decimal(1))
            elif by == "index":
                stays = Decimal(1 if i <= first else 0 if i >= last else 0)
                if first < i < last:
                    stays = Decimal(last - i) / (last - first)
            want = (stays * f + (1 - stays) * f / Decimal(factor)) / (2 * PI)
            worst = max(worst, abs(Decimal(int(got[i])) / 2 ** 64 - want))
    assert worst <= Decimal(2) ** -51 + Decimal(2) ** -64


@pytest.mark.gpu
def test_angles():
    """Angles next to whole, half and quarter turns, where a large amplitude shows what they are off by: 2^-25 of a turn."""
    import torch

    import __graft_entry__ as g
    from paper_2609_38706_gb300 import service
    g.build()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rng, amp = random.Random(2), 2.0 ** 20
    for pos in (1, 3, 131071, 2 ** 24 + 5, 2 ** 31 - 1):
        # turns t with t * pos mod 2^64 near q quarters of a turn: pos is odd, so it has an inverse
        near = [(rng.randint(0, 3) << 62) + rng.choice((-1, 1)) * int(2 ** rng.uniform(20, 44)) for _ in range(32)]
        turns = np.array([x * pow(pos, -1, 2 ** 64) % 2 ** 64 for x in near], np.uint64)
        assert all(int(t) * pos % 2 ** 64 == x % 2 ** 64 for t, x in zip(turns, near))
        x = torch.zeros((1, 1, 64), dtype=torch.bfloat16, device="cuda")
        x[..., :32] = 1
        none = torch.zeros((1, 0, 64), dtype=torch.bfloat16, device="cuda")
        out, _ = service.rotate(x, none, torch.tensor([0, 1], device="cuda"), torch.tensor([pos], dtype=torch.int32, device="cuda"),
                                service.Rotary(64, turns=turns, amplitude=amp))
        got = out.double().cpu().numpy().reshape(2, 32)
        for i, v in enumerate(near):
            quarter, rest = (v + 2 ** 61) >> 62, (v + 2 ** 61) % 2 ** 62 - 2 ** 61
            t = rest * 2.0 ** -64 * 2 * math.pi
            c, s = [(math.cos(t), math.sin(t)), (-math.sin(t), math.cos(t)), (-math.cos(t), -math.sin(t)),
                    (math.sin(t), -math.cos(t))][quarter % 4]
            for want, have in ((c, got[0, i]), (s, got[1, i])):
                # the angle; sine and cosine to 2 units and a product with amp, of 32 bits; rounded to bfloat16
                slack = amp * (2 * math.pi * 2.0 ** -25 + abs(want) * 3 * 2.0 ** -23)
                assert abs(have - amp * want) <= slack * (1 + 2.0 ** -8) + abs(amp * want) * 2.0 ** -8, (pos, i)
