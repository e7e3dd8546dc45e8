"""The turns of a rotary table against 60 decimal digits."""
import math
from decimal import Decimal, getcontext

import pytest

from paper_2609_32869_gb300 import binding as B

PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620900")


@pytest.mark.parametrize("rot", [2, 6, 64, 96, 128, 256])
@pytest.mark.parametrize("base", [10000.0, 500000.0, 1.5, 1e8])
def test_plain_turns(rot, base):
    """base^(-2i / rot) / 2 pi: pow to a step (2^-52), its exponent's rounding times ln base, 2 pi's and the division's halves of a step;
    then the cut to a whole number of 2^-64."""
    getcontext().prec = 60
    t = B.wf_rope_init(256, rot, base=base)
    for i in range(rot // 2):
        want = (Decimal(base).ln() * (Decimal(-2 * i) / rot)).exp() / (2 * PI)
        err = abs(Decimal(t.turns[i]) / 2 ** 64 - want)
        assert err <= want * Decimal((5 + math.log(base)) * 2.0 ** -53) + Decimal(2) ** -64


@pytest.mark.parametrize("pos", [1 << 20, 1 << 24, 2 ** 31 - 1, -2 ** 31])
def test_far_angles(pos):
    """A far position's angle, as the calls compute it, is off by no more than its turns times the turn's error and 2^-32 of a turn."""
    getcontext().prec = 60
    t = B.wf_rope_init(128)
    for i in range(64):
        turn = (Decimal(10000).ln() * (Decimal(-2 * i) / 128)).exp() / (2 * PI)
        got = Decimal(pos * t.turns[i] % 2 ** 64 >> 32) / 2 ** 32
        off = (got - pos * turn) % 1
        off = min(off, 1 - off)
        assert off <= abs(pos) * (turn * Decimal((5 + math.log(10000)) * 2.0 ** -53) + Decimal(2) ** -64) + Decimal(2) ** -32
