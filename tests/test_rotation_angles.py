"""The frequencies of a rotation against decimal arithmetic (CPU)."""
from decimal import Decimal, getcontext

import pytest

import paper_2604_16429_amd as M
from paper_2604_16429_amd import binding

getcontext().prec = 70
TWO_PI = 2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640629")


def decimal_frequencies(d, theta=10000, kind="none", factor=1, original=0):
    """Radians per position of each pair."""
    theta, factor = Decimal(theta), Decimal(factor)
    if kind == "base":
        theta *= factor ** (Decimal(d) / (d - 2))
    out = []
    for i in range(d // 2):
        w = theta ** (Decimal(-2 * i) / d)
        if kind == "linear":
            w /= factor
        if kind == "ramp":
            keep = min(Decimal(1), max(Decimal(0), (original * w / TWO_PI - 1) / 31))
            w = keep * w + (1 - keep) * w / factor
        out.append(w)
    return out


def fraction(x):
    return x - x.to_integral_value(rounding="ROUND_FLOOR")


CASES = [
    ("none", dict(rotary_dim=128), dict(d=128)),
    ("theta", dict(rotary_dim=64, theta=500000.0), dict(d=64, theta=500000)),
    ("axes", dict(rotary_dim=64, axes=2), dict(d=32)),
    ("linear", dict(rotary_dim=48, scaling=binding.SCALE_LINEAR, factor=8.0), dict(d=48, kind="linear", factor=8)),
    ("base", dict(rotary_dim=128, scaling=binding.SCALE_BASE, factor=4.0), dict(d=128, kind="base", factor=4)),
    ("ramp", dict(rotary_dim=128, scaling=binding.SCALE_RAMP, factor=8.0, original_tokens=4096),
     dict(d=128, kind="ramp", factor=8, original=4096)),
    ("given", dict(rotary_dim=8, inv_freq=[1.0, -0.75, 0.3, 1e-7]), None),
]


@pytest.mark.parametrize("name,kw,exact", CASES, ids=[c[0] for c in CASES])
def test_angles_of_any_position(name, kw, exact):
    """The turn's fraction that the kernels take, the upper half of the low 64 bits of position x
    turns, is within 2^-31 of the exact one: 2^-32 is cut off, 2^31 positions times half of 2^-64
    are 2^-34, and what rounding a frequency in 64 bits adds is less."""
    turns = list(M.Rotation(**kw).c.turns)
    freq = decimal_frequencies(**exact) if exact else [Decimal(x) for x in kw["inv_freq"]]
    for i, w in enumerate(freq):
        for pos in (1, 4000, (1 << 24) + 1, 1000000007, (1 << 31) - 1, -1, -(1 << 31)):
            have = Decimal(((pos * turns[i]) % (1 << 64)) >> 32) / (1 << 32)
            off = fraction(have - pos * w / TWO_PI + Decimal("0.5")) - Decimal("0.5")
            assert abs(off) <= Decimal(1) / (1 << 31), (i, pos, float(off) * 2.0 ** 32)
