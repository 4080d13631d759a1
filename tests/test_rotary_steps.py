"""Steps of rotary positions against their formula in 60 decimal digits, and what is left of their error at the farthest positions."""
from decimal import Decimal, getcontext

import pytest

import paper_2605_30010_amd as et

getcontext().prec = 60
PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459")


def exact_steps(n, base, scaling):
    """2^64 f_i / (2 pi), not rounded."""
    sc = scaling or {}
    kind, s, base = sc.get("kind"), Decimal(sc.get("factor", 1.0)), Decimal(base)
    if kind == "ntk" and n > 2:
        base = base * (s.ln() * n / (n - 2)).exp()
    f = [(base.ln() * -2 * i / n).exp() for i in range(n // 2)]
    if kind == "linear" or (kind == "ntk" and n == 2):
        f = [x / s for x in f]
    elif kind == "yarn":
        index = lambda turns: n * (Decimal(sc["original_len"]) / (2 * PI * Decimal(turns))).ln() / (2 * base.ln())
        fast, slow = index(sc.get("fast", 32.0)), index(sc.get("slow", 1.0))
        assert all(abs(x - x.to_integral_value()) > Decimal(1e-9) for x in (fast, slow))      # (no border that float64 could miss)
        first, last = max(fast.to_integral_value("ROUND_FLOOR"), 0), min(slow.to_integral_value("ROUND_CEILING"), n - 1)
        share = [min(max((i - first) / max(last - first, Decimal("0.001")), Decimal(0)), Decimal(1)) for i in range(n // 2)]
        f = [x / s * r + x * (1 - r) for x, r in zip(f, share)]
    elif kind == "turns":
        slow, fast = Decimal(sc.get("slow", 1.0)), Decimal(sc.get("fast", 4.0))
        keep = [min(max((Decimal(sc["original_len"]) * x / (2 * PI) - slow) / (fast - slow), Decimal(0)), Decimal(1)) for x in f]
        f = [x / s * (1 - r) + x * r for x, r in zip(f, keep)]
    return [x / (2 * PI) * 2 ** 64 for x in f]


@pytest.mark.parametrize("scaling", [None, dict(kind="linear", factor=3.0), dict(kind="ntk", factor=8.0), dict(kind="yarn", factor=4.0, original_len=32768),
                                     dict(kind="yarn", factor=40.0, original_len=4096), dict(kind="turns", factor=8.0, original_len=8192)])
@pytest.mark.parametrize("rot_dim", [2, 64, 86, 128, 256, 512])
@pytest.mark.parametrize("base", [10000.0, 500000.0, 1e6, 1.5, 1e30])
def test_steps_are_within_two_units(base, rot_dim, scaling):
    """With 64 bits, in units of 2^-64 of a turn: f <= 1 is 0.16 * 2^64 of them, so a rounding of it (2^-64 relatively at most) is 0.16, of a
    constant or a quotient behind it 0.08; the exponent's, x 2^-64 with x e^-x <= 0.37, 0.06; a base that was changed has up to four such; the mix of two
    three more (the share by turns has few turns, so f is small there); the whole number 0.5.  Less than two in all."""
    exact = exact_steps(rot_dim, base, scaling)
    steps, _ = et.et_rotary_steps(rot_dim, base, scaling)
    off = [abs(Decimal(int(s)) - x) for s, x in zip(steps, exact)]
    assert max(off) <= 2, (float(max(off)), off.index(max(off)))


def test_the_farthest_positions_keep_their_angle():
    """Two units at position -2^31 are 1.5e-9 radians: far below the 2^-22 that cosine and sine are stated with."""
    for base, n in ((1e6, 128), (1e4, 256), (5e5, 128)):
        exact = exact_steps(n, base, None)
        steps, _ = et.et_rotary_steps(n, base)
        for p in (2 ** 31 - 1, -2 ** 31, 10 ** 9 + 7):
            off = [abs(p * (Decimal(int(s)) - x)) / 2 ** 64 * 2 * PI for s, x in zip(steps, exact)]
            assert max(off) <= Decimal(2) ** -29
