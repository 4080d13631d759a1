"""Float64 definition of rotary positions.  numpy and whole numbers only; shares nothing with the device code."""
import math

import numpy as np


def frequencies(rot_dim, base, scaling=None):
    """(f_i in radians per position, as Python floats; the factor A)."""
    sc = scaling or {}
    kind, s, n = sc.get("kind"), sc.get("factor", 1.0), rot_dim
    if kind == "ntk" and n > 2:
        base = base * s ** (n / (n - 2))
    f = [base ** (-2 * i / n) for i in range(n // 2)]
    if kind == "linear" or (kind == "ntk" and n == 2):
        return [x / s for x in f], 1.0
    if kind == "yarn":
        slow, fast, length = sc.get("slow", 1.0), sc.get("fast", 32.0), sc["original_len"]
        index = lambda turns: n * math.log(length / (2 * math.pi * turns)) / (2 * math.log(base))
        first, last = max(math.floor(index(fast)), 0), min(math.ceil(index(slow)), n - 1)
        r = [min(max((i - first) / max(last - first, 0.001), 0.0), 1.0) for i in range(n // 2)]
        return [x / s * a + x * (1 - a) for x, a in zip(f, r)], 0.1 * math.log(s) + 1.0
    if kind == "turns":
        slow, fast, length = sc.get("slow", 1.0), sc.get("fast", 4.0), sc["original_len"]
        keep = [min(max((length * x / (2 * math.pi) - slow) / (fast - slow), 0.0), 1.0) for x in f]
        return [x / s * (1 - a) + x * a for x, a in zip(f, keep)], 1.0
    return f, 1.0


def angles(positions, steps):
    """[rows, pairs] radians: position * step is a whole number of 2^-64 turns, and exact as such."""
    return np.array([[((int(p) * int(s)) % 2 ** 64) / 2.0 ** 64 for s in steps] for p in positions]).reshape(len(positions), len(steps)) * 2 * math.pi


def apply(x, angle, amplitude, rot_dim, layout, transpose=False):
    """x float64 [rows, heads, head_dim] -> (turned, sum of magnitudes that each result is made of)."""
    c, s = np.cos(angle)[:, None] * amplitude, np.sin(angle)[:, None] * amplitude * (-1 if transpose else 1)
    half = rot_dim // 2
    at = (slice(0, half), slice(half, rot_dim)) if layout == "half" else (slice(0, rot_dim, 2), slice(1, rot_dim, 2))
    a, b = x[..., at[0]], x[..., at[1]]
    y, mass = x.copy(), np.zeros_like(x)
    y[..., at[0]], y[..., at[1]] = a * c - b * s, b * c + a * s
    mass[..., at[0]] = mass[..., at[1]] = np.abs(a) + np.abs(b)
    return y, mass * abs(amplitude)
