"""Cosine and sine at the farthest positions against angles of 96 bits that do not come from the library."""
import math

import numpy as np
import pytest
import torch

import paper_2605_30010_amd as et
from tests._util import dev_to_f64
from tests.test_gpu_kv import dev
from tests.test_rotary_steps import exact_steps

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("base,rot_dim,scaling", [(1e6, 128, None), (1e4, 256, None), (5e5, 64, dict(kind="ntk", factor=8.0)),
                                                  (1e6, 128, dict(kind="yarn", factor=4.0, original_len=32768))])
@pytest.mark.parametrize("first", [2 ** 31 - 4000, -2 ** 31, 10 ** 9])
def test_far_positions(base, rot_dim, scaling, first):
    """Row 2 i + j has the position, of four thousand, at which the sine (j = 0) or cosine of pair i is nearest to 0, where the result's own
    rounding (2^-8) hides least; a pair (1, 0) becomes A (cos, sin), each within 2^-22 of A."""
    turns = [round(x * 2 ** 32) for x in exact_steps(rot_dim, base, scaling)]                 # 2^-96 of a turn
    rows, angles = [], []
    for s in turns:
        at = np.array([(p * s) % 2 ** 96 / 2.0 ** 96 for p in range(first, first + 4000)]) * 2 * math.pi
        for fn in (np.sin, np.cos):
            best = int(np.abs(fn(at)).argmin())
            rows.append(first + best)
            angles.append(at[best])
    r = et.Rotary(rot_dim, base=base, layout="interleaved", scaling=scaling)
    x = torch.zeros((len(rows), rot_dim), dtype=torch.bfloat16, device="cuda:0")
    x[:, 0::2] = 1.0
    got = dev_to_f64(r.apply(x, None, dev(np.array(rows, dtype=np.int32)))[0]).reshape(len(rows), -1, 2)
    for row, angle in enumerate(angles):
        for value, ref in zip(got[row, row // 2], (r.amplitude * math.cos(angle), r.amplitude * math.sin(angle))):
            assert abs(value - ref) <= 2.0 ** -8 * abs(ref) + 2.0 ** -22 * r.amplitude, (row, rows[row], value, ref)
