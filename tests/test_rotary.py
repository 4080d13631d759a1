"""Rotary positions without a GPU: the steps against a definition of their own, and what is refused."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2605_30010_amd as et
from oracle import rotary_oracle as O
from paper_2605_30010_amd import binding as B

SCALINGS = [None, dict(kind="linear", factor=4.0), dict(kind="ntk", factor=8.0), dict(kind="yarn", factor=4.0, original_len=32768),
            dict(kind="yarn", factor=1.0, original_len=64), dict(kind="yarn", factor=16.0, original_len=4096, slow=2.0, fast=20.0),
            dict(kind="turns", factor=8.0, original_len=8192), dict(kind="turns", factor=3.0, original_len=100, slow=0.5, fast=9.0)]


@pytest.mark.parametrize("scaling", SCALINGS)
@pytest.mark.parametrize("rot_dim", [2, 4, 32, 86, 128, 512])
@pytest.mark.parametrize("base", [10000.0, 500000.0, 1.5])
def test_steps_are_the_frequencies(rot_dim, base, scaling):
    """Within a few roundings of float64 (pow, log and the mix), relatively."""
    steps, amplitude = et.et_rotary_steps(rot_dim, base, scaling)
    f, a = O.frequencies(rot_dim, base, scaling)
    got = [int(s) * 2 * math.pi / 2.0 ** 64 for s in steps]
    assert len(got) == rot_dim // 2 and np.allclose(got, f, rtol=1e-13, atol=2.0 ** -60) and abs(amplitude - a) <= 2.0 ** -24 * a


def test_the_fastest_pair_turns_by_one_radian():
    steps, a = et.et_rotary_steps(128)
    assert a == 1.0 and abs(int(steps[0]) - round(2 ** 64 / (2 * math.pi))) <= 2 ** 12 and (np.diff(steps.astype(np.float64)) < 0).all()


def test_refused_steps():
    for args in ((0,), (3,), (-2,), (514,), (128, 0.5), (128, math.nan), (128, math.inf), (128, 1e31)):
        with pytest.raises(et.EtError):
            et.et_rotary_steps(*args)
    for bad in (dict(kind="linear", factor=0.5), dict(kind="linear", factor=math.nan), dict(kind="yarn", factor=2.0, original_len=0),
                dict(kind="yarn", factor=2.0, original_len=100, slow=4.0, fast=4.0), dict(kind="turns", factor=2.0, original_len=100, slow=0.0),
                dict(kind="turns", factor=2.0, original_len=math.nan)):
        with pytest.raises(et.EtError):
            et.et_rotary_steps(128, 10000.0, bad)
    with pytest.raises(et.EtError):
        et.et_rotary_steps(128, 1.0, dict(kind="yarn", factor=2.0, original_len=100))
    for bad in (dict(kind="other", factor=2.0), dict(kind="linear", factor=2.0, original_len=3)):
        with pytest.raises(ValueError):
            et.et_rotary_steps(128, 10000.0, bad)
    with pytest.raises(KeyError):
        et.et_rotary_steps(128, 10000.0, dict(kind="yarn", factor=2.0))
    lib, steps, a = et.load_library(), (C.c_uint64 * 64)(), C.c_float()
    assert lib.et_rotary_steps(None, 128, 1e4, None, C.byref(a)) == -1 and lib.et_rotary_steps(None, 128, 1e4, steps, None) == -1
    bad = B._RotaryScaling(7, 1.0, 1.0, 1.0, 2.0)
    assert lib.et_rotary_steps(C.byref(bad), 128, 1e4, steps, C.byref(a)) == -1


FAKE = 4096                                              # never dereferenced


def call(rotary=None, positions=FAKE, rows=3, q=None, k=None, transpose=0, **kw):
    r = B._Rotary(**dict(dict(steps_dev=FAKE, head_dim=64, rot_dim=64, layout=0, amplitude=1.0), **(rotary or {})))
    x = lambda d: B._RotaryRows(**dict(dict(in_dev=FAKE, in_stride=256, out_dev=FAKE * 4, out_stride=256, n_heads=4), **d))
    q = x(q or {})
    k = None if k is None else x(k)
    return et.load_library().et_rotary_apply(C.byref(r), positions, rows, C.byref(q), None if k is None else C.byref(k), transpose, None)


@pytest.mark.parametrize("bad", [dict(rotary=dict(head_dim=0)), dict(rotary=dict(head_dim=63)), dict(rotary=dict(head_dim=514)), dict(rotary=dict(rot_dim=66)),
                                 dict(rotary=dict(rot_dim=0)), dict(rotary=dict(rot_dim=31)), dict(rotary=dict(layout=2)),
                                 dict(rotary=dict(amplitude=math.inf)), dict(rotary=dict(steps_dev=None)), dict(rotary=dict(steps_dev=FAKE + 4)),
                                 dict(positions=None), dict(rows=-1), dict(rows=2 ** 27 - 7), dict(transpose=2)] +
                         [{x: bad} for x in "qk" for bad in (dict(in_dev=None), dict(out_dev=None), dict(in_dev=FAKE + 1), dict(in_stride=255), dict(out_stride=192),
                                                             dict(n_heads=-1), dict(n_heads=65537, in_stride=1 << 40, out_stride=1 << 40),
                                                             dict(out_dev=FAKE, out_stride=264))])
def test_refused_calls(bad):
    assert call(**bad) == -1 and et.et_last_error()


def test_null_descriptors_and_empty_calls():
    lib, r, x = et.load_library(), B._Rotary(FAKE, 64, 64, 0, 1.0), B._RotaryRows(FAKE, 256, FAKE, 256, 4)
    assert lib.et_rotary_apply(None, FAKE, 3, C.byref(x), None, 0, None) == -1 and lib.et_rotary_apply(C.byref(r), FAKE, 3, None, None, 0, None) == -1
    assert call(rows=0, positions=None) == 0 and call(q=dict(n_heads=0, in_dev=None, out_dev=None), k=dict(n_heads=0)) == 0


def test_binding_refuses_shapes():
    for bad in (dict(head_dim=63), dict(head_dim=64, rot_dim=66), dict(head_dim=64, rot_dim=3), dict(head_dim=1024), dict(head_dim=64, layout="other")):
        with pytest.raises(ValueError):
            et.Rotary(device="cpu", **bad)
    r = et.Rotary(64, device="cpu")                      # (no library call is reached with host tensors)
    x = torch.zeros((3, 128), dtype=torch.bfloat16)
    pos = torch.zeros(3, dtype=torch.int32)
    r._here = lambda stream: 0
    for q, p in ((x, pos.long()), (x.float(), pos)):
        with pytest.raises(TypeError):
            r.apply(q, None, p)
    for q, p in ((x[:2], pos), (x[:, :100], pos), (x.t(), pos), (x, pos[None]), (x, torch.zeros(6, dtype=torch.int32)[::2])):
        with pytest.raises(ValueError):
            r.apply(q, None, p)
    with pytest.raises(ValueError):
        r.apply(x, None, pos, out=(x[:, :64], None))


def test_refuses_results_that_lie_on_something_else():
    """Two results in one place, a result on the other's rows or in part on its own; columns of one matrix keep apart (no row: nothing runs)."""
    at, row = FAKE * 16, dict(in_stride=1024, out_stride=1024)            # 4 heads of 64: 256 of 1024 columns
    q = dict(row, in_dev=at, out_dev=at)
    for k in (dict(out_dev=at), dict(in_dev=at), dict(out_dev=at + 2 * 255), dict(in_dev=at + 2 * 1024 * 2 - 2), dict(out_dev=at - 2 * 255), dict(out_stride=1025),
              dict(out_dev=at + 2 * 1024 - 2)):
        k = dict(dict(row, in_dev=at + 2 * 256, out_dev=at + 2 * 512), **k)
        assert call(q=q, k=k) == -1 and "lies on" in et.et_last_error(), k
    for out, stride in ((at + 2, 1024), (at + 2 * 255, 1024), (at - 2 * 769, 1024), (at + 2 * 256, 1000)):
        assert call(q=dict(in_dev=at, in_stride=1024, out_dev=out, out_stride=stride)) == -1 and "itself" in et.et_last_error(), (out, stride)
