"""Rotary positions on the device against their float64 definition."""
import numpy as np
import pytest
import torch

import paper_2605_30010_amd as et
from oracle import rotary_oracle as O
from tests._util import bits_to_dev, dev_to_f64, f64_to_bits
from tests.test_gpu_kv import bf16, dev

pytestmark = pytest.mark.gpu


def check(r, layout, x, positions, got, transpose=False, angle=None):
    """x float64 [rows, heads, head_dim] (bfloat16 values).  One rounding of the result, 2^-8; cosine and sine within 2^-22, and a product
    and a sum in float32, 2^-24 each, of the two magnitudes."""
    angle = O.angles(positions, r.steps.cpu().numpy().view(np.uint64)) if angle is None else angle
    ref, mass = O.apply(x, angle, r.amplitude, r.rot_dim, layout, transpose)
    got = dev_to_f64(got).reshape(ref.shape)
    off = np.abs(got - ref) - (2.0 ** -8 * np.abs(ref) + (2.0 ** -22 + 2.0 ** -23) * mass + 2.0 ** -133)
    assert (off <= 0).all(), (float(off.max()), np.argwhere(off > 0)[:4])
    assert np.array_equal(got[..., r.rot_dim:], x[..., r.rot_dim:])
    return ref


POSITIONS = [0, 1, 2, 3, 7, 100, 4999, 131071, 1000003, 2 ** 31 - 1, -1, -2, -77777, -2 ** 31]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("heads,kv,d,rot", [(8, 2, 128, 128), (3, 1, 64, 32), (28, 4, 128, 64), (5, 5, 80, 80), (2, 1, 96, 24), (4, 4, 256, 256), (6, 3, 80, 86 - 20),
                                            (1, 1, 2, 2), (7, 1, 72, 72), (2, 2, 512, 512), (3, 2, 10, 6), (130, 2, 64, 62), (2, 1, 510, 510)])
def test_turned_rows(layout, heads, kv, d, rot):
    rng = np.random.default_rng(heads + d + rot)
    rows = len(POSITIONS)
    x = bf16(rng.normal(size=(rows, heads + kv, d)) * np.exp(rng.normal(size=(rows, heads + kv, 1)) * 3))
    r = et.Rotary(d, rot_dim=rot, layout=layout)
    t = bits_to_dev(f64_to_bits(x.reshape(rows, -1)))
    q, k = t[:, :heads * d], t[:, heads * d:]                        # columns of a wider matrix
    before = t.clone()
    pos = dev(np.array(POSITIONS, dtype=np.int32))
    for transpose in (False, True):
        a, b = r.apply(q, k, pos, transpose=transpose)
        check(r, layout, x[:, :heads], POSITIONS, a, transpose)
        check(r, layout, x[:, heads:], POSITIONS, b, transpose)
        alone, none = r.apply(q.contiguous().view(rows, heads, d), None, pos, transpose=transpose)
        assert none is None and torch.equal(alone.view(rows, -1), a)
    assert torch.equal(t, before)
    a, b = r.apply(q, k, pos)
    out = r.apply(q, k, pos, out=(q, k))                             # in place
    assert out[0] is q and out[1] is k and torch.equal(q, a) and torch.equal(k, b)


@pytest.mark.parametrize("scaling", [dict(kind="linear", factor=4.0), dict(kind="ntk", factor=8.0), dict(kind="yarn", factor=4.0, original_len=32768),
                                     dict(kind="turns", factor=8.0, original_len=8192)])
def test_scaled_positions(scaling):
    """The angle as the formula has it, position times f_i in float64: 2^-53 of up to 131071 radians besides."""
    rng = np.random.default_rng(3)
    positions = [0, 5, 4096, 40000, 131071]
    for layout in ("half", "interleaved"):
        r = et.Rotary(128, base=500000.0, layout=layout, scaling=scaling)
        f, a = O.frequencies(128, 500000.0, scaling)
        assert abs(a - r.amplitude) <= 2.0 ** -24 * a
        x = bf16(rng.normal(size=(5, 3, 128)))
        got, _ = r.apply(bits_to_dev(f64_to_bits(x)), None, dev(np.array(positions, dtype=np.int32)))
        check(r, layout, x, positions, got, angle=np.array(positions, dtype=np.float64)[:, None] * np.array(f))


@pytest.mark.parametrize("rows", [0, 1, 2, 511, 512, 1025, 4099, 5000])
def test_many_rows(rows):
    rng = np.random.default_rng(rows)
    positions = rng.integers(0, 200000, rows).astype(np.int32)
    x = bf16(rng.normal(size=(rows, 5, 64)))
    r = et.Rotary(64, rot_dim=48)
    got, _ = r.apply(bits_to_dev(f64_to_bits(x)) if rows else torch.empty((0, 5, 64), dtype=torch.bfloat16, device="cuda:0"), None, dev(positions))
    assert got.shape == (rows, 5, 64)
    if rows:
        check(r, "half", x, positions, got)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("shift,pad", [(0, 0), (8, 8), (4, 4), (2, 2), (1, 1), (0, 1), (3, 0)])
def test_any_stride_and_alignment(layout, shift, pad):
    """Rows that begin off 16 bytes, at odd strides; the result is the same, and what lies between the rows stays."""
    rng = np.random.default_rng(9)
    x = bf16(rng.normal(size=(40, 4, 64)))
    r = et.Rotary(64, rot_dim=32, layout=layout)
    pos = dev(np.arange(1000, 1040, dtype=np.int32))
    plain, _ = r.apply(bits_to_dev(f64_to_bits(x)), None, pos)
    check(r, layout, x, range(1000, 1040), plain)
    buf = torch.full((2, 40 * (256 + pad) + 64), 3.0, dtype=torch.bfloat16, device="cuda:0")
    views = [b[shift:shift + 40 * (256 + pad)].view(40, 256 + pad)[:, :256] for b in buf]
    views[0].copy_(bits_to_dev(f64_to_bits(x.reshape(40, -1))))
    r.apply(views[0], None, pos, out=(views[1], None))
    assert torch.equal(views[1], plain.view(40, -1)) and int((buf[1] == 3.0).sum()) >= buf.shape[1] - 40 * 256
    views[1].fill_(3.0)
    assert bool((buf[1] == 3.0).all())
    r.apply(views[0], None, pos, out=(views[0], None))
    assert torch.equal(views[0], plain.view(40, -1))


def test_one_of_two_in_place():
    rng = np.random.default_rng(10)
    t = bits_to_dev(f64_to_bits(bf16(rng.normal(size=(20, 6 * 80)))))
    r = et.Rotary(80, rot_dim=32)
    pos = dev(np.arange(20, dtype=np.int32))
    q, k = t[:, :320], t[:, 320:]
    a, b = r.apply(q, k, pos)
    k2 = torch.empty_like(b)
    r.apply(q, k, pos, out=(q, k2))
    assert torch.equal(q, a) and torch.equal(k2, b)


def test_the_transposed_matrix_is_the_gradient():
    """<y, R x> = <R^T y, x>, R^T as the call has it, and differences of the call along each dimension of one pair give the same columns."""
    rng = np.random.default_rng(11)
    sc = dict(kind="yarn", factor=4.0, original_len=1024)
    for layout in ("half", "interleaved"):
        r = et.Rotary(64, layout=layout, scaling=sc)
        x, y = (bf16(rng.normal(size=(50, 2, 64))) for _ in range(2))
        pos = dev(rng.integers(0, 5000, 50).astype(np.int32))
        rx = dev_to_f64(r.apply(bits_to_dev(f64_to_bits(x)), None, pos)[0])
        ry = dev_to_f64(r.apply(bits_to_dev(f64_to_bits(y)), None, pos, transpose=True)[0])
        # both sides carry one rounding of 2^-8 a value
        left, right = (y * rx).sum(-1), (ry * x).sum(-1)
        tol = 2.0 ** -8 * (np.abs(y * rx).sum(-1) + np.abs(ry * x).sum(-1)) + 1e-5
        assert (np.abs(left - right) <= tol).all()
        for d in (0, 1, 31, 32, 63):
            e = np.zeros((50, 2, 64))
            e[..., d] = 1.0
            up, down = (dev_to_f64(r.apply(bits_to_dev(f64_to_bits(s * e)), None, pos)[0]) for s in (1.0, -1.0))
            column = (up - down) / 2                                 # of R; row d of R^T
            back = dev_to_f64(r.apply(bits_to_dev(f64_to_bits(y)), None, pos, transpose=True)[0])[..., d]
            tol = 2.0 ** -8 * (np.abs(back) + np.abs(column * y).sum(-1)) + 1e-5
            assert (np.abs((column * y).sum(-1) - back) <= tol).all()


def test_there_and_back():
    """With A = 1 the transposed matrix is the inverse, up to two roundings."""
    rng = np.random.default_rng(12)
    x = bf16(rng.normal(size=(30, 3, 128)))
    r = et.Rotary(128)
    pos = dev(rng.integers(0, 10 ** 6, 30).astype(np.int32))
    t = bits_to_dev(f64_to_bits(x))
    back = r.apply(r.apply(t, None, pos)[0], None, pos, transpose=True)[0]
    size = np.abs(x[..., :64]) + np.abs(x[..., 64:])
    assert (np.abs(dev_to_f64(back) - x) <= 2.0 ** -8 * np.abs(x) + (2.0 ** -8 * 1.01 + 2.0 ** -19) * np.concatenate([size, size], -1)).all()


def test_numbers_without_end_stay_in_their_pair():
    x = bf16(np.random.default_rng(13).normal(size=(4, 2, 64)))
    x[1, 0, 5], x[2, 1, 40], x[3, 0, 63] = np.inf, np.nan, -np.inf
    r = et.Rotary(64, rot_dim=32)
    got = dev_to_f64(r.apply(bits_to_dev(f64_to_bits(x)), None, dev(np.array([3, 4, 5, 6], dtype=np.int32)))[0])
    bad = ~np.isfinite(got)
    assert bad.sum() == 4 and bad[1, 0, 5] and bad[1, 0, 21] and np.isnan(got[2, 1, 40]) and got[3, 0, 63] == -np.inf


def test_replayed_and_on_other_streams():
    """A captured call reads positions and rows as they are when it is replayed; two streams at once."""
    rng = np.random.default_rng(14)
    r = et.Rotary(128)
    q, k = (torch.randn((9, w), device="cuda:0").to(torch.bfloat16) for w in (512, 256))
    pos = torch.zeros(9, dtype=torch.int32, device="cuda:0")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r.apply(q, k, pos)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a, b = r.apply(q, k, pos)
    for _ in range(4):
        pos.copy_(dev(rng.integers(0, 10 ** 5, 9).astype(np.int32)))
        q.copy_(torch.randn((9, 512), device="cuda:0"))
        g.replay()
        c, d = r.apply(q, k, pos)
        torch.cuda.synchronize()
        assert torch.equal(a, c) and torch.equal(b, d)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [r.apply(q, k, pos, stream=s) for s in streams for _ in range(5)]
    torch.cuda.synchronize()
    assert all(torch.equal(x, c) and torch.equal(y, d) for x, y in got)


def test_columns_of_one_matrix():
    """Queries, keys and values side by side: turned in place, or from some columns into others of the same rows."""
    rows, heads, kv, d = 9, 4, 2, 64
    g = torch.Generator("cuda:0").manual_seed(4)
    r, pos = et.Rotary(d), torch.arange(5, 5 + rows, dtype=torch.int32, device="cuda:0")
    fused = torch.randn((rows, (2 * heads + 2 * kv) * d), generator=g, device="cuda:0").to(torch.bfloat16)
    q, k = fused[:, :heads * d], fused[:, heads * d:(heads + kv) * d]
    want, kept = r.apply(q, k, pos), fused.clone()
    to = fused[:, (heads + 2 * kv) * d:]
    got = r.apply(q, None, pos, out=(to, None))[0]
    assert got is to and torch.equal(to, want[0]) and torch.equal(fused[:, :(heads + 2 * kv) * d], kept[:, :(heads + 2 * kv) * d])
    r.apply(q, k, pos, out=(q, k))
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(fused[:, (heads + kv) * d:(heads + 2 * kv) * d], kept[:, (heads + kv) * d:(heads + 2 * kv) * d])
    for a, b, out in ((q, q, (q, q)), (q, None, (fused[:, 1:heads * d + 1], None)), (k, k, (k, None)), (q, k, (to, fused[:, -kv * d:]))):
        with pytest.raises(et.EtError):
            r.apply(a, b, pos, out=out)
    both = r.apply(q, q, pos)                             # one tensor as both is fine where nothing of it is written
    assert torch.equal(both[0], both[1])


@pytest.mark.parametrize("layout,heads,kv,d,rot,in_place", [("half", 14, 2, 128, 128, False), ("interleaved", 14, 2, 128, 64, False), ("interleaved", 32, 0, 64, 64, True),
                                                            ("half", 12, 4, 256, 128, True), ("interleaved", 23, 2, 80, 32, False)])
def test_large_calls_equal_small_ones(layout, heads, kv, d, rot, in_place):
    """More than the caches hold (134 MB written), against the same rows a thousand at a time."""
    rows = 2 ** 26 // ((heads + kv) * d) + 77
    g = torch.Generator("cuda:0").manual_seed(6)
    q, k = (torch.randn((rows, n * d), generator=g, device="cuda:0").to(torch.bfloat16) if n else None for n in (heads, kv))
    pos = torch.randint(-2 ** 31, 2 ** 31, (rows,), generator=g, device="cuda:0").int()
    r = et.Rotary(d, rot, layout=layout)
    want = [], []
    for i in range(0, rows, 1000):
        for w, x in zip(want, r.apply(q[i:i + 1000], None if k is None else k[i:i + 1000], pos[i:i + 1000])):
            w.append(x)
    got = r.apply(q, k, pos, out=(q, k) if in_place else None)
    assert torch.equal(got[0], torch.cat(want[0])) and (k is None or torch.equal(got[1], torch.cat(want[1])))
