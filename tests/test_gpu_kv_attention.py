"""Attention over the paged key-value cache: how much of a weight is kept, and where values are
infinite."""
import math

import numpy as np
import pytest

from oracle import kv_oracle as O
from tests._util import bits_to_dev, dev_to_f64, f64_to_bits
from tests.test_gpu_kv import FORMATS, Pages, bf16, dev, fill, tables

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("page,kv,heads,d,lens,window", [
    (16, 2, 6, 64, [2, 3, 5, 17, 40], 0),
    (32, 1, 5, 80, [2, 4, 33, 300], 0),
    (16, 2, 4, 96, [3, 129, 40], 7),
    (64, 1, 20, 128, [2, 3, 200], 0),
    (128, 1, 3, 256, [2, 5, 260], 0),
    (32, 1, 20, 128, [1500, 700, 2], 0),                  # shared out over several workgroups and joined
    (64, 1, 4, 256, [1200], 0),
])
def test_weights_keep_fifteen_bits(fmt, page, kv, heads, d, lens, window):
    """A few tokens carry each head, with values of either sign: what a weight loses shows beside the result's own rounding."""
    rng = np.random.default_rng(31 * page + heads + d)
    table, n_pages = tables(rng, lens, page)
    host = Pages(n_pages, page, kv, d, fmt, fill=0xFF)
    tokens = fill(host, table, lens, rng, size=2.0)
    q = bf16(rng.normal(size=(len(lens), heads, d)))
    scale = 1.0 / math.sqrt(d)
    got = dev_to_f64(host.on_device().attend(bits_to_dev(f64_to_bits(q.reshape(len(lens), -1))), dev(table),
                                             dev(np.array(lens, dtype=np.int32)), max(lens), window=window)).reshape(q.shape)
    for b, n in enumerate(lens):
        lo = max(0, n - window) if window else 0
        k, v = tokens[b][0][lo:n], tokens[b][1][lo:n]
        ref, mass, size = O.attend_one(q[b], k, v, scale)
        # The result's rounding: half a step, 2^-8 of it.  Everything else is relative to sum w |v|: what cutting a weight to 8 bits leaves,
        # 2^-7 of it, is rounded to 8 bits, 2^-8 of that, and 2^-20 of the weight is added; the logits' d products and sums, factors and
        # maximum in float32 (2^-24 each of at most `size`, times log2 e, in numerator and denominator); the sums over the tokens; exp2
        # to 2^-22, twice.
        rest = (2.0 ** -15 + 2.0 ** -20 + 2 * (d + 8) * 2.0 ** -24 * 1.45 * size[:, None] + 2 * (n - lo) * 2.0 ** -24 + 2.0 ** -21) * mass
        off = np.abs(got[b] - ref) - (2.0 ** -8 * np.abs(ref) + 1.01 * rest)
        assert (off <= 0).all(), (b, n, float((off / mass).max()), int((off > 0).sum()), off.size)


@pytest.mark.parametrize("n,bound", [(1, 1), (40, 40), (300, 300), (700, 700), (700, 5000)])
def test_infinite_values_stay_infinite(n, bound):
    """A positive weight times an infinite value is that infinity; two of either sign are NaN; a masked one does not count."""
    rng = np.random.default_rng(33)
    page, d, window = 16, 64, max(n - 1, 1)
    table, n_pages = tables(rng, [n], page)
    host = Pages(n_pages, page, 1, d, "bf16", fill=0xFF)
    tokens = fill(host, table, [n], rng)
    for pos, at, x in ((n - 1, 0, np.inf), (n // 2, 1, -np.inf), (0, 2, np.inf), (n - 1, 3, np.nan), (n - 1, 4, np.inf), (n // 2, 4, -np.inf)):
        v = tokens[0][1][pos].copy()
        v[0, at] = x
        tokens[0][1][pos] = v
        host.put(*O.place(pos, table[0], n_pages, page), v, True)
    wide = np.full((1, -(-bound // page)), -1, dtype=np.int32)
    wide[:, :table.shape[1]] = table
    q = bf16(rng.normal(size=(1, 3, d)))
    args = bits_to_dev(f64_to_bits(q.reshape(1, -1))), dev(wide), dev(np.array([n], dtype=np.int32)), bound
    cache = host.on_device()
    for w in (0, window):
        got = dev_to_f64(cache.attend(*args, window=w)).reshape(3, d)
        assert (got[:, 0] == np.inf).all() and np.isnan(got[:, 3]).all() and np.isfinite(got[:, 5:]).all()
        assert (got[:, 1] == -np.inf).all()
        assert (got[:, 2] == np.inf).all() if w == 0 or n == 1 else np.isfinite(got[:, 2]).all()
        # (of one token alone, the last of the two that are written into it stays)
        assert np.isnan(got[:, 4]).all() if n > 1 else (got[:, 4] == -np.inf).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n,bound", [(1, 16), (40, 40), (300, 300), (100, 5000), (700, 5000)])
def test_heads_with_logits_of_minus_infinity_only_get_zeros_whatever_the_values(fmt, n, bound):
    rng = np.random.default_rng(34)
    page, d = 16, 64
    table, n_pages = tables(rng, [n], page)
    host = Pages(n_pages, page, 1, d, fmt, fill=0xFF)
    for pos in range(n):
        at = O.place(pos, table[0], n_pages, page)
        host.put(*at, bf16(np.abs(rng.normal(size=(1, d))) + 0.5), False)
        v = bf16(rng.normal(size=(1, d)))
        v[0, :3] = np.inf, -np.inf, np.nan
        host.put(*at, v, True)
    wide = np.full((1, -(-bound // page)), -1, dtype=np.int32)
    wide[:, :table.shape[1]] = table
    q = bf16(np.abs(rng.normal(size=(3, d))) + 0.5)
    q[1, 7] = -np.inf                                                 # (keys are positive: every logit of head 1 is minus infinity)
    got = dev_to_f64(host.on_device().attend(bits_to_dev(f64_to_bits(q.reshape(1, -1))), dev(wide), dev(np.array([n], dtype=np.int32)),
                                             bound)).reshape(3, d)
    assert np.isnan(got[0, 2]) and np.isnan(got[2, 2]) and not got[1].any()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("lens", [[40, 3], [1500, 900]])
@pytest.mark.parametrize("q_exp,k_exp,v_exp", [(0, 0, -88), (0, 0, 97), (95, -95, 0), (-95, 95, 0)])
def test_sizes_up_to_the_stated_limits(fmt, lens, q_exp, k_exp, v_exp):
    """Queries and values up to 2^100, value rows down to 2^-90; the bound is that of the weights' test (all sizes are powers of
    two times ordinary ones, and nothing leaves the range of normal float32 numbers)."""
    rng = np.random.default_rng(35)
    page, kv, heads, d = 32, 1, 6, 64
    table, n_pages = tables(rng, lens, page)
    host = Pages(n_pages, page, kv, d, fmt, fill=0xFF)
    tokens = []
    for b, n in enumerate(lens):
        rows = [], []
        for pos in range(n):
            at = O.place(pos, table[b], n_pages, page)
            for j, e in ((0, k_exp), (1, v_exp)):
                host.put(*at, bf16(np.clip(rng.normal(size=(kv, d)), -4, 4)) * 2.0 ** e, bool(j))
                rows[j].append(host.get(*at, bool(j)))
        tokens.append([np.array(r) for r in rows])
    q = bf16(np.clip(rng.normal(size=(len(lens), heads, d)), -4, 4)) * 2.0 ** q_exp
    got = dev_to_f64(host.on_device().attend(bits_to_dev(f64_to_bits(q.reshape(len(lens), -1))), dev(table),
                                             dev(np.array(lens, dtype=np.int32)), max(lens))).reshape(q.shape)
    for b, n in enumerate(lens):
        ref, mass, size = O.attend_one(q[b], *tokens[b], 1.0 / math.sqrt(d))
        rest = (2.0 ** -15 + 2.0 ** -20 + 2 * (d + 8) * 2.0 ** -24 * 1.45 * size[:, None] + 2 * n * 2.0 ** -24 + 2.0 ** -21) * mass
        off = np.abs(got[b] - ref) - (2.0 ** -8 * np.abs(ref) + 1.01 * rest)
        assert (off <= 0).all(), (b, n, float((off / mass).max()), int((off > 0).sum()), off.size)
