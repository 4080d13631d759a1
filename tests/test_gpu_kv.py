"""The paged key-value cache on the device against its float64 definition: codes and values bit for bit, attention within
bounds that the arithmetic gives."""
import math

import numpy as np
import pytest
import torch

import paper_2605_30010_amd as et
from oracle import kv_oracle as O
from tests._util import bits_to_dev, dev_to_bits, dev_to_f64, f64_to_bits

pytestmark = pytest.mark.gpu
FORMATS = ["bf16", "e4m3", "int8"]


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")


def bf16(a):
    """float64 array rounded to bfloat16 values."""
    return torch.from_numpy(np.asarray(a, dtype=np.float64)).to(torch.bfloat16).double().numpy()


class Pages:
    """A cache in host memory, written token by token as the layout says."""

    def __init__(self, n_pages, page, kv, d, fmt, fill=0xA5):
        self.n_pages, self.page, self.kv, self.d, self.fmt = n_pages, page, kv, d, fmt
        self.e = 2 if fmt == "bf16" else 1
        self.part = 2 * page * d * self.e + (0 if fmt == "bf16" else 4 * page)
        self.data = np.full((n_pages, kv * self.part), fill, dtype=np.uint8)

    def cells(self, page, at, head, value):
        """(slice of the row's bytes, slice of its maximum's)."""
        base, row = head * self.part, self.d * self.e
        first = base + (self.page * row if value else 0) + at * row
        top = base + 2 * self.page * row + (2 * self.page if value else 0) + 2 * at
        return slice(first, first + row), slice(top, top + 2)

    def put(self, page, at, x, value):
        """x [kv, d] float64 (bfloat16 values)."""
        for h in range(self.kv):
            cell, top = self.cells(page, at, h, value)
            if self.fmt == "bf16":
                self.data[page, cell] = f64_to_bits(x[h]).view(np.uint8)
            else:
                codes, m = O.hold(x[h], self.fmt)
                self.data[page, cell] = codes
                self.data[page, top] = np.array([0x7FC0 if np.isnan(m) else f64_to_bits(m)], dtype=np.uint16).view(np.uint8)

    def get(self, page, at, value):
        """float64 [kv, d]: what the token's row stands for."""
        out = np.empty((self.kv, self.d))
        for h in range(self.kv):
            cell, top = self.cells(page, at, h, value)
            if self.fmt == "bf16":
                out[h] = (self.data[page, cell].view(np.uint16).astype(np.uint32) << 16).view(np.float32)
            else:
                m = (self.data[page, top].view(np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)
                out[h] = O.stands_for(self.data[page, cell], m, self.fmt)
        return out

    def on_device(self):
        return et.KVCache(self.n_pages, self.page, self.kv, self.d, fmt=self.fmt, data=dev(self.data))


def tables(rng, lens, page, extra=2, holes=()):
    """(table int32 [n, wide], pages): random pages for every sequence, -1 behind them, `holes` = (sequence, entry) without one."""
    used = [-(-n // page) for n in lens]
    n_pages = sum(used) + extra
    free, table = list(rng.permutation(n_pages)), np.full((len(lens), max(used + [1])), -1, dtype=np.int32)
    for b, n in enumerate(used):
        for i in range(n):
            table[b, i] = free.pop()
    for b, i in holes:
        table[b, i] = -1
    return table, n_pages


def fill(pages, table, lens, rng, size=1.0):
    """Stores random keys and values for all tokens; returns what they stand for, [(k, v)] per sequence, and which have a page."""
    out = []
    for b, n in enumerate(lens):
        ks, vs, have = [], [], []
        for pos in range(n):
            at = O.place(pos, table[b], pages.n_pages, pages.page)
            have.append(at is not None)
            if at is None:
                ks.append(np.zeros((pages.kv, pages.d)))
                vs.append(ks[-1])
                continue
            pages.put(*at, bf16(rng.normal(size=(pages.kv, pages.d)) * size + 0.3), False)
            pages.put(*at, bf16(rng.normal(size=(pages.kv, pages.d))), True)
            ks.append(pages.get(*at, False))
            vs.append(pages.get(*at, True))
        shape = (n, pages.kv, pages.d)
        out.append((np.array(ks).reshape(shape), np.array(vs).reshape(shape), np.array(have, dtype=bool)))
    return out


# ---------------------------------------------------------------------------------------------- storing and reading back

SPECIAL = [0.0, -0.0, 1.0, -1.0, 0.5, -0.5, 254.0, 127.0, 448.0, 2.0 ** 127, -3.3895313892515355e38, 2.0 ** -126, 2.0 ** -133, -2.0 ** -130,
           3 * 2.0 ** -133, 1e-20]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("page,kv,d", [(16, 1, 64), (32, 3, 80), (64, 2, 96), (16, 4, 128), (256, 8, 128), (128, 2, 256), (16, 17, 64)])
def test_append_writes_the_oracles_bytes_and_no_others(fmt, page, kv, d):
    rng = np.random.default_rng(page + kv + d)
    new = [3, 0, 37, 1, 18]
    lens = [5, 0, 37, 70, 18 + page]
    table, n_pages = tables(rng, lens, page, holes=[(2, 0)])
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    rows = int(cu[-1]) + 4                                             # four rows of padding behind the last sequence
    kv_rows = bf16(rng.normal(size=(rows, 2, kv, d)) * np.exp(rng.normal(size=(rows, 2, kv, 1)) * 5))
    few = rng.integers(0, len(SPECIAL), size=(10, d))
    for i in range(10):                                                # rows of special numbers, ties among them
        kv_rows[4 + i, i % 2, 0] = np.array(SPECIAL)[few[i] if i < 5 else few[i] % 8]
    kv_rows[14, 0, kv - 1], kv_rows[15, 1, 0, 3], kv_rows[16, 0, 0, d - 1], kv_rows[17, 1, kv - 1, 0] = 0.0, np.inf, np.nan, -np.inf
    host = Pages(n_pages, page, kv, d, fmt)
    cache = host.on_device()
    width = kv * d
    fused = torch.zeros((rows, 3 * width + 8), dtype=torch.bfloat16, device="cuda:0")          # the rows are columns of a wider matrix
    k, v = fused[:, 8:8 + width], fused[:, 8 + 2 * width:]
    k.copy_(bits_to_dev(f64_to_bits(kv_rows[:, 0].reshape(rows, width))))
    v.copy_(bits_to_dev(f64_to_bits(kv_rows[:, 1].reshape(rows, width))))
    cache.append(k, v, dev(table), dev(np.array(lens, dtype=np.int32)), dev(cu))
    for b in range(len(lens)):
        for i in range(new[b]):
            at = O.place(lens[b] - new[b] + i, table[b], n_pages, page)
            if at is not None:
                for j in range(2):
                    host.put(*at, kv_rows[cu[b] + i, j], bool(j))
    got = cache.data.cpu().numpy()
    if fmt == "bf16":                                                  # (a NaN's payload is kept; the helper's is another)
        a, b = (torch.from_numpy(x.copy()).view(torch.bfloat16) for x in (got, host.data))
        assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.nan_to_num(a.float(), 7.0), torch.nan_to_num(b.float(), 7.0))
    else:
        assert np.array_equal(got, host.data), np.argwhere(got != host.data)[:5]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("page,kv,d", [(16, 1, 64), (32, 3, 80), (64, 2, 96), (16, 4, 128), (256, 8, 128), (128, 2, 256)])
def test_read_gives_the_values_rounded_once(fmt, page, kv, d):
    rng = np.random.default_rng(7 * page + kv + d)
    lens, want = [70, 3, 0, 1, 2 * page + 5], [70, 2, 0, 1, page + 9]
    table, n_pages = tables(rng, lens, page, holes=[(0, 0)])
    host = Pages(n_pages, page, kv, d, fmt)
    for p in range(n_pages):                                           # every code and odd maxima
        for at in range(page):
            for value in (False, True):
                host.put(p, at, bf16(rng.normal(size=(kv, d)) * np.exp(rng.normal() * 6)), value)
    p, at = O.place(0, table[4], n_pages, page)
    p2, at2 = O.place(2 * page + 1, table[4], n_pages, page)
    host.put(p2, at2, bf16(np.resize(SPECIAL, (kv, d))), False)
    host.put(p2, at2, bf16(np.resize([0.0, np.inf, 1.0], (kv, d))), True)
    cu = np.concatenate([[0], np.cumsum(want)]).astype(np.int32)
    rows = int(cu[-1]) + 3
    out = tuple(torch.full((rows, kv * d + 8 * j), 77.0, dtype=torch.bfloat16, device="cuda:0")[:, :kv * d] for j in (1, 2))
    k, v = host.on_device().read(dev(table), dev(np.array(lens, dtype=np.int32)), dev(cu), rows, out=out)
    ref = np.full((2, rows, kv, d), 77.0)
    for b in range(len(lens)):
        for i in range(want[b]):
            at = O.place(lens[b] - want[b] + i, table[b], n_pages, page)
            for j in range(2):
                ref[j, cu[b] + i] = 0.0 if at is None else host.get(*at, bool(j))
    for j, t in enumerate((k, v)):
        got, exp = dev_to_f64(t), bf16(ref[j].reshape(rows, kv * d))
        # (a value below 2^-126 may be rounded twice: to float32's last step there and to bfloat16's)
        same = (got == exp) | (np.isnan(got) & np.isnan(exp)) | ((np.abs(exp) < 2.0 ** -125) & (np.abs(got - exp) <= 2.0 ** -133))
        assert same.all(), (fmt, j, np.argwhere(~same)[:5])


def test_rows_of_many_sequences_find_their_own():
    """200 and 5000 sequences (the search takes two and three steps), many of them without rows."""
    rng = np.random.default_rng(1)
    for n in (64, 65, 200, 4100, 5000):
        new = rng.integers(0, 3, n)
        new[rng.random(n) < 0.5] = 0
        lens = new + rng.integers(0, 5, n)
        table, n_pages = tables(rng, list(lens), 16)
        cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        rows = int(cu[-1])
        x = rng.integers(-128, 128, (rows, 64)).astype(np.float64)
        cache = et.KVCache(n_pages, 16, 1, 64)
        args = dev(table), dev(lens.astype(np.int32)), dev(cu)
        cache.append(bits_to_dev(f64_to_bits(x)), bits_to_dev(f64_to_bits(-x)), *args)
        view = cache.data.view(torch.bfloat16).view(n_pages, 2, 16, 64).double().cpu().numpy()
        seq = np.repeat(np.arange(n), new)
        pos = (lens - new)[seq] + np.arange(rows) - cu[seq]
        assert np.array_equal(view[table[seq, pos // 16], 0, pos % 16], x) and np.array_equal(view[table[seq, pos // 16], 1, pos % 16], -x)
        k, v = cache.read(*args, rows)
        assert np.array_equal(dev_to_f64(k), x) and np.array_equal(dev_to_f64(v), -x)


def test_one_row_per_sequence_without_row_ranges():
    rng = np.random.default_rng(2)
    lens = np.array([1, 0, 40, 16, 17], dtype=np.int32)               # an idle slot among them
    table, n_pages = tables(rng, list(lens), 16)
    host = Pages(n_pages, 16, 2, 128, "int8")
    cache = host.on_device()
    x = bf16(rng.normal(size=(5, 2, 2, 128)))
    k, v = (bits_to_dev(f64_to_bits(x[:, j])) for j in range(2))      # [rows, heads, head_dim]
    cache.append(k, v, dev(table), dev(lens))
    for b, n in enumerate(lens):
        at = O.place(int(n) - 1, table[b], n_pages, 16)
        if at is not None:
            host.put(*at, x[b, 0], False)
            host.put(*at, x[b, 1], True)
    assert np.array_equal(cache.data.cpu().numpy(), host.data)
    got, _ = cache.read(dev(table), dev(lens))
    assert not got[1].any() and got[0].any()


def test_tables_and_lengths_outside_the_cache_are_no_places():
    """Page numbers out of range, lengths past the table, ranges that do not ascend: nothing is written, zeros are read."""
    rng = np.random.default_rng(5)
    cache = et.KVCache(4, 16, 2, 64, fmt="e4m3")
    cache.data.fill_(0x31)
    before = cache.data.clone()
    table = dev(np.array([[4, -7], [2 ** 31 - 1, -2 ** 31], [-1, -1]], dtype=np.int32))
    k = bits_to_dev(f64_to_bits(bf16(rng.normal(size=(6, 128)))))
    cu = dev(np.array([0, 2, 4, 6], dtype=np.int32))
    for lens in ([32, 32, 32], [2, 2, 2], [33, 2 ** 31 - 1, 10 ** 6], [0, -5, -2 ** 31]):
        lens = dev(np.array(lens, dtype=np.int32))
        cache.append(k, k, table, lens, cu)
        out = cache.read(table, lens, cu, 6)
        assert not out[0].any() and not out[1].any()
        assert not cache.attend(k[:3], table, lens, 2 ** 31 - 1).any()
    good = dev(np.array([[0, 1], [2, 3], [1, 2]], dtype=np.int32))
    for lens in ([34, 40, 2 ** 31 - 1], [0, -1, -2 ** 31]):
        cache.append(k, k, good, dev(np.array(lens, dtype=np.int32)), cu)
    for ranges in ([6, 4, 2, 0], [7, 8, 9, 10], [-9, -6, -3, 0]):
        cache.append(k, k, good, dev(np.array([9, 9, 9], dtype=np.int32)), dev(np.array(ranges, dtype=np.int32)))
    assert torch.equal(cache.data, before)


# ---------------------------------------------------------------------------------------------- attention of one new token

def check_attention(host, table, lens, tokens, q, heads, window=0, scale=None, max_len=None, cache=None, q_dev=None):
    """q float64 [n, heads, d] (bfloat16 values); tokens as fill() gives them."""
    n, d = len(lens), host.d
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    cache = host.on_device() if cache is None else cache
    if q_dev is None:
        q_dev = bits_to_dev(f64_to_bits(q.reshape(n, heads * d)))
    max_len = max(list(lens) + [1]) if max_len is None else max_len
    got = dev_to_f64(cache.attend(q_dev, dev(table), dev(np.array(lens, dtype=np.int32)), max_len, window=window, scale=scale))
    got = got.reshape(n, heads, d)
    for b in range(n):
        k, v, have = tokens[b]
        seen = have & (np.arange(lens[b]) >= (lens[b] - window if window else 0)) & (np.arange(lens[b]) < max_len)
        ref, mass, size = O.attend_one(q[b], k[seen], v[seen], scale)
        # One rounding of the result (half a step, 2^-8) and one of every weight (2^-8 of sum w |v|).  Logits: d products and
        # sums, the scale and the running maximum in float32, 2^-24 each of at most `size` times log2 e; a shift of a
        # logit moves numerator and denominator.  Sums over the tokens: at most their number of float32 roundings, in
        # numerator and denominator; exp2 is good to 2^-22.
        logit = 2 * (d + 8) * 2.0 ** -24 * 1.45 * size[:, None]
        tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + logit + 2 * seen.sum() * 2.0 ** -24 + 2.0 ** -21) * mass + 1e-37
        off = np.abs(got[b] - ref) - tol
        assert (off <= 0).all(), (b, lens[b], float(off.max()), np.argwhere(off > 0)[:3])
    return got


GRID = [  # page, kv heads, heads, head width, lengths, window
    (16, 1, 1, 64, [1, 2, 15, 16, 17, 31, 32, 33], 0),
    (16, 2, 8, 128, [63, 64, 65, 127, 128, 129, 0], 0),
    (32, 3, 15, 80, [0, 1, 100, 333], 0),
    (64, 2, 32, 96, [700, 5, 129], 0),
    (256, 2, 14, 128, [1000, 257, 256, 1], 0),
    (128, 1, 20, 256, [400, 129], 0),
    (16, 1, 33, 64, [90, 1], 0),
    (32, 4, 4, 256, [77], 0),
    (16, 2, 10, 128, [200, 30, 1, 0, 17], 1),
    (16, 2, 10, 128, [200, 30, 1, 0, 17], 16),
    (32, 2, 4, 80, [500, 33], 33),
    (64, 1, 7, 64, [500, 130], 100),
]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("page,kv,heads,d,lens,window", GRID)
def test_attention_of_one_token(fmt, page, kv, heads, d, lens, window):
    rng = np.random.default_rng(page + heads + d + window)
    table, n_pages = tables(rng, lens, page)
    host = Pages(n_pages, page, kv, d, fmt, fill=0xFF)                # unwritten places are NaN in every format
    tokens = fill(host, table, lens, rng)
    q = bf16(rng.normal(size=(len(lens), heads, d)))
    got = check_attention(host, table, lens, tokens, q, heads, window)
    for b, n in enumerate(lens):
        assert n > 0 or not got[b].any()


@pytest.mark.parametrize("fmt", FORMATS)
def test_attention_over_long_sequences(fmt):
    """Lengths that are split over many workgroups, a longer bound than any of them, and a short sequence beside them."""
    rng = np.random.default_rng(11)
    lens, kv, heads, d, page = [9001, 3, 5000, 0], 1, 4, 128, 64
    table, n_pages = tables(rng, lens, page)
    host = Pages(n_pages, page, kv, d, fmt, fill=0xFF)
    tokens = fill(host, table, lens, rng)
    q = bf16(rng.normal(size=(len(lens), heads, d)))
    cache = host.on_device()
    check_attention(host, table, lens, tokens, q, heads, cache=cache)
    check_attention(host, table, lens, tokens, q, heads, cache=cache, max_len=10 ** 6)
    check_attention(host, table, lens, tokens, q, heads, cache=cache, max_len=4999)
    check_attention(host, table, lens, tokens, q, heads, cache=cache, window=4000, max_len=2 ** 31 - 1)


@pytest.mark.parametrize("fmt", FORMATS)
def test_attention_leaves_out_what_has_no_page(fmt):
    """Holes in the table (evicted pages): at the start, in the middle, the newest, everything."""
    rng = np.random.default_rng(12)
    lens, page = [100, 100, 100, 100, 260], 16
    holes = [(0, 0), (0, 3), (1, 6), (2, 5), (2, 6)] + [(3, i) for i in range(7)] + [(4, i) for i in range(1, 16)]
    table, n_pages = tables(rng, lens, page, holes=holes)
    host = Pages(n_pages, page, 2, 64, fmt, fill=0xFF)
    tokens = fill(host, table, lens, rng)
    q = bf16(rng.normal(size=(len(lens), 6, 64)))
    got = check_attention(host, table, lens, tokens, q, 6)
    assert not got[3].any()
    got = check_attention(host, table, lens, tokens, q, 6, window=4)  # the last page of 1 and 2 is gone: nothing left
    assert not got[1:4].any() and got[0].any() and got[4].any()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("size", [0.01, 8.0, 60.0])
def test_attention_with_small_and_large_logits(fmt, size):
    """Nearly equal weights, and logits of thousands whose maximum moves all the time."""
    rng = np.random.default_rng(13)
    lens, page = [600, 601], 32
    table, n_pages = tables(rng, lens, page)
    host = Pages(n_pages, page, 1, 128, fmt, fill=0xFF)
    tokens = fill(host, table, lens, rng, size=size)
    q = bf16(rng.normal(size=(2, 5, 128)) * max(size, 1.0))
    check_attention(host, table, lens, tokens, q, 5)
    check_attention(host, table, lens, tokens, q, 5, scale=-0.25)
    check_attention(host, table, lens, tokens, q, 5, scale=0.0)


def test_attention_of_infinities_and_nan():
    """In keys: minus infinity takes a token out, only such logits give zeros, plus infinity and NaN give NaN to the heads that
    see them and to no others.  (bfloat16 cache: the 8-bit forms hold no infinities.)"""
    rng = np.random.default_rng(14)
    lens, page, d = [40, 40, 40, 40, 40], 16, 64
    table, n_pages = tables(rng, lens, page)
    host = Pages(n_pages, page, 2, d, "bf16", fill=0xFF)
    tokens = fill(host, table, lens, rng)
    q = bf16(np.abs(rng.normal(size=(5, 4, d))) + 0.1)                # positive: the sign of an infinite logit is the key's
    for b, places, x in ((0, [3, 39], -np.inf), (1, range(40), -np.inf), (2, [17], np.inf), (3, [17], np.nan)):
        for pos in places:
            page_at = O.place(pos, table[b], n_pages, page)
            k = tokens[b][0][pos].copy()
            k[0] = x                                                  # head 0 alone
            host.put(*page_at, k, False)
            tokens[b][0][pos] = k
    got = dev_to_f64(host.on_device().attend(bits_to_dev(f64_to_bits(q.reshape(5, -1))), dev(table), dev(np.array(lens, dtype=np.int32)),
                                             40)).reshape(5, 4, d)
    assert np.isnan(got[2:4, :2]).all() and not np.isnan(got[2:4, 2:]).any()
    assert not got[1, :2].any() and got[1, 2:].any()
    keep = np.setdiff1d(np.arange(40), [3, 39])
    for h in range(2):
        ref, mass, _ = O.attend_one(q[0, h:h + 1], tokens[0][0][keep][:, :1], tokens[0][1][keep][:, :1], d ** -0.5)
        assert (np.abs(got[0, h] - ref[0]) <= 2.0 ** -8 * np.abs(ref[0]) + (2.0 ** -8 + 1e-4) * mass[0]).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("window", [1, 7, 16, 40])
def test_attention_does_not_see_what_is_masked(fmt, window):
    """Rows of NaN and infinities in front of the window, in the window's first group of 16 too, change nothing."""
    rng = np.random.default_rng(18)
    lens, page = [50, 33, 200, 17], 16
    table, n_pages = tables(rng, lens, page)
    host = Pages(n_pages, page, 2, 80, fmt, fill=0xFF)
    tokens = fill(host, table, lens, rng)
    for b, n in enumerate(lens):
        for pos in range(max(0, n - window)):
            row = np.full((2, 80), [np.nan, np.inf, -np.inf][pos % 3])
            for value in (False, True):
                host.put(*O.place(pos, table[b], n_pages, page), row, value)
    q = bf16(rng.normal(size=(len(lens), 6, 80)))
    got = check_attention(host, table, lens, tokens, q, 6, window=window)
    assert np.isfinite(got).all() and got.any()


def test_attention_reads_strided_queries_and_tables_and_repeats_its_bits():
    rng = np.random.default_rng(15)
    lens, page, heads, d = [3000, 77, 1500], 32, 14, 128
    table, n_pages = tables(rng, lens, page)
    host = Pages(n_pages, page, 2, d, "int8", fill=0xFF)
    tokens = fill(host, table, lens, rng)
    q = bf16(rng.normal(size=(3, heads, d)))
    fused = torch.full((3, heads * d + 512), float("nan"), dtype=torch.bfloat16, device="cuda:0")
    fused[:, 256:256 + heads * d] = bits_to_dev(f64_to_bits(q.reshape(3, -1)))
    cache = host.on_device()
    a = check_attention(host, table, lens, tokens, q, heads, cache=cache, q_dev=fused[:, 256:256 + heads * d])
    wide = torch.full((3, table.shape[1] + 9), -1, dtype=torch.int32, device="cuda:0")
    wide[:, :table.shape[1]] = dev(table)
    args = wide[:, :table.shape[1]], dev(np.array(lens, dtype=np.int32)), 3000
    q3 = fused[:, 256:256 + heads * d].unflatten(1, (heads, d))
    for _ in range(3):
        out = torch.full((3, heads * d), 9.0, dtype=torch.bfloat16, device="cuda:0")
        assert cache.attend(q3, *args, out=out) is out
        assert np.array_equal(dev_to_f64(out).reshape(a.shape), a)
    longer = dev_to_f64(cache.attend(q3, wide, dev(np.array(lens, dtype=np.int32)), wide.shape[1] * page)).reshape(a.shape)
    assert np.abs(longer - a).max() <= 2.0 ** -6 * np.abs(a).max()    # another split: other roundings only


@pytest.mark.parametrize("fmt,page,kv,heads,d,lens,window", [
    ("int8", 16, 2, 8, 64, [0, 1, 700, 33, 129, 16, 0, 511] * 19, 0),             # 152 sequences: their lengths are scanned in three steps
    ("bf16", 32, 1, 5, 80, list(range(0, 130)), 0),
    ("e4m3", 16, 1, 4, 96, [1000, 0, 3, 640, 1500] * 14, 600),
    ("bf16", 64, 16, 32, 64, [9000, 1, 7000, 0, 12000, 300, 9500], 0),             # long parts, and shorter ones in their place
    ("e4m3", 256, 32, 32, 128, [5000, 4097, 128, 6000], 0),
    ("int8", 128, 8, 24, 256, [20000], 0),                                          # a single sequence in many parts
    ("bf16", 16, 8, 8, 128, [513], 0),
    ("bf16", 16, 8, 8, 128, [40000, 513, 2], 520),
    ("int8", 16, 64, 64, 64, [45000], 0),                                          # parts of more than 64 groups of 16 tokens a wavefront
    ("e4m3", 64, 64, 64, 80, [61000, 61003, 4], 0),
])
def test_attention_of_many_and_of_long_sequences(fmt, page, kv, heads, d, lens, window):
    """Against float64 on what the cache reads back, with the bound of check_attention."""
    rng = np.random.default_rng(17)
    g = torch.Generator("cuda:0").manual_seed(17)
    table, n_pages = tables(rng, lens, page)
    cache = et.KVCache(n_pages, page, kv, d, fmt=fmt)
    cache.data.fill_(0xFF)
    rows = sum(lens)
    x = torch.randn((rows, 2 * kv * d), generator=g, device="cuda:0").to(torch.bfloat16)
    q = torch.randn((len(lens), heads * d), generator=g, device="cuda:0").to(torch.bfloat16)
    args = dev(table), dev(np.array(lens, dtype=np.int32))
    cu = dev(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32))
    cache.append(x[:, :kv * d], x[:, kv * d:], *args, cu)
    # float64 values of what is held: the codes are those of the rows (tested above)
    held = x.double().reshape(rows, 2, kv, d)
    if fmt != "bf16":
        m = held.abs().amax(-1, keepdim=True)
        y = held * O.QMAX[fmt] / m
        held = (torch.round(y) if fmt == "int8" else y.float().to(torch.float8_e4m3fn).double()) * m / O.QMAX[fmt]
    got = cache.attend(q, *args, max(lens), window=window).double().reshape(len(lens), kv, heads // kv, d)
    at = 0
    for b, n in enumerate(lens):
        lo = at + (max(0, n - window) if window else 0)
        k, v = (held[lo:at + n, j].transpose(0, 1).contiguous() for j in range(2))            # [kv, tokens, d]
        qb = q[b].double().reshape(kv, heads // kv, d)
        if n == 0:
            assert not got[b].any()
            continue
        w = torch.softmax(qb @ k.transpose(1, 2).contiguous() / math.sqrt(d), -1)
        size = (qb.abs() @ k.abs().transpose(1, 2).contiguous()).amax(-1, keepdim=True) / math.sqrt(d)
        ref, mass = w @ v, w @ v.abs()
        tol = 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2 * (d + 8) * 2.0 ** -24 * 1.45 * size + 2 * n * 2.0 ** -24 + 2.0 ** -21) * mass
        assert ((got[b] - ref).abs() <= tol).all(), (b, n, float(((got[b] - ref).abs() - tol).max()))
        at += n


def test_pages_past_four_gigabytes():
    """Pages whose byte offset needs more than 32 bits: stored, read back and attended to."""
    rng = np.random.default_rng(16)
    page, kv, d = 256, 16, 256
    size = et.et_kv_page_bytes(page, kv, d, "bf16")                   # 4 MiB
    n_pages = 2 ** 32 // size + 40
    cache = et.KVCache(n_pages, page, kv, d)
    low = cache.data[:64].clone()
    lens = [300, 5]
    table = np.array([[n_pages - 1, n_pages - 3], [n_pages - 2, -1]], dtype=np.int32)
    x = bf16(rng.normal(size=(305, 2, kv, d)))
    k, v = (bits_to_dev(f64_to_bits(x[:, j].reshape(305, -1))) for j in range(2))
    args = dev(table), dev(np.array(lens, dtype=np.int32))
    cu = dev(np.array([0, 300, 305], dtype=np.int32))
    cache.append(k, v, *args, cu)
    got = cache.read(*args, cu, 305)
    assert torch.equal(got[0], k) and torch.equal(got[1], v) and torch.equal(cache.data[:64].view(torch.int64), low.view(torch.int64))
    q = bf16(rng.normal(size=(2, kv, d)))
    out = dev_to_f64(cache.attend(bits_to_dev(f64_to_bits(q.reshape(2, -1))), *args, 300)).reshape(2, kv, d)
    for b, (lo, hi) in enumerate(((0, 300), (300, 305))):
        ref, mass, _ = O.attend_one(q[b], x[lo:hi, 0], x[lo:hi, 1], 1 / 16)
        assert (np.abs(out[b] - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 1e-4) * mass).all()


# ---------------------------------------------------------------------------------------------- together, captured, side by side

@pytest.mark.parametrize("fmt", FORMATS)
def test_prompts_and_steps_through_one_cache(fmt):
    """As a decoder uses it: prompts of two users go in, then tokens one by one, each attending to all before it; at the end
    the cache reads back what went in."""
    rng = np.random.default_rng(21)
    page, kv, heads, d, prompt, steps = 16, 2, 8, 128, [45, 7], 12
    total = [n + steps for n in prompt]
    table, n_pages = tables(rng, total, page)
    host = Pages(n_pages, page, kv, d, fmt, fill=0xFF)
    cache = host.on_device()
    x = [bf16(rng.normal(size=(n, 2, kv, d))) for n in total]
    q = bf16(rng.normal(size=(steps, 2, heads, d)))

    def rows(parts, j):
        return bits_to_dev(f64_to_bits(np.concatenate(parts)[:, j].reshape(-1, kv * d)))

    def store(parts, lens, cu):
        cache.append(rows(parts, 0), rows(parts, 1), dev(table), dev(np.array(lens, dtype=np.int32)), cu)

    for b in range(2):
        for pos in range(total[b]):
            for j in range(2):
                host.put(*O.place(pos, table[b], n_pages, page), x[b][pos, j], bool(j))
    stand = [tuple(np.array([host.get(*O.place(p, table[b], n_pages, page), bool(j)) for p in range(total[b])]) for j in range(2))
             for b in range(2)]
    store([x[b][:prompt[b]] for b in range(2)], prompt, dev(np.array([0, 45, 52], dtype=np.int32)))
    for t in range(steps):
        lens = [n + t + 1 for n in prompt]
        store([x[b][lens[b] - 1:lens[b]] for b in range(2)], lens, None)
        tokens = [(stand[b][0][:lens[b]], stand[b][1][:lens[b]], np.ones(lens[b], dtype=bool)) for b in range(2)]
        check_attention(host, table, lens, tokens, q[t], heads, cache=cache)
    assert np.array_equal(cache.data.cpu().numpy(), host.data)
    k, v = cache.read(dev(table), dev(np.array(total, dtype=np.int32)), dev(np.array([0, 57, 76], dtype=np.int32)), 76)
    for j, t in enumerate((k, v)):
        assert np.array_equal(dev_to_f64(t), bf16(np.concatenate([stand[b][j] for b in range(2)]).reshape(76, -1)))


@pytest.mark.parametrize("fmt", ["bf16", "int8"])
def test_a_captured_step_is_replayed_as_the_sequences_grow(fmt):
    """Append and attention in one graph with a generous bound; lengths, rows and queries change in place, eager work runs
    between the replays, and a second graph of the same cache replays beside it."""
    rng = np.random.default_rng(22)
    page, kv, heads, d, n = 16, 2, 6, 64, 3
    lens = np.array([30, 1, 250], dtype=np.int32)
    table, n_pages = tables(rng, [300, 300, 300], page)
    cache, eager = (et.KVCache(n_pages, page, kv, d, fmt=fmt) for _ in range(2))
    seed = torch.randint(0, 100, cache.data.shape, dtype=torch.uint8, generator=torch.Generator().manual_seed(1))
    cache.data.copy_(seed)
    eager.data.copy_(seed)
    tab, length = dev(table), dev(lens)
    k, v, q = (torch.zeros((n, w * d), dtype=torch.bfloat16, device="cuda:0") for w in (kv, kv, heads))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cache.append(k, v, tab, length)
        cache.attend(q, tab, length, 300)
    torch.cuda.current_stream().wait_stream(side)
    cache.data.copy_(seed)
    graphs = []
    for window in (0, 40):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            cache.append(k, v, tab, length)
            out = cache.attend(q, tab, length, 300, window=window)
        graphs.append((g, out, window))
    for step in range(5):
        for t in (k, v, q):
            t.copy_(torch.from_numpy(rng.normal(size=tuple(t.shape))).to(torch.bfloat16))
        length += 1
        for g, out, window in graphs:
            g.replay()
            eager.append(k, v, tab, length)
            ref = eager.attend(q, tab, length, 300, window=window)
            torch.cuda.synchronize()
            assert torch.equal(cache.data, eager.data) and torch.equal(out, ref) and out.any()


def test_calls_on_several_streams_at_once():
    """Two streams attend to one cache at the same time, a third stores into another one; results are those of one after
    the other, also for a stream that is not the current one."""
    rng = np.random.default_rng(23)
    page, kv, heads, d = 64, 4, 28, 128
    lens = np.array([6000, 300], dtype=np.int32)
    table, n_pages = tables(rng, list(lens), page)
    cache, other = (et.KVCache(n_pages, page, kv, d, fmt="e4m3") for _ in range(2))
    x = torch.randn((6300, kv * d), generator=torch.Generator("cuda:0").manual_seed(2), device="cuda:0").to(torch.bfloat16)
    args = dev(table), dev(lens)
    cu = dev(np.array([0, 6000, 6300], dtype=np.int32))
    cache.append(x, -x, *args, cu)
    qs = [torch.randn((2, heads * d), device="cuda:0").to(torch.bfloat16) for _ in range(2)]
    ref = [cache.attend(q, *args, 6000) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = [[], []]
    for _ in range(10):
        for i in range(2):
            got[i].append(cache.attend(qs[i], *args, 6000, stream=streams[i]))
        other.append(x, -x, *args, cu, stream=streams[2])
        read = other.read(*args, cu, 6300, stream=streams[2])
    torch.cuda.synchronize()
    assert all(torch.equal(t, ref[i]) for i in range(2) for t in got[i])
    # (places that no token has been stored in keep what the allocator gave)
    back = cache.read(*args, cu, 6300)
    assert torch.equal(back[0], read[0]) and torch.equal(back[1], read[1])


def test_binding_refusals():
    cache = et.KVCache(4, 16, 2, 64)
    tab, lens = torch.zeros((3, 2), dtype=torch.int32, device="cuda:0"), torch.ones(3, dtype=torch.int32, device="cuda:0")
    x = torch.zeros((3, 128), dtype=torch.bfloat16, device="cuda:0")
    for bad in (x.float(), x.cpu()):
        with pytest.raises(TypeError):
            cache.append(bad, x, tab, lens)
        with pytest.raises(TypeError):
            cache.attend(bad, tab, lens, 16)
    for bad in (x[:, :64], x.t(), x[:2], x[None]):
        with pytest.raises(ValueError):
            cache.append(x, bad, tab, lens)
    with pytest.raises(et.EtError):
        cache.append(x[:2], x[:2], tab, lens)                         # no row ranges: one row for each sequence
    with pytest.raises(et.EtError):
        cache.attend(torch.zeros((3, 192), dtype=torch.bfloat16, device="cuda:0"), tab, lens, 16)   # 3 heads, 2 key-value heads
    with pytest.raises(et.EtError):
        cache.attend(x, tab, lens, 0)
    with pytest.raises(et.EtError):
        cache.append(torch.zeros((3, 132), dtype=torch.bfloat16, device="cuda:0")[:, 2:130], x, tab, lens)   # not aligned
    for bad in (tab.long(), tab.cpu()):
        with pytest.raises(TypeError):
            cache.read(bad, lens)
    for bad_tab, bad_lens in ((tab[0], lens), (tab.t(), lens), (tab[:2], lens), (tab, lens[:, None]), (tab, lens.repeat(2)[::2])):
        with pytest.raises(ValueError):
            cache.read(bad_tab, bad_lens)
    with pytest.raises(ValueError):
        cache.read(tab, lens, torch.zeros(3, dtype=torch.int32, device="cuda:0"))
    with pytest.raises(ValueError):
        cache.read(tab, lens, out=(x[:2], x))
    with pytest.raises(ValueError):
        cache.attend(x, tab, lens, 16, out=x[:2])
