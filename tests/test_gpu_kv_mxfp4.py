"""The paged key-value cache in 4 bits on the device against its float64 definition: codes, exponents and values bit for bit, attention
within bounds that the arithmetic gives."""
import math

import numpy as np
import pytest
import torch

import paper_2605_30010_amd as et
from oracle import kv_oracle as O
from tests._util import bits_to_dev, dev_to_f64, f64_to_bits
from tests.test_gpu_kv import bf16, check_attention, dev, fill, tables

pytestmark = pytest.mark.gpu


class Pages4:
    """A cache in host memory, written token by token as the layout says."""

    def __init__(self, n_pages, page, kv, d, fill=0xFF):
        self.n_pages, self.page, self.kv, self.d, self.nb = n_pages, page, kv, d, O.mx_blocks(d)
        self.part = page * (d + 2 * self.nb)
        self.data = np.full((n_pages, kv * self.part), fill, dtype=np.uint8)

    def cells(self, at, head, value):
        """(slice of the row's bytes, slice of its exponents)."""
        base, row, page = head * self.part, self.d // 2, self.page
        first = base + (page * row if value else 0) + at * row
        exps = base + 2 * page * row
        if value:
            return slice(first, first + row), slice(exps + page * self.nb + at, exps + 2 * page * self.nb, page)
        return slice(first, first + row), slice(exps + at * self.nb, exps + (at + 1) * self.nb)

    def put(self, page, at, x, value):
        for h in range(self.kv):
            row, exps = self.cells(at, h, value)
            self.data[page, row], self.data[page, exps] = O.mx_hold(x[h])

    def get(self, page, at, value):
        return np.array([O.mx_stands_for(*(self.data[page, c] for c in self.cells(at, h, value))) for h in range(self.kv)])

    def on_device(self):
        return et.KVCache(self.n_pages, self.page, self.kv, self.d, fmt="mxfp4", data=dev(self.data))


# ties and neighbours of ties, the exponent's border at 7, its limits, subnormal numbers, both zeros
SPECIAL = [0.0, -0.0, 0.25, -0.25, 0.75, 1.25, -1.75, 2.5, 3.5, -5.0, 6.0, 7.0, -7.03125, 0.251953125, 1.0, 2.0 ** 127, -3.3895313892515355e38,
           1.75 * 2.0 ** 127, 2.0 ** -126, -2.0 ** -127, 2.0 ** -133, -2.0 ** -130, 1.5 * 2.0 ** -127, 1e-20]
SHAPES = [(16, 1, 64), (32, 3, 80), (64, 2, 96), (16, 4, 128), (256, 8, 128), (128, 2, 256), (16, 17, 64)]


@pytest.mark.parametrize("page,kv,d", SHAPES)
def test_append_writes_the_oracles_bytes_and_no_others(page, kv, d):
    rng = np.random.default_rng(page + kv + d)
    new, lens = [3, 0, 137, 1, 18], [5, 0, 137, 70, 18 + page]
    table, n_pages = tables(rng, lens, page, holes=[(2, 0)])
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    rows = int(cu[-1]) + 4                                             # four rows of padding behind the last sequence
    x = bf16(rng.normal(size=(rows, 2, kv, d)) * np.exp(rng.normal(size=(rows, 2, kv, 1)) * 5))
    first = lens[2] - new[2]
    at = cu[2] + page - first                                          # rows behind the hole
    for i in range(60):
        few = np.array(SPECIAL)[rng.integers(0, len(SPECIAL) if i % 3 == 0 else 15, d)]
        if i % 3 == 1:                                                 # blocks between 3.5 and 7 times a power of two, whole of eighths
            few = rng.integers(-56, 57, d) / 8.0
        x[(at + i) % (rows - 4), i % 2, i % kv] = few * (1.0 if i % 3 == 0 else 2.0 ** rng.integers(-100, 100))
    x = bf16(x)
    x[at % rows, 0, kv - 1] = 0.0
    x[1, 1, 0, 3], x[1, 0, 0, d - 1], x[2, 1, kv - 1, 0] = np.inf, np.nan, -np.inf   # their blocks are NaN, the row's others are not
    host = Pages4(n_pages, page, kv, d, fill=0xA5)
    cache = host.on_device()
    width = kv * d
    fused = torch.zeros((rows, 3 * width + 8), dtype=torch.bfloat16, device="cuda:0")          # the rows are columns of a wider matrix
    k, v = fused[:, 8:8 + width], fused[:, 8 + 2 * width:]
    k.copy_(bits_to_dev(f64_to_bits(x[:, 0].reshape(rows, width))))
    v.copy_(bits_to_dev(f64_to_bits(x[:, 1].reshape(rows, width))))
    cache.append(k, v, dev(table), dev(np.array(lens, dtype=np.int32)), dev(cu))
    for b in range(len(lens)):
        for i in range(new[b]):
            place = O.place(lens[b] - new[b] + i, table[b], n_pages, page)
            if place is not None:
                for j in range(2):
                    host.put(*place, x[cu[b] + i, j], bool(j))
    got = cache.data.cpu().numpy()
    assert np.array_equal(got, host.data), [(p.tolist(), int(got[tuple(p)]), int(host.data[tuple(p)])) for p in np.argwhere(got != host.data)[:5]]


@pytest.mark.parametrize("page,kv,d", SHAPES)
def test_read_gives_the_values_of_any_bytes(page, kv, d):
    """Every code with every exponent byte, 0, 254 and 255 (NaN) among them: exact, but for what bfloat16 cannot hold."""
    rng = np.random.default_rng(7 * page + kv + d)
    lens, want = [70, 3, 0, 1, 2 * page + 5], [70, 2, 0, 1, page + 9]
    table, n_pages = tables(rng, lens, page, holes=[(0, 0)])
    host = Pages4(n_pages, page, kv, d)
    host.data[:] = rng.integers(0, 256, host.data.shape)
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
        assert np.array_equal(dev_to_f64(t), bf16(ref[j].reshape(rows, kv * d)), equal_nan=True)


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
    (64, 1, 5, 96, [1100], 0),
]


@pytest.mark.parametrize("page,kv,heads,d,lens,window", GRID)
def test_attention_of_one_token(page, kv, heads, d, lens, window):
    rng = np.random.default_rng(page + heads + d + window)
    table, n_pages = tables(rng, lens, page)
    host = Pages4(n_pages, page, kv, d)                               # unwritten places are NaN
    tokens = fill(host, table, lens, rng)
    q = bf16(rng.normal(size=(len(lens), heads, d)))
    got = check_attention(host, table, lens, tokens, q, heads, window)
    for b, n in enumerate(lens):
        assert n > 0 or not got[b].any()


def test_attention_over_long_sequences():
    """Lengths that are split over many workgroups, a longer bound than any of them, and a short sequence beside them."""
    rng = np.random.default_rng(11)
    lens, kv, heads, d, page = [9001, 3, 5000, 0], 1, 4, 128, 64
    table, n_pages = tables(rng, lens, page)
    host = Pages4(n_pages, page, kv, d)
    tokens = fill(host, table, lens, rng)
    q = bf16(rng.normal(size=(len(lens), heads, d)))
    cache = host.on_device()
    check_attention(host, table, lens, tokens, q, heads, cache=cache)
    check_attention(host, table, lens, tokens, q, heads, cache=cache, max_len=10 ** 6)
    check_attention(host, table, lens, tokens, q, heads, cache=cache, max_len=4999)
    check_attention(host, table, lens, tokens, q, heads, cache=cache, window=4000, max_len=2 ** 31 - 1)


def test_attention_leaves_out_what_has_no_page():
    """Holes in the table (evicted pages): at the start, in the middle, the newest, everything."""
    rng = np.random.default_rng(12)
    lens, page = [100, 100, 100, 100, 260], 16
    holes = [(0, 0), (0, 3), (1, 6), (2, 5), (2, 6)] + [(3, i) for i in range(7)] + [(4, i) for i in range(1, 16)]
    table, n_pages = tables(rng, lens, page, holes=holes)
    host = Pages4(n_pages, page, 2, 64)
    tokens = fill(host, table, lens, rng)
    q = bf16(rng.normal(size=(len(lens), 6, 64)))
    got = check_attention(host, table, lens, tokens, q, 6)
    assert not got[3].any()
    got = check_attention(host, table, lens, tokens, q, 6, window=4)  # the last page of 1 and 2 is gone: nothing left
    assert not got[1:4].any() and got[0].any() and got[4].any()


def test_long_parts_leave_out_what_has_no_page():
    """The same where eight wavefronts share a part: holes all over, a sequence without any page, places of NaN around."""
    rng = np.random.default_rng(21)
    lens, page, kv = [650, 600, 20, 0, 530, 64, 1, 300], 16, 8
    holes = [(0, i) for i in range(0, 41, 3)] + [(1, i) for i in range(38)] + [(4, i) for i in range(2, 34)] + [(7, 18), (2, 0)]
    table, n_pages = tables(rng, lens, page, holes=holes)
    host = Pages4(n_pages, page, kv, 64)
    tokens = fill(host, table, lens, rng)
    q = bf16(rng.normal(size=(len(lens), kv, 64)))
    got = check_attention(host, table, lens, tokens, q, kv, max_len=1024)
    assert not got[1].any() and not got[3].any() and got[0].any() and got[2].any()
    check_attention(host, table, lens, tokens, q, kv, window=530, max_len=1024)


@pytest.mark.parametrize("size", [0.01, 8.0, 60.0])
def test_attention_with_small_and_large_logits(size):
    """Nearly equal weights, and logits of thousands whose maximum moves all the time."""
    rng = np.random.default_rng(13)
    lens, page = [600, 601], 32
    table, n_pages = tables(rng, lens, page)
    host = Pages4(n_pages, page, 1, 128)
    tokens = fill(host, table, lens, rng, size=size)
    q = bf16(rng.normal(size=(2, 5, 128)) * max(size, 1.0))
    check_attention(host, table, lens, tokens, q, 5)
    check_attention(host, table, lens, tokens, q, 5, scale=-0.25)
    check_attention(host, table, lens, tokens, q, 5, scale=0.0)


def test_attention_with_blocks_of_very_different_sizes():
    """Blocks from 2^-60 to 2^60 of one another, in keys and values, and queries that bring them together."""
    rng = np.random.default_rng(19)
    for d in (64, 80, 96, 128, 256):
        lens, page, heads = [150, 31], 16, 4
        table, n_pages = tables(rng, lens, page)
        host = Pages4(n_pages, page, 2, d)
        tokens = fill(host, table, lens, rng)
        size = 2.0 ** rng.integers(-60, 61, d // 16).repeat(16)
        for b, n in enumerate(lens):
            for pos in range(n):
                at = O.place(pos, table[b], n_pages, page)
                host.put(*at, bf16(rng.normal(size=(2, d)) * size), False)
                host.put(*at, bf16(rng.normal(size=(2, d)) * size[::-1]), True)
                tokens[b][0][pos], tokens[b][1][pos] = host.get(*at, False), host.get(*at, True)
        q = bf16(rng.normal(size=(2, heads, d)) / size)
        check_attention(host, table, lens, tokens, q, heads)


@pytest.mark.parametrize("d", [64, 80, 96, 128, 256])
def test_blocks_that_are_not_numbers(d):
    """A block of NaN in a key makes its head's results NaN; one in a value those of its 32 dimensions alone; other heads and sequences
    see nothing of it."""
    rng = np.random.default_rng(14)
    lens, page, heads, nb = [40, 40, 40], 16, 4, O.mx_blocks(d)
    table, n_pages = tables(rng, lens, page)
    host = Pages4(n_pages, page, 2, d)
    tokens = fill(host, table, lens, rng)
    q = bf16(rng.normal(size=(3, heads, d)))
    for block in range(nb):
        host2 = Pages4(n_pages, page, 2, d)
        host2.data[:] = host.data
        for b, value in ((0, False), (1, True)):
            p, at = O.place(17, table[b], n_pages, page)
            _, exps = host2.cells(at, 1, value)
            host2.data[p, np.arange(host2.data.shape[1])[exps][block]] = 255
        got = dev_to_f64(host2.on_device().attend(bits_to_dev(f64_to_bits(q.reshape(3, -1))), dev(table), dev(np.array(lens, dtype=np.int32)),
                                                  40)).reshape(3, heads, d)
        inside = np.arange(d) // 32 == block
        assert np.isnan(got[0, 2:]).all() and not np.isnan(got[0, :2]).any() and not np.isnan(got[2]).any()
        assert np.isnan(got[1, 2:][:, inside]).all() and not np.isnan(got[1, 2:][:, ~inside]).any() and not np.isnan(got[1, :2]).any()


@pytest.mark.parametrize("window", [1, 7, 16, 40])
@pytest.mark.parametrize("d", [64, 80, 96, 256])
def test_attention_does_not_see_what_is_masked(d, window):
    """Rows of NaN and infinities in front of the window, in the window's first group of 16 too, change nothing."""
    rng = np.random.default_rng(18)
    lens, page = [50, 33, 200, 17], 16
    table, n_pages = tables(rng, lens, page)
    host = Pages4(n_pages, page, 2, d)
    tokens = fill(host, table, lens, rng)
    for b, n in enumerate(lens):
        for pos in range(max(0, n - window)):
            row = np.full((2, d), [np.nan, np.inf, -np.inf][pos % 3])
            for value in (False, True):
                host.put(*O.place(pos, table[b], n_pages, page), row, value)
    q = bf16(rng.normal(size=(len(lens), 6, d)))
    got = check_attention(host, table, lens, tokens, q, 6, window=window)
    assert np.isfinite(got).all() and got.any()


def test_attention_reads_strided_queries_and_tables_and_repeats_its_bits():
    rng = np.random.default_rng(15)
    lens, page, heads, d = [3000, 77, 1500], 32, 14, 128
    table, n_pages = tables(rng, lens, page)
    host = Pages4(n_pages, page, 2, d)
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


def held(x):
    """float64 values that rows x [..., d] (torch, any device, finite) stand for."""
    out = []
    for b in x.double().split(32, -1):
        e = torch.ceil(torch.log2(b.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -100) / 7)).clamp(-125, 125)
        a = b / torch.exp2(e)
        step = torch.where(a.abs() < 2, 0.5, torch.where(a.abs() < 4, 1.0, 2.0))
        out.append((torch.round(a / step) * step).clamp(-6, 6) * torch.exp2(e))
    return torch.cat(out, -1)


MIDDLE = [1000, 0, 1, 33, 513, 700, 128, 129, 255, 1023, 64, 900]


@pytest.mark.parametrize("page,kv,heads,d,lens,window", [
    (16, 2, 8, 64, [0, 1, 700, 33, 129, 16, 0, 511] * 19, 0),         # 152 sequences: their lengths are scanned in three steps
    (32, 1, 5, 80, list(range(0, 130)), 0),
    (16, 1, 4, 96, [1000, 0, 3, 640, 1500] * 14, 600),
    (64, 16, 32, 64, [9000, 1, 7000, 0, 12000, 300, 9500], 0),        # long parts, and shorter ones in their place
    (256, 32, 32, 128, [5000, 4097, 128, 6000], 0),
    (128, 8, 24, 256, [20000], 0),                                    # a single sequence in many parts
    (16, 8, 8, 128, [513], 0),
    (16, 8, 8, 128, [40000, 513, 2], 520),
    (16, 64, 64, 64, [45000], 0),                                     # parts of more than 64 groups of 16 tokens a wavefront
    (64, 64, 64, 80, [61000, 61003, 4], 0),
    (64, 4, 4, 128, [70] * 4100, 0),                                  # more than 4096 sequences are one part each
    # one part each by eight wavefronts, of every head width, several row tiles, a window
    (16, 8, 16, 64, MIDDLE, 0), (32, 8, 8, 80, MIDDLE, 0), (64, 8, 24, 96, MIDDLE, 0), (16, 8, 8, 128, MIDDLE, 600), (128, 8, 16, 256, MIDDLE, 0),
    (16, 8, 144, 128, MIDDLE, 0), (16, 24, 24, 80, [9001, 5000, 2047, 2048, 2049, 1, 0, 3000, 2100], 2047),
    (64, 8, 8, 64, [2048, 5, 1999, 0] * 16, 0),                       # and by four
])
def test_attention_of_many_and_of_long_sequences(page, kv, heads, d, lens, window):
    """Against float64 on what the cache holds, with the bound of check_attention."""
    rng = np.random.default_rng(17)
    g = torch.Generator("cuda:0").manual_seed(17)
    table, n_pages = tables(rng, lens, page)
    cache = et.KVCache(n_pages, page, kv, d, fmt="mxfp4")
    cache.data.fill_(0xFF)
    rows = sum(lens)
    x = torch.randn((rows, 2 * kv * d), generator=g, device="cuda:0").to(torch.bfloat16)
    q = torch.randn((len(lens), heads * d), generator=g, device="cuda:0").to(torch.bfloat16)
    args = dev(table), dev(np.array(lens, dtype=np.int32))
    cu = dev(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32))
    cache.append(x[:, :kv * d], x[:, kv * d:], *args, cu)
    stand = held(x.reshape(rows, 2, kv, d))
    back = cache.read(*args, cu, rows)
    for j in range(2):
        assert torch.equal(back[j].double(), stand[:, j].flatten(1))
    got = cache.attend(q, *args, max(lens), window=window).double().reshape(len(lens), kv, heads // kv, d)
    at = 0
    for b, n in enumerate(lens):
        lo = at + (max(0, n - window) if window else 0)
        k, v = (stand[lo:at + n, j].transpose(0, 1).contiguous() for j in range(2))           # [kv, tokens, d]
        qb = q[b].double().reshape(kv, heads // kv, d)
        if n == 0:
            assert not got[b].any()
            continue
        w = torch.softmax(qb @ k.transpose(1, 2).contiguous() / math.sqrt(d), -1)
        size = (qb.abs() @ k.abs().transpose(1, 2).contiguous()).amax(-1, keepdim=True) / math.sqrt(d)
        ref, mass = w @ v, w @ v.abs()
        tol = 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2 * (d + 8) * 2.0 ** -24 * 1.45 * size + 2 * n * 2.0 ** -24 + 2.0 ** -21) * mass
        if b % 64 == 0 or len(lens) < 1000:
            assert ((got[b] - ref).abs() <= tol).all(), (b, n, float(((got[b] - ref).abs() - tol).max()))
        at += n


@pytest.mark.parametrize("d", [64, 80, 96, 128, 256])
@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 7, 8, 9, 16, 17])
def test_every_number_of_query_heads_a_key_value_head(group, d):
    """Short sequences, several at once and one alone; parts by eight wavefronts; parts that are joined; a window."""
    for page, kv, lens, window in ((16, 2, [40, 1, 0, 129], 0), (32, 1, [300], 0), (64, 16, [700, 530, 3, 0], 0), (16, 1, [2100, 33], 0), (128, 2, [2500], 1300)):
        test_attention_of_many_and_of_long_sequences(page, kv, kv * group, d, lens, window)


def test_pages_past_four_gigabytes():
    """Pages whose byte offset needs more than 32 bits: stored, read back and attended to."""
    rng = np.random.default_rng(16)
    page, kv, d = 256, 64, 256
    size = et.et_kv_page_bytes(page, kv, d, "mxfp4")                  # 4.25 MiB
    n_pages = 2 ** 32 // size + 40
    cache = et.KVCache(n_pages, page, kv, d, fmt="mxfp4")
    cache.data[:64].fill_(0x5A)
    lens = [300, 5]
    table = np.array([[n_pages - 1, n_pages - 3], [n_pages - 2, -1]], dtype=np.int32)
    x = torch.randn((305, 2, kv, d), generator=torch.Generator("cuda:0").manual_seed(3), device="cuda:0").to(torch.bfloat16)
    k, v = (x[:, j].reshape(305, -1) for j in range(2))
    args = dev(table), dev(np.array(lens, dtype=np.int32))
    cu = dev(np.array([0, 300, 305], dtype=np.int32))
    cache.append(k, v, *args, cu)
    got = cache.read(*args, cu, 305)
    stand = held(x)
    assert all(torch.equal(got[j].double(), stand[:, j].flatten(1)) for j in range(2)) and bool((cache.data[:64] == 0x5A).all())
    q = bf16(rng.normal(size=(2, kv, d)))
    out = dev_to_f64(cache.attend(bits_to_dev(f64_to_bits(q.reshape(2, -1))), *args, 300)).reshape(2, kv, d)
    stand = stand.cpu().numpy()
    for b, (lo, hi) in enumerate(((0, 300), (300, 305))):
        ref, mass, _ = O.attend_one(q[b], stand[lo:hi, 0], stand[lo:hi, 1], 1 / 16)
        assert (np.abs(out[b] - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 1e-4) * mass).all()


def test_a_captured_step_is_replayed_as_the_sequences_grow():
    """Append and attention in one graph with a generous bound; lengths, rows and queries change in place, eager work runs
    between the replays, and a second graph of the same cache replays beside it."""
    rng = np.random.default_rng(22)
    page, kv, heads, d, n = 16, 2, 6, 64, 3
    lens = np.array([30, 1, 250], dtype=np.int32)
    table, n_pages = tables(rng, [900, 900, 900], page)
    cache, eager = (et.KVCache(n_pages, page, kv, d, fmt="mxfp4") for _ in range(2))
    for c in (cache, eager):
        c.data.fill_(0x7A)
    tab, length = dev(table), dev(lens)
    k, v, q = (torch.zeros((n, w * d), dtype=torch.bfloat16, device="cuda:0") for w in (kv, kv, heads))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cache.append(k, v, tab, length)
        cache.attend(q, tab, length, 900)
    torch.cuda.current_stream().wait_stream(side)
    cache.data.fill_(0x7A)
    graphs = []
    for window in (0, 40):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            cache.append(k, v, tab, length)
            out = cache.attend(q, tab, length, 900, window=window)
        graphs.append((g, out, window))
    for step in range(5):
        for t in (k, v, q):
            t.copy_(torch.from_numpy(rng.normal(size=tuple(t.shape))).to(torch.bfloat16))
        length += 100
        for g, out, window in graphs:
            g.replay()
            eager.append(k, v, tab, length)
            ref = eager.attend(q, tab, length, 900, window=window)
            torch.cuda.synchronize()
            assert torch.equal(cache.data, eager.data) and torch.equal(out, ref) and out.any()


def test_calls_on_several_streams_at_once():
    """Two streams attend to one cache at the same time, a third stores into another one."""
    rng = np.random.default_rng(23)
    page, kv, heads, d = 64, 4, 28, 128
    lens = np.array([6000, 300], dtype=np.int32)
    table, n_pages = tables(rng, list(lens), page)
    cache, other = (et.KVCache(n_pages, page, kv, d, fmt="mxfp4") for _ in range(2))
    x = torch.randn((6300, kv * d), generator=torch.Generator("cuda:0").manual_seed(2), device="cuda:0").to(torch.bfloat16)
    args = dev(table), dev(lens)
    cu = dev(np.array([0, 6000, 6300], dtype=np.int32))
    cache.append(x, -x, *args, cu)
    qs = [torch.randn((2, heads * d), device="cuda:0").to(torch.bfloat16) for _ in range(2)]
    ref = [cache.attend(q, *args, 6000) for q in qs]
    minus = -x                                                        # (kept, and done, before another stream reads it)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = [[], []]
    for _ in range(10):
        for i in range(2):
            got[i].append(cache.attend(qs[i], *args, 6000, stream=streams[i]))
        other.append(x, minus, *args, cu, stream=streams[2])
        read = other.read(*args, cu, 6300, stream=streams[2])
    torch.cuda.synchronize()
    assert all(torch.equal(t, ref[i]) for i in range(2) for t in got[i])
    back = cache.read(*args, cu, 6300)
    assert torch.equal(back[0], read[0]) and torch.equal(back[1], read[1]) and torch.equal(back[0], -back[1])


@pytest.mark.parametrize("kv,heads,d,lens,bound", [(8, 8, 80, [700, 650, 900, 1], 1024),      # one part each by eight wavefronts
                                                   (2, 6, 96, [9000, 40, 5000], 9000),         # several parts, joined
                                                   (1, 2, 256, [3000], 3000)])
def test_blocks_that_are_not_numbers_in_long_sequences(kv, heads, d, lens, bound):
    """As above where wavefronts, or parts, are added up: a block of NaN stays in its 32 dimensions of a value and in its head of a key."""
    rng = np.random.default_rng(27)
    page, nb = 16, O.mx_blocks(d)
    table, n_pages = tables(rng, lens, page)
    cache = et.KVCache(n_pages, page, kv, d, fmt="mxfp4")
    x = torch.randn((sum(lens), 2 * kv * d), generator=torch.Generator("cuda:0").manual_seed(27), device="cuda:0").to(torch.bfloat16)
    args = dev(table), dev(np.array(lens, dtype=np.int32))
    cache.append(x[:, :kv * d], x[:, kv * d:], *args, dev(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)))
    q = torch.randn((len(lens), heads * d), generator=torch.Generator("cuda:0").manual_seed(28), device="cuda:0").to(torch.bfloat16)
    clean = dev_to_f64(cache.attend(q, *args, bound)).reshape(len(lens), kv, heads // kv, d)
    host, kept = Pages4(n_pages, page, kv, d), cache.data.clone()
    assert np.isfinite(clean).all()
    for block, pos in ((0, 0), (nb - 1, lens[0] - 1), (nb // 2, lens[0] // 2)):
        for value in (False, True):
            p, at = O.place(pos, table[0], n_pages, page)
            exps = np.arange(host.data.shape[1])[host.cells(at, kv - 1, value)[1]]
            cache.data.copy_(kept)
            cache.data[int(p), int(exps[block])] = 255
            got = dev_to_f64(cache.attend(q, *args, bound)).reshape(clean.shape)
            hit = np.zeros(clean.shape, dtype=bool)
            hit[0, kv - 1] = np.arange(d) // 32 == block if value else True
            assert np.isnan(got[hit]).all() and np.array_equal(got[~hit], clean[~hit])
