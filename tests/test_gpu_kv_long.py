"""Attention over the paged cache where sequences are cut into parts: every token counts once, keys and values are of the same token, more than
16 query heads per key-value head, and steps captured while sequences go from one part to several."""
import numpy as np
import pytest
import torch

import paper_2605_30010_amd as et
from tests._util import bits_to_dev, dev_to_f64, f64_to_bits
from tests.test_gpu_kv import dev, tables

pytestmark = pytest.mark.gpu


def lengths(lens):
    return dev(np.array(lens, dtype=np.int32))


def stored(fmt, page, kv, d, lens, k, v, rng, holes=()):
    """A cache that holds rows k, v (device, [sum of lens, kv * d]); everything else in it is NaN."""
    table, n_pages = tables(rng, lens, page, holes=holes)
    cache = et.KVCache(n_pages, page, kv, d, fmt=fmt)
    cache.data.fill_(0xFF)
    cache.append(k, v, dev(table), lengths(lens), dev(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)))
    return cache, dev(table)


SPLIT = [  # format, page, kv heads, heads, head width, lengths, window
    ("bf16", 16, 8, 8, 64, [45000], 0),                                            # one sequence: parts of consecutive blocks
    ("int8", 64, 4, 28, 128, [9001, 3, 5000, 0, 131, 513], 0),
    ("e4m3", 128, 8, 32, 128, [20000, 16384, 1000, 7777], 0),
    ("bf16", 32, 16, 16, 96, [40000, 1, 33000, 0, 12000, 300, 39999], 0),          # long parts, and shorter ones in their place
    ("int8", 16, 64, 64, 64, [45000], 0),                                          # parts of more than 64 groups of 16 tokens a wavefront
    ("e4m3", 64, 32, 32, 80, [61000, 61003, 4], 0),
    ("bf16", 16, 2, 2, 64, [600, 0, 513, 1000, 12] * 30, 0),                       # lengths scanned in three steps
    ("bf16", 16, 2, 8, 64, [3000, 0, 513, 9000, 12], 2500),
    ("int8", 16, 1, 16, 128, [12000], 12000 - 5),
    # more than 16 query heads per key-value head
    ("bf16", 32, 1, 20, 256, [3000, 2999, 513, 0, 1, 9001, 700], 1024),
    ("bf16", 64, 1, 17, 128, [5000], 0),
    ("int8", 16, 2, 40, 64, [5000], 0),
    ("e4m3", 32, 3, 99, 80, [2500, 700, 1], 0),
    ("bf16", 16, 5, 85, 64, [1500] * 9, 0),                                        # several full turns of eight places and a partial one
    ("e4m3", 256, 1, 33, 96, [4000, 4000, 4000], 900),
    ("int8", 64, 1, 128, 128, [10000, 2], 0),
    ("bf16", 16, 1, 33, 64, [1, 600, 30, 512] * 25, 0),
]


@pytest.mark.parametrize("fmt,page,kv,heads,d,lens,window", SPLIT)
@pytest.mark.parametrize("bound", ["exact", "generous"])
def test_every_token_counts_once(fmt, page, kv, heads, d, lens, window, bound):
    """Keys of zero: every weight is 1 / n.  Token t's value is 1 in dimension t of the kv * d that the key-value heads have
    together (t modulo their number) and 0 elsewhere, so each result is the number of visible tokens of its class by n.  A token
    lost or counted twice moves a class of c <= 100 tokens by more than twice the bound: (1 - c / n) / n > 2 * 2^-8 c / n."""
    rng = np.random.default_rng(41)
    classes, rows = kv * d, sum(lens)
    pos = torch.cat([torch.arange(n, device="cuda:0") for n in lens])
    v = torch.zeros((rows, classes), dtype=torch.bfloat16, device="cuda:0")
    v[torch.arange(rows, device="cuda:0"), pos % classes] = 1.0
    cache, table = stored(fmt, page, kv, d, lens, torch.zeros_like(v), v, rng)
    q = torch.randn((len(lens), heads * d), device="cuda:0").to(torch.bfloat16)
    if bound == "generous":
        table = torch.cat([table, torch.full((len(lens), 4000), -1, dtype=torch.int32, device="cuda:0")], 1)
    most = max(lens) if bound == "exact" else table.shape[1] * page
    got = dev_to_f64(cache.attend(q, table, lengths(lens), most, window=window)).reshape(len(lens), kv, heads // kv, d)
    for b, n in enumerate(lens):
        lo = max(0, n - window) if window else 0
        count = np.bincount(np.arange(lo, n) % classes, minlength=classes).reshape(kv, 1, d)
        assert count.max() <= 100
        # The weights, their sum and the sums of values are exact; a division, a factor of 8-bit formats, a product and exp2(0) in
        # float32, the 2^-20 that is added to a weight, and the result's rounding are not.
        ref = count / max(n - lo, 1)
        off = np.abs(got[b] - ref) - ref * (2.0 ** -8 + 2.0 ** -19)
        assert (off <= 0).all(), (b, n, np.argwhere(off > 0)[:5])


@pytest.mark.parametrize("fmt,page,kv,heads,d,n,window", [
    ("bf16", 16, 1, 16, 64, 9001, 0), ("int8", 64, 2, 34, 64, 5000, 0), ("e4m3", 32, 1, 20, 80, 7000, 0), ("bf16", 128, 4, 16, 128, 20000, 0),
    ("int8", 256, 1, 40, 256, 6000, 3000), ("e4m3", 16, 8, 8, 96, 33333, 0), ("bf16", 16, 1, 4, 64, 500, 0), ("int8", 16, 1, 17, 128, 513, 0),
])
def test_a_single_token_is_found_at_every_cut(fmt, page, kv, heads, d, n, window):
    """One key per dimension stands out, at the first and last tokens of groups, tiles, blocks and parts, at both ends of the
    sequence and of the window; query head h asks for one of them, and its result is that token's value.  As one sequence
    alone, and as several that share their pages."""
    rng = np.random.default_rng(42)
    lo = max(0, n - window) if window else 0
    cuts = {lo, n - 1, lo + 1, n - 2}
    edges = [c + e for c in range(lo // 128 * 128, n, 128) for e in (-1, 0, 1, 15, 16, 31, 32) if lo <= c + e < n]
    cuts |= set(rng.choice(edges, min(d - len(cuts), len(edges)), replace=False).tolist())
    cuts = sorted(cuts)[:d]
    k = torch.zeros((n, kv, d), dtype=torch.bfloat16, device="cuda:0")
    for i, pos in enumerate(cuts):
        k[pos, :, i] = 8.0
    if lo:
        k[lo - 1] = 8.0                                                # in front of the window: would win everywhere
    v = torch.from_numpy(rng.normal(size=(n, kv, d))).to(torch.bfloat16).to("cuda:0")
    cache, table = stored(fmt, page, kv, d, [n], k.flatten(1), v.flatten(1), rng)
    held = v.double().cpu().numpy()
    if fmt != "bf16":
        m = np.abs(held).max(-1, keepdims=True)
        y = torch.from_numpy(held * {"int8": 127.0, "e4m3": 448.0}[fmt] / m)
        y = torch.round(y) if fmt == "int8" else y.float().to(torch.float8_e4m3fn).double()
        held = y.numpy() * m / {"int8": 127.0, "e4m3": 448.0}[fmt]
    seqs = -(-len(cuts) // heads) + 1
    want = (np.arange(seqs)[:, None] * heads + np.arange(heads)) % len(cuts)             # the cut that sequence b's head h asks for
    q = np.zeros((seqs, heads, d))
    np.put_along_axis(q, want[..., None], 8.0, -1)
    q = bits_to_dev(f64_to_bits(q.reshape(seqs, -1)))
    ref = held[np.array(cuts)[want], np.arange(heads) // (heads // kv)]                   # [seqs, heads, d]
    # scale 1: a logit of 64 against 0, n weights of e^-64 and values below 8 beside it; weight and sum as above
    tol = np.abs(ref) * (2.0 ** -8 + 2.0 ** -19) + 8 * n * np.exp(-64.0)
    together = cache.attend(q, table.repeat(seqs, 1), lengths([n] * seqs), n, window=window, scale=1.0)
    assert (np.abs(dev_to_f64(together).reshape(ref.shape) - ref) <= tol).all()
    for b in range(seqs):
        alone = cache.attend(q[b:b + 1], table, lengths([n]), n, window=window, scale=1.0)
        assert (np.abs(dev_to_f64(alone).reshape(ref[b].shape) - ref[b]) <= tol[b]).all(), b


@pytest.mark.parametrize("window", [0, 700])
def test_more_than_4096_sequences(window):
    """One part each, under a bound of many blocks; a few long ones among them."""
    rng = np.random.default_rng(43)
    lens = rng.integers(0, 40, 5000)
    lens[[0, 77, 2500, 4999]] = 3000, 1, 2900, 2049
    lens = lens.tolist()
    pos = torch.cat([torch.arange(n, device="cuda:0") for n in lens])
    v = torch.zeros((len(pos), 64), dtype=torch.bfloat16, device="cuda:0")
    v[torch.arange(len(pos), device="cuda:0"), pos % 64] = 1.0
    cache, table = stored("bf16", 16, 1, 64, lens, torch.zeros_like(v), v, rng)
    q = torch.randn((5000, 2 * 64), device="cuda:0").to(torch.bfloat16)
    got = dev_to_f64(cache.attend(q, table, lengths(lens), 3000, window=window)).reshape(5000, 2, 64)
    for b, n in enumerate(lens):
        lo = max(0, n - window) if window else 0
        ref = np.bincount(np.arange(lo, n) % 64, minlength=64) / max(n - lo, 1)
        assert (np.abs(got[b] - ref) <= ref * (2.0 ** -8 + 2.0 ** -19)).all(), (b, n)


@pytest.mark.parametrize("fmt,kv,heads,d,page", [("bf16", 2, 6, 64, 16), ("int8", 1, 20, 128, 64), ("e4m3", 4, 28, 80, 32)])
def test_captured_steps_follow_the_lengths_from_one_part_to_several(fmt, kv, heads, d, page):
    """Append and attention in graphs with a bound of 4096 tokens, whose workspaces and joins are captured with them; lengths move
    from a few tokens to thousands and back between the replays, eager calls on the same cache run in between."""
    rng = np.random.default_rng(44)
    n, bound = 3, 4096
    g = torch.Generator("cuda:0").manual_seed(44)
    x = torch.randn((n * bound, 2 * kv * d), generator=g, device="cuda:0").to(torch.bfloat16)
    cache, tab = stored(fmt, page, kv, d, [bound] * n, x[:, :kv * d], x[:, kv * d:], rng)
    eager = et.KVCache(cache.n_pages, page, kv, d, fmt=fmt, data=cache.data.clone())
    length = lengths([1, 1, 1])
    k, v, q = (torch.zeros((n, w * d), dtype=torch.bfloat16, device="cuda:0") for w in (kv, kv, heads))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cache.append(k, v, tab, length)
        cache.attend(q, tab, length, bound)
    torch.cuda.current_stream().wait_stream(side)
    cache.data.copy_(eager.data)
    graphs = []
    for window in (0, 700):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cache.append(k, v, tab, length)
            out = cache.attend(q, tab, length, bound, window=window)
        graphs.append((graph, out, window))
    for lens in ([100, 1, 0], [128, 129, 130], [2000, 5, 700], [4096, 4095, 4000], [3, 4096, 2], [513, 0, 1025], [1, 1, 1]):
        for t in (k, v, q):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda:0"))
        length.copy_(lengths(lens))
        outs = []
        for graph, out, window in graphs:
            graph.replay()
            eager.append(k, v, tab, length)
            ref = eager.attend(q, tab, length, bound, window=window)
            again = cache.attend(q, tab, length, bound, window=window)
            outs.append((out.clone(), ref, again))
        torch.cuda.synchronize()
        assert torch.equal(cache.data, eager.data)
        for out, ref, again in outs:
            assert torch.equal(out, ref) and torch.equal(out, again)
            assert all(bool(out[b].any()) == (m > 0) for b, m in enumerate(lens))
