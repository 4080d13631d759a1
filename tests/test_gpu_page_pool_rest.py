"""A resize whose `rows` is a bound: what positions and slots hold behind the last sequence's rows, and that rows stored by them go nowhere else."""
import numpy as np
import pytest
import torch

import paper_2605_30010_amd as et
from oracle import pool_oracle as O
from tests.test_gpu_decoding import D, HEADS, KV, PAGE, Decoder
from tests.test_gpu_page_pool import World, ints

pytestmark = pytest.mark.gpu


def leave_zeros(*sizes):
    """Gives memory of these many bytes back full of zeros: what is allocated next finds places (slot 0) there, as a step before leaves them."""
    held = [torch.zeros(n, dtype=torch.uint8, device="cuda:0") for n in sizes for _ in range(3)]
    del held


def used_sizes(n, rows):
    """Bytes of cu_rows, positions and slots, in one piece and each."""
    each = [(x + 127) // 128 * 128 for x in (4 * (n + 1), 4 * rows, 8 * rows)]
    return [sum(each)] + each


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("apart", [True, False])
@pytest.mark.parametrize("n,extra", [(1, 1), (5, 3), (5, 9000), (64, 70000), (1024, 1), (1100, 500), (4096, 3000), (4200, 1), (4200, 9000), (0, 5)])
def test_rows_behind_the_last_sequences_have_no_place(n, extra, apart, native):
    rng = np.random.default_rng(n + extra)
    lens = [int(x) for x in rng.integers(0, 60, n)]
    w = World(rng, n, 8, 8 * n + 3, 16, lens)
    new = [int(rng.integers(0, 60)) if p < 0.3 else 0 if p < 0.6 else x for p, x in zip(rng.random(n), lens)]
    ring, state, table, cu, positions, slots = O.resize(w.ring, w.state, w.table, lens, new, 16)
    total = len(positions)
    rows = total + extra
    if not native:
        w.pool._calls = None
    to = torch.zeros(4, dtype=torch.int32, device="cuda:0") if apart else None
    leave_zeros(*used_sizes(n, rows))
    got = w.pool.resize(w.dev_table, ints(lens), ints(new), rows, state_out=to)
    same = lambda t, x: np.array_equal(t.cpu().numpy(), np.array(x).reshape(t.shape))
    assert same(got[0], cu) and same(w.pool.state if to is None else to, state) and same(w.pool.ring, ring) and same(w.dev_table, table)
    assert same(got[1], positions + [0] * extra)
    assert same(got[2], slots + [-1] * extra)


def test_no_new_token_at_all():
    for n in (3, 1100, 4200):
        w = World(np.random.default_rng(1), n, 4, 4 * n, 16, [20] * n)
        for new in ([20] * n, [3] * n, [0] * n):
            leave_zeros(*used_sizes(n, 300))
            cu, positions, slots = w.pool.resize(w.dev_table, ints([20] * n), ints(new), 300, state_out=torch.zeros_like(w.pool.state))
            assert not cu.any() and not positions.any() and bool((slots == -1).all()), n


def test_lengths_without_end_fill_the_rows():
    """More new tokens than 32 bits count: there is no row behind them."""
    w = World(np.random.default_rng(2), 3, 2, 20, 16, [5, 0, 40])
    cu, positions, slots = w.pool.resize(w.dev_table, ints([0, 0, 0]), ints([2 ** 31 - 1] * 3), 5000, state_out=torch.zeros_like(w.pool.state))
    assert cu.tolist() == [0] + [2 ** 31 - 1] * 3 and positions.tolist() == list(range(5000)) and bool((slots[32:] == -1).all())


class Steps:
    """A cache and its pool, whose sequences grow by a token, end, are idle, or are let in again."""

    def __init__(self, n, fmt):
        self.n, self.page, wide = n, 16, 6
        self.pool = et.PagePool(wide * n, self.page)
        self.cache = et.KVCache(wide * n, self.page, 2, 64, fmt=fmt)
        self.cache.data.fill_(0x5B)
        self.table = torch.full((n, wide), -1, dtype=torch.int32, device="cuda:0")
        self.len = torch.zeros(n, dtype=torch.int32, device="cuda:0")


def next_lengths(rng, lens, step):
    """Most sequences get a token; some end, some stay as they are, some start over with one."""
    p = rng.random(len(lens))
    return [1 if x == 0 and a < 0.5 else 0 if a < 0.25 else x if a < 0.4 or x == 0 else x + 1 for a, x in zip(p, lens)] if step else [1] * len(lens)


@pytest.mark.parametrize("fmt", ["bf16", "int8", "mxfp4"])
@pytest.mark.parametrize("n", [6, 1100, 4200])
def test_a_bound_stores_every_row_once(n, fmt):
    """Step by step against a cache whose rows are stored by ranges (append) of the exact number; the whole cache is compared."""
    rng = np.random.default_rng(n)
    a, b = Steps(n, fmt), Steps(n, fmt)
    lens, less = [0] * n, 0
    for step in range(8):
        new = next_lengths(rng, lens, step)
        rows = sum(max(y - x, 0) for x, y in zip(lens, new))
        less += rows < n
        x = torch.randn((2, n, 128), device="cuda:0").to(torch.bfloat16)
        _, _, slots = a.pool.resize(a.table, a.len, ints(new), n)
        a.cache.append_at(x[0], x[1], slots)
        del slots
        cu, *_ = b.pool.resize(b.table, b.len, ints(new), rows)
        b.cache.append(x[0, :rows], x[1, :rows], b.table, ints(new), cu)
        for s in (a, b):
            s.len.copy_(ints(new))
        assert torch.equal(a.table, b.table) and torch.equal(a.cache.data, b.cache.data), step
        lens = new
    assert less >= 6


@pytest.mark.parametrize("n", [6, 1100, 4200])
def test_a_captured_step_with_a_bound(n):
    """The same by replays of one graph, in which `rows` cannot change, with eager work between them."""
    rng = np.random.default_rng(n + 1)
    a, b = Steps(n, "mxfp4"), Steps(n, "mxfp4")
    x, want = torch.zeros((2, n, 128), dtype=torch.bfloat16, device="cuda:0"), torch.zeros(n, dtype=torch.int32, device="cuda:0")

    def body():
        _, _, slots = a.pool.resize(a.table, a.len, want, n)
        a.cache.append_at(x[0], x[1], slots)
        a.len.copy_(want)

    keep = [t.clone() for t in (a.pool.state, a.pool.ring, a.table, a.len, a.cache.data)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        body()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        body()
    for t, was in zip((a.pool.state, a.pool.ring, a.table, a.len, a.cache.data), keep):
        t.copy_(was)
    lens = [0] * n
    for step in range(8):
        new = next_lengths(rng, lens, step)
        rows = sum(max(q - p, 0) for p, q in zip(lens, new))
        x.copy_(torch.randn((2, n, 128), device="cuda:0"))
        want.copy_(ints(new))
        g.replay()
        cu, *_ = b.pool.resize(b.table, b.len, ints(new), rows)
        b.cache.append(x[0, :rows], x[1, :rows], b.table, ints(new), cu)
        b.len.copy_(ints(new))
        torch.cuda.synchronize()
        assert torch.equal(a.table, b.table) and torch.equal(a.cache.data, b.cache.data), step
        lens = new
        torch.ones(1000, device="cuda:0").sum()


def test_the_whole_step_with_a_bound():
    """Pages, positions, storing and attention with `rows` one for each sequence, whether it has a token or not, against the exact number."""
    rng = np.random.default_rng(5)
    n = 5
    a, b = (Decoder(n, 8, 8 * n, "mxfp4") for _ in range(2))
    lens = [0] * n
    for step in range(8):
        new = next_lengths(rng, lens, step)
        rows = sum(max(y - x, 0) for x, y in zip(lens, new))
        cu = np.concatenate([[0], np.cumsum([max(y - x, 0) for x, y in zip(lens, new)])])
        last = torch.from_numpy(np.maximum(cu[1:] - 1, 0)).to("cuda:0")
        x = torch.randn((n, (HEADS + 2 * KV) * D), device="cuda:0").to(torch.bfloat16)
        q, _, _ = a.store(ints(new), n, x)
        q2, _, _ = b.store(ints(new), rows, x[:rows])
        assert torch.equal(q[:rows], q2) and torch.equal(a.cache.data, b.cache.data) and torch.equal(a.table, b.table)
        out = a.attend(q[last], 8 * PAGE)
        assert torch.equal(out, b.attend(q2[last.clamp(max=rows - 1)] if rows else torch.zeros_like(q), 8 * PAGE))
        assert [bool(t.any()) for t in out] == [m > 0 for m in new]
        lens = new
