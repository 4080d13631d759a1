"""The page pool on the device against its definition: whole numbers, all equal."""
import numpy as np
import pytest
import torch

import paper_2605_30010_amd as et
from oracle import pool_oracle as O
from tests.test_gpu_kv import dev

pytestmark = pytest.mark.gpu


def ints(x):
    return dev(np.array(x, dtype=np.int32))


class World:
    """Sequences, their table and the pool, on the device and as lists."""

    def __init__(self, rng, n_seqs, wide, n_pages, page, lens, pad=0):
        self.page, self.wide, self.n = page, wide, n_pages
        free = list(rng.permutation(n_pages))
        self.table = [[-1] * wide for _ in range(n_seqs)]
        for row, m in zip(self.table, lens):
            for i in range(min(-(-m // page), wide)):
                row[i] = int(free.pop()) if free else -1
        first = int(rng.integers(0, n_pages))
        self.ring = [-9] * n_pages
        for i, x in enumerate(free):
            self.ring[(first + i) % n_pages] = int(x)
        self.state, self.lens = [first, len(free), 0, 0], list(lens)
        whole = torch.full((max(n_seqs, 1), wide + pad), -7, dtype=torch.int32, device="cuda:0")
        self.whole, self.dev_table = whole, whole[:n_seqs, :wide]
        if n_seqs:
            self.dev_table.copy_(ints(self.table))
        self.pool = et.PagePool(n_pages, page, ring=ints(self.ring), state=ints(self.state))

    def step(self, new, rows=None, extra=0):
        """Resizes both; compares everything."""
        ring, state, table, cu, positions, slots = O.resize(self.ring, self.state, self.table, self.lens, new, self.page)
        rows = len(positions) + extra if rows is None else rows
        out = (torch.full((len(new) + 1,), -5, dtype=torch.int32, device="cuda:0"), torch.full((rows,), -5, dtype=torch.int32, device="cuda:0"),
               torch.full((rows,), -5, dtype=torch.int64, device="cuda:0"))
        old, want = ints(self.lens), ints(new)
        got = self.pool.resize(self.dev_table, old, want, rows, out=out)
        assert got is out
        assert old.tolist() == list(self.lens) and want.tolist() == list(new)
        assert self.pool.state.tolist() == state, (self.pool.state.tolist(), state)
        assert self.pool.ring.tolist() == ring and self.dev_table.tolist() == table
        assert bool((self.whole[:, self.wide:] == -7).all())
        assert out[0].tolist() == cu
        n = min(rows, len(positions))
        assert out[1][:n].tolist() == positions[:n] and out[2][:n].tolist() == slots[:n]
        assert bool((out[1][n:] == -5).all()) and bool((out[2][n:] == -5).all())
        self.ring, self.state, self.table, self.lens = ring, state, table, list(new)


@pytest.mark.parametrize("n_seqs,wide,page,pages,most", [
    (1, 1, 16, 1, 16), (1, 9, 16, 8, 150), (5, 6, 32, 40, 200), (64, 20, 16, 500, 330), (65, 3, 64, 150, 200), (256, 12, 64, 2000, 800),
    (1024, 4, 16, 2500, 64), (1025, 4, 16, 2500, 64), (3000, 3, 256, 5000, 800), (4096, 3, 32, 7000, 100), (4097, 3, 32, 7000, 100), (9000, 2, 16, 9000, 40), (7, 700, 16, 4000, 11000), (2, 3000, 16, 5000, 48000),
])
def test_steps_that_grow_shrink_and_end(n_seqs, wide, page, pages, most):
    """Random steps with pages missing now and then, lengths past the table's end among them; all forms (up to 1024, up to 4096 and more
    sequences, a few rows and thousands)."""
    rng = np.random.default_rng(n_seqs + wide + page)
    lens = [int(x) for x in rng.integers(0, most + 1, n_seqs) * (rng.random(n_seqs) < 0.5)]
    w = World(rng, n_seqs, wide, pages, page, lens, pad=int(rng.integers(0, 4)))
    for i in range(12):
        what = rng.random(n_seqs)
        new = [int(rng.integers(0, most + page)) if p < 0.2 else 0 if p < 0.3 else x + 1 if p < 0.8 else x for p, x in zip(what, w.lens)]
        w.step(new, extra=[0, 3, 9000][i % 3])
    w.step([0] * n_seqs)
    assert w.lens == [0] * n_seqs


def test_no_sequences_and_empty_ones():
    rng = np.random.default_rng(2)
    w = World(rng, 0, 4, 5, 16, [])
    w.step([], rows=3)
    w = World(rng, 4, 4, 5, 16, [0, 0, 0, 0])
    w.step([0, 0, 0, 0], rows=2)
    w.step([-3, 1, -2 ** 31, 0])
    w.step([17, 1, 5, -1])


def test_fewer_rows_than_new_tokens():
    """positions and slots end where the caller says; pages are given all the same."""
    for n, rows in ((4, 0), (4, 7), (4, 100), (1100, 50), (4200, 50)):
        rng = np.random.default_rng(rows)
        w = World(rng, n, 8, n * 4, 16, [int(x) for x in rng.integers(0, 30, n)])
        w.step([x + int(rng.integers(0, 60)) for x in w.lens], rows=rows)


def test_tables_that_are_too_short_and_lengths_without_end():
    """A length past the table takes the pages that the table has room for; the places behind it are none."""
    w = World(np.random.default_rng(3), 3, 2, 20, 16, [5, 0, 40])
    w.step([100, 33, 7], rows=200)
    w.step([31, 32, 2000], rows=3000)
    new, state = [10, 2 ** 31 - 1, 5], torch.zeros(4, dtype=torch.int32, device="cuda:0")
    cu, positions, slots = w.pool.resize(w.dev_table, ints(w.lens), ints(new), 64, state_out=state)
    assert cu.tolist() == [0, 0, 2 ** 31 - 1 - 32, 2 ** 31 - 1 - 32] and positions.tolist() == list(range(32, 96)) and slots.tolist() == [-1] * 64
    cu, *_ = w.pool.resize(w.dev_table, ints([0, 0, 0]), ints([2 ** 31 - 1] * 3), 4, state_out=state)
    assert cu.tolist() == [0] + [2 ** 31 - 1] * 3


def test_holes_and_strange_entries_give_nothing_back():
    w = World(np.random.default_rng(4), 3, 6, 18, 16, [96, 50, 20])
    w.table[0][2], w.table[0][4], w.table[1][1], w.table[2][0] = -1, 99, -2 ** 31, 18
    w.dev_table.copy_(ints(w.table))
    w.step([5, 0, 0])
    w.step([96, 96, 96])


def test_states_that_are_no_states():
    """Whatever the state says, ring, table and results are those of the definition, and nothing outside is touched."""
    for state in ([-5, 3, 0, 0], [17, 3, 1, 1], [2 ** 31 - 1, 4, 0, 0], [0, -1, 0, 0], [3, 10 ** 6, 0, 0], [-2 ** 31, 2 ** 31 - 1, 0, 0]):
        w = World(np.random.default_rng(5), 4, 5, 8, 16, [30, 0, 70, 16])
        w.state = state
        w.pool.state.copy_(ints(state))
        w.step([31, 40, 0, 64])
        w.step([0, 0, 0, 0])


@pytest.mark.parametrize("n,most", [(6, 100), (6, 4000), (1100, 40), (4200, 20)])
def test_a_call_is_taken_back_by_the_old_state(n, most):
    """With its state elsewhere, a call (one that lacks pages) changes nothing that the old state and lengths reach: another one
    follows as if it had not been."""
    rng = np.random.default_rng(6)
    lens = [int(x) for x in rng.integers(0, most, n)]
    pages = sum(-(-x // 16) for x in lens) + 5
    w = World(rng, n, -(-2 * most // 16), pages, 16, lens)
    other = torch.zeros(4, dtype=torch.int32, device="cuda:0")
    for _ in range(3):
        new = [int(x) for x in rng.integers(0, 2 * most, n)]
        w.pool.resize(w.dev_table, ints(w.lens), ints(new), sum(max(b - a, 0) for a, b in zip(w.lens, new)), state_out=other)
    assert w.pool.state.tolist() == w.state and other.tolist() != w.state
    # dead cells and entries hold what the calls left there: the definition goes on from these
    ring, table = w.pool.ring.tolist(), w.dev_table.tolist()
    free = [(w.state[0] + i) % pages for i in range(w.state[1])]
    assert [ring[c] for c in free] == [w.ring[c] for c in free]
    assert all(a[:-(-m // 16)] == b[:-(-m // 16)] for a, b, m in zip(table, w.table, w.lens))
    w.ring, w.table = ring, table
    w.step([x + 1 for x in w.lens])


def test_positions_or_slots_alone():
    """NULL for either at the C boundary."""
    import ctypes as C
    from paper_2605_30010_amd import binding as B
    lib = et.load_library()
    for n in (3, 1100, 4200):
        for keep in ((True, False), (False, True), (False, False)):
            w = World(np.random.default_rng(7), n, 4, 4 * n, 16, [3] * n)
            new = [20] * n
            ring, state, table, cu, positions, slots = O.resize(w.ring, w.state, w.table, w.lens, new, 16)
            old, want, cu_dev = ints(w.lens), ints(new), torch.zeros(n + 1, dtype=torch.int32, device="cuda:0")
            p = torch.zeros(len(positions), dtype=torch.int32, device="cuda:0")
            s = torch.zeros(len(positions), dtype=torch.int64, device="cuda:0")
            ws = torch.zeros(1 << 17, dtype=torch.uint8, device="cuda:0")
            rc = lib.et_kv_resize(C.byref(w.pool._pool), w.pool.state.data_ptr(), w.pool.state.data_ptr(), w.dev_table.data_ptr(), 4, 4, old.data_ptr(),
                                  want.data_ptr(), n, len(positions), cu_dev.data_ptr(), p.data_ptr() if keep[0] else None,
                                  s.data_ptr() if keep[1] else None, ws.data_ptr(), ws.numel(), B._raw_stream(0))
            torch.cuda.synchronize()
            assert rc == 0 and cu_dev.tolist() == cu and w.pool.state.tolist() == state and w.dev_table.tolist() == table
            assert p.tolist() == (positions if keep[0] else [0] * len(positions)) and s.tolist() == (slots if keep[1] else [0] * len(slots))


@pytest.mark.parametrize("n", [5, 1100, 4200])
def test_a_captured_step_takes_a_page_when_it_needs_one(n):
    """Replays of one graph, in which the lengths are counted up too, against the definition; eager work between them."""
    rng = np.random.default_rng(8)
    page = 16
    lens = [int(x) for x in rng.integers(0, 40, n)]
    w = World(rng, n, 8, 8 * n, page, lens)
    old, one = ints(lens), torch.ones(n, dtype=torch.int32, device="cuda:0")
    keep = w.pool.state.clone(), w.pool.ring.clone(), w.dev_table.clone(), old.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def body():
        new = old + one
        out = w.pool.resize(w.dev_table, old, new, n)
        old.copy_(new)
        return out

    with torch.cuda.stream(side):
        body()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cu, positions, slots = body()
    for t, k in zip((w.pool.state, w.pool.ring, w.dev_table, old), keep):
        t.copy_(k)
    for step in range(20):
        g.replay()
        new = [x + 1 for x in lens]
        ring, state, table, ref_cu, ref_pos, ref_slots = O.resize(w.ring, w.state, w.table, lens, new, page)
        torch.cuda.synchronize()
        assert (cu.tolist(), positions.tolist(), slots.tolist()) == (ref_cu, ref_pos, ref_slots)
        assert w.pool.state.tolist() == state and w.dev_table.tolist() == table and old.tolist() == new
        w.ring, w.state, w.table, lens = ring, state, table, new
        torch.ones(1000, device="cuda:0").sum()


def test_default_pool_and_refusals():
    pool = et.PagePool(10, 16)
    assert pool.ring.tolist() == list(range(10)) and pool.state.tolist() == [0, 10, 0, 0]
    tab, old, new = torch.full((3, 4), -1, dtype=torch.int32, device="cuda:0"), ints([0, 0, 0]), ints([20, 0, 16])
    cu, positions, slots = pool.resize(tab, old, new, 36)
    assert cu.tolist() == [0, 20, 20, 36] and tab.tolist() == [[0, 1, -1, -1], [-1] * 4, [2, -1, -1, -1]] and pool.state.tolist() == [3, 7, 0, 0]
    assert slots.tolist() == list(range(20)) + list(range(32, 48))
    for bad in (tab.long(), tab.cpu()):
        with pytest.raises(TypeError):
            pool.resize(bad, old, new, 3)
    with pytest.raises(TypeError):
        pool.resize(tab, old.long(), new, 3)
    for args in ((tab[0], old, new), (tab.t(), old, new), (tab[:2], old, new), (tab, old, new[:2]), (tab, old.repeat(2)[::2], new)):
        with pytest.raises(ValueError):
            pool.resize(*args, 3)
    for extra in (dict(rows=-1), dict(rows=2 ** 31), dict(rows=3, state_out=ints([0, 0])), dict(rows=3, out=(old, old, old))):
        with pytest.raises(ValueError):
            pool.resize(tab, old, new, **extra)
    with pytest.raises(ValueError):
        et.PagePool(10, 16, ring=ints([0, 1]))


@pytest.mark.parametrize("fmt", ["bf16", "int8", "mxfp4"])
def test_rows_at_slots_are_rows_at_their_places(fmt):
    """append_at with the slots of a resize stores what append does; slots that are none store nothing."""
    rng = np.random.default_rng(9)
    w = World(rng, 4, 6, 9, 16, [3, 0, 40, 17])
    new = [30, 20, 41, 90]                                            # pages are missing for the last
    old, want = ints(w.lens), ints(new)
    rows = sum(b - a for a, b in zip(w.lens, new))
    cu, positions, slots = w.pool.resize(w.dev_table, old, want, rows)
    assert w.pool.state.tolist()[2] > 0 and (slots < 0).any() and (slots >= 0).any()
    caches = [et.KVCache(9, 16, 2, 64, fmt=fmt) for _ in range(2)]
    for c in caches:
        c.data.fill_(0x5B)
    k, v = (torch.randn((rows, 128), device="cuda:0").to(torch.bfloat16) for _ in range(2))
    caches[0].append(k, v, w.dev_table, want, cu)
    caches[1].append_at(k, v, slots)
    assert torch.equal(caches[0].data, caches[1].data) and not bool((caches[1].data == 0x5B).all())
    strange = slots.clone()
    strange[:5] = torch.tensor([-1, 9 * 16, 2 ** 40, -2 ** 63, 2 ** 63 - 1], device="cuda:0")
    before = caches[1].data.clone()
    caches[1].append_at(k[:5], v[:5], strange[:5].contiguous())
    assert torch.equal(before, caches[1].data)
    for bad in (slots.int(), slots.cpu()):
        with pytest.raises(TypeError):
            caches[1].append_at(k, v, bad)
    for bad in (slots[1:], slots[None]):
        with pytest.raises(ValueError):
            caches[1].append_at(k, v, bad)
    with pytest.raises(ValueError):
        caches[1].append_at(k, v[:3], slots)
