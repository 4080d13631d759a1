"""The page pool with the new state in a buffer of its own, where one workgroup gives pages back beside those that fill tables, positions and
places: every step against its definition, the next one from the new state."""
import numpy as np
import pytest
import torch

from oracle import pool_oracle as O
from tests.test_gpu_page_pool import World, ints

pytestmark = pytest.mark.gpu


class Apart(World):
    """Steps alternate between two states; the one that was read stays as it is."""

    def step(self, new, extra=0):
        ring, state, table, cu, positions, slots = O.resize(self.ring, self.state, self.table, self.lens, new, self.page)
        rows, was = len(positions) + extra, self.pool.state
        to = torch.full((4,), -3, dtype=torch.int32, device="cuda:0")
        out = (torch.full((len(new) + 1,), -5, dtype=torch.int32, device="cuda:0"), torch.full((rows,), -5, dtype=torch.int32, device="cuda:0"),
               torch.full((rows,), -5, dtype=torch.int64, device="cuda:0"))
        self.pool.resize(self.dev_table, ints(self.lens), ints(new), rows, state_out=to, out=out)
        n = len(positions)
        assert was.tolist() == self.state and to.tolist() == state, (to.tolist(), state)
        assert self.pool.ring.tolist() == ring and self.dev_table.tolist() == table and bool((self.whole[:, self.wide:] == -7).all())
        assert out[0].tolist() == cu and out[1][:n].tolist() == positions and out[2][:n].tolist() == slots
        assert bool((out[1][n:] == -5).all()) and bool((out[2][n:] == -5).all())
        self.ring, self.state, self.table, self.lens, self.pool.state = ring, state, table, list(new), to
        return state


@pytest.mark.parametrize("n_seqs,wide,page,pages,most", [
    (1, 1, 16, 1, 16), (1, 9, 16, 8, 150), (5, 6, 32, 40, 200), (64, 20, 16, 500, 330), (256, 12, 64, 2000, 800), (1024, 4, 16, 2500, 64),
    (1025, 4, 16, 2500, 64), (3000, 3, 256, 5000, 800), (4096, 3, 32, 7000, 100), (4097, 3, 32, 7000, 100), (9000, 2, 16, 9000, 40),
    (7, 700, 16, 4000, 11000), (2, 3000, 16, 5000, 48000), (9, 1500, 16, 12000, 24000), (1500, 12, 16, 15000, 190), (4500, 4, 16, 16000, 64),
])
def test_steps_that_grow_shrink_and_end(n_seqs, wide, page, pages, most):
    """Random steps, pages missing now and then; up to four turns of pages given back (4096 each) at the end."""
    rng = np.random.default_rng(n_seqs + wide + page + 1)
    lens = [int(x) for x in rng.integers(0, most + 1, n_seqs) * (rng.random(n_seqs) < 0.5)]
    w = Apart(rng, n_seqs, wide, pages, page, lens, pad=int(rng.integers(0, 4)))
    for i in range(12):
        what = rng.random(n_seqs)
        new = [int(rng.integers(0, most + page)) if p < 0.2 else 0 if p < 0.3 else x + 1 if p < 0.8 else x for p, x in zip(what, w.lens)]
        w.step(new, extra=[0, 3, 9000][i % 3])
    w.step([most] * n_seqs)
    given = sum(x >= 0 for row in w.table for x in row)
    state = w.step([0] * n_seqs)
    assert state[1] >= given and state[1] == pages                    # every page is back


def test_many_pages_are_given_while_others_are_taken():
    """More than 4096 entries given back in the step in which as many are taken, more than are free: those given are for the next step."""
    n, wide, page = 40, 700, 16
    rng = np.random.default_rng(3)
    lens = [11000 if i % 2 else 0 for i in range(n)]
    w = Apart(rng, n, wide, 20 * 688 + 3000, page, lens)
    state = w.step([0 if i % 2 else 11000 for i in range(n)])
    assert state[2] == 20 * 688 - 3000 and state[1] == 20 * 688
    state = w.step([0] * n)
    assert state[1:3] == [20 * 688 + 3000, 0]


def test_holes_and_states_that_are_no_states():
    for state in (None, [-5, 3, 0, 0], [17, 3, 1, 1], [2 ** 31 - 1, 4, 0, 0], [0, -1, 0, 0], [3, 10 ** 6, 0, 0]):
        w = Apart(np.random.default_rng(4), 3, 6, 18, 16, [96, 50, 20])
        w.table[0][2], w.table[0][4], w.table[1][1], w.table[2][0] = -1, 99, -2 ** 31, 18
        w.dev_table.copy_(ints(w.table))
        if state is not None:
            w.state = state
            w.pool.state.copy_(ints(state))
        w.step([5, 0, 0])
        w.step([96, 96, 96])
        w.step([0, 0, 1])
