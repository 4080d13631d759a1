"""The page pool without a GPU: its definition's own properties, workspace sizes, and what is refused."""
import numpy as np
import pytest
import torch

import ctypes as C

import paper_2605_30010_amd as et
from oracle import pool_oracle as O
from paper_2605_30010_amd import binding as B


def test_the_definition_keeps_every_page_in_one_place():
    rng = np.random.default_rng(1)
    n, page, wide = 40, 16, 12
    ring, state, table = list(rng.permutation(n)), [7, n, 0, 0], [[-1] * wide for _ in range(6)]
    lens = [0] * 6
    for _ in range(200):
        new = [int(rng.integers(0, wide * page + 1)) if rng.random() < 0.4 else x for x in lens]
        ring, state, table, cu, positions, slots = O.resize(ring, state, table, lens, new, page)
        lens = new
        live = [x for row, m in zip(table, lens) for x in row[:-(-m // page)] if x >= 0]
        free = [ring[(state[0] + i) % n] for i in range(state[1])]
        assert sorted(live + free) == list(range(n)) and cu[-1] == len(positions) == len(slots)
        assert len(set(s for s in slots if s >= 0)) == sum(s >= 0 for s in slots)


FAKE = 4096                                              # never dereferenced


def call(pool=None, state=FAKE, state_out=FAKE, table=FAKE, stride=4, pages=4, old=FAKE, new=FAKE, n=3, rows=5, cu=FAKE, pos=FAKE, slots=FAKE,
         ws=FAKE, ws_bytes=1 << 40):
    p = B._KvPool(**dict(dict(ring_dev=FAKE, n_pages=8, page_size=16), **(pool or {})))
    return et.load_library().et_kv_resize(C.byref(p), state, state_out, table, stride, pages, old, new, n, rows, cu, pos, slots, ws, ws_bytes, None)


@pytest.mark.parametrize("bad", [dict(pool=dict(ring_dev=None)), dict(pool=dict(n_pages=0)), dict(pool=dict(n_pages=-3)), dict(pool=dict(page_size=8)),
                                 dict(pool=dict(page_size=48)), dict(pool=dict(page_size=512)), dict(pool=dict(page_size=0)), dict(state=None),
                                 dict(state=FAKE + 8), dict(state_out=None), dict(state_out=FAKE + 4), dict(table=None), dict(old=None), dict(new=None),
                                 dict(n=-1), dict(n=2 ** 20 + 1), dict(stride=3), dict(pages=0), dict(pages=1 << 27, stride=1 << 27),
                                 dict(n=1 << 16, pages=1 << 15, stride=1 << 15), dict(rows=-1), dict(cu=None), dict(slots=FAKE + 4),
                                 dict(n=5000, ws=None), dict(n=5000, ws=FAKE + 8)])
def test_refused_calls(bad):
    assert call(**bad) == -1 and et.et_last_error()


def test_null_pool_and_workspace():
    lib = et.load_library()
    assert lib.et_kv_resize(None, FAKE, FAKE, FAKE, 4, 4, FAKE, FAKE, 3, 5, FAKE, FAKE, FAKE, FAKE, 1 << 40, None) == -1
    need = lib.et_kv_resize_workspace_bytes
    assert need(-1) == need(0) == need(1) == need(4096) == 0
    assert 0 < need(4097) < need(2 ** 20) < 1 << 24
    assert call(n=5000, ws_bytes=need(5000) - 1) == -2 and "workspace" in et.et_last_error()


def test_refused_slots():
    lib = et.load_library()
    c = B._KvCache(data_dev=FAKE, n_pages=8, page_size=16, n_kv_heads=2, head_dim=64, format=0)
    fn = lambda c=c, slots=FAKE, rows=5, k=FAKE, ks=128, v=FAKE, vs=128: lib.et_kv_append_slots(c and C.byref(c), slots, rows, k, ks, v, vs, None)
    for bad in (dict(c=None), dict(slots=None), dict(slots=FAKE + 4), dict(rows=-1), dict(rows=2 ** 30), dict(k=None), dict(v=FAKE + 8), dict(ks=120),
                dict(vs=132)):
        assert fn(**bad) == -1 and et.et_last_error(), bad
    assert fn(c=B._KvCache(data_dev=FAKE, n_pages=8, page_size=24, n_kv_heads=2, head_dim=64, format=0)) == -5
    assert fn(rows=0, slots=None, k=None, v=None) == 0


def test_binding_refuses():
    for bad in ((0, 16), (4, 24), (4, 0), (2 ** 31, 16)):
        with pytest.raises(ValueError):
            et.PagePool(*bad)
    with pytest.raises(TypeError):
        et.PagePool(4, 16, ring=torch.arange(4, dtype=torch.int32))  # a host tensor
