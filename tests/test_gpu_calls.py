"""The binding's native part against the rest of it: the same results, the same refusals."""
import numpy as np
import pytest
import torch

import paper_2605_30010_amd as et
from tests.test_gpu_kv import dev, tables

pytestmark = pytest.mark.gpu


def outcome(call):
    """What a call gives: its tensors' values, or its error's type and text."""
    try:
        got = call()
    except Exception as e:                                            # noqa: BLE001 (errors are compared)
        return type(e), str(e)
    torch.cuda.synchronize()
    got = got if isinstance(got, tuple) else (got,)
    return tuple(None if t is None else (t.dtype, tuple(t.shape), t.is_contiguous(), t.clone().view(torch.uint8).cpu().numpy().tobytes()) for t in got)


def both(thing, call):
    """The same with and without the native part."""
    native = thing._calls
    assert native is not None
    first = outcome(call)
    thing._calls = None
    try:
        second = outcome(call)
    finally:
        thing._calls = native
    assert first == second, (first[:2], second[:2])
    return first


def randn(*shape):
    return torch.randn(shape, device="cuda:0").to(torch.bfloat16)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "mxfp4"])
def test_the_caches_calls(fmt):
    torch.manual_seed(1)
    rng = np.random.default_rng(1)
    lens = [700, 3, 0, 40]
    table, n_pages = tables(rng, lens, 16)
    c = et.KVCache(n_pages, 16, 2, 64, fmt=fmt)
    c.data.fill_(0x22)
    tab, ln, cu = dev(table), dev(np.array(lens, dtype=np.int32)), dev(np.array([0, 5, 6, 6, 9], dtype=np.int32))
    k, v, q = randn(9, 300)[:, 4:132], randn(9, 2, 64), randn(4, 6, 64)
    for x in (k, randn(9, 128)):                                      # (4 values off 16 bytes: refused)
        both(c, lambda: c.append(x, v, tab, ln, cu))
        both(c, lambda: c.append_at(x, v, torch.arange(9, device="cuda:0")))
    assert c.append(randn(9, 128), v, tab, ln, cu) is None
    for args in ((tab, ln, cu, 9), (tab, ln), (tab, ln, None, 4), (tab, ln, cu), (tab, ln, cu, -1), (tab, ln, None, 3), (tab, ln.long(), cu, 9), (tab[:3], ln, cu, 9),
                 (tab, ln, cu[:3], 9), (tab, ln, cu, 9.0), (tab.cpu(), ln, cu, 9)):
        both(c, lambda: c.read(*args))
    for args, kw in (((q, tab, ln, 700), {}), ((q, tab, ln, 2 ** 40), {}), ((q, tab, ln, 700), dict(window=5)), ((q, tab, ln, 700), dict(window=2 ** 33)),
                     ((q, tab, ln, 64), dict(scale=0.5)), ((q, tab, ln, 64), dict(scale=1)), ((q, tab, ln, 64), dict(scale=float("nan"))), ((q, tab, ln, 0), {}),
                     ((q, tab, ln, -5), {}), ((q, tab, ln, 64), dict(window=-1)), ((q[:3], tab, ln, 64), {}), ((q[:, :3], tab, ln, 64), {}),
                     ((q[:, ::2], tab, ln, 64), {}), ((q.float(), tab, ln, 64), {}), ((q.flatten(1), tab, ln, np.int64(700)), {}),
                     ((q.flatten(1)[:, 8:], tab, ln, 64), {}), ((q[:1], tab[:1], ln[:1], 700), {}), ((q[:0], tab[:0], ln[:0], 700), {})):
        both(c, lambda: c.attend(*args, **kw))
    for args in ((k[:8], v, tab, ln, cu), (v, v, tab, ln), (v[:4], v[:4], tab, ln), (v, v, tab.t(), ln, cu), (v, v, tab, ln[None], cu), (v.cpu(), v, tab, ln, cu)):
        both(c, lambda: c.append(*args))


def test_the_pools_calls():
    pool = et.PagePool(50, 16)
    tab, old, new = torch.full((3, 9), -1, dtype=torch.int32, device="cuda:0"), *(dev(np.array(x, dtype=np.int32)) for x in ([0, 5, 33], [40, 0, 100]))
    state = torch.zeros(4, dtype=torch.int32, device="cuda:0")
    # (rows behind the last sequence's hold anything)
    for args, kw in (((tab, old, new, 107), {}), ((tab[:, :5], old, new, 107), {}), ((tab, old, new, 0), {}), ((tab, old, new, -1), {}),
                     ((tab, old, new, 2 ** 31), {}), ((tab, old, new[:2], 107), {}), ((tab.t(), old, new, 107), {}), ((tab, old.long(), new, 107), {}),
                     ((tab, old, new, 107.0), {}), ((tab[:1], old[:1], new[:1], 40), {}), ((tab[:0], old[:0], new[:0], 0), {}), ((tab, old, new, 107), dict(state_out=state[:3]))):
        both(pool, lambda: pool.resize(*args, **dict(dict(state_out=state), **kw)))


def test_the_rotary_calls():
    torch.manual_seed(2)
    r = et.Rotary(64, rot_dim=32)
    q, k, pos = randn(7, 500), randn(7, 2, 64), torch.arange(7, dtype=torch.int32, device="cuda:0")
    for x in (q[:, :256], q[:, 1:257], q[:, 8:200], k, k[:, :1], k[:1], q[:, :60], q.t(), k.float(), k[:6], k[:0], q[:, ::2]):
        for y in (None, k, k[:6], q[:, 64:192]):
            for kw in ({}, dict(transpose=True), dict(transpose=1)):
                both(r, lambda: r.apply(x, y, pos, **kw))
    both(r, lambda: r.apply(k[:0], None, pos[:0]))
    for p in (pos.long(), pos[::2], pos[None], pos.cpu()):
        both(r, lambda: r.apply(k, None, p))
    to = [torch.zeros_like(k), torch.zeros((7, 640), dtype=torch.bfloat16, device="cuda:0")]
    for out in ((to[0], None), (None, to[1][:, 3:131]), (to[0], to[1][:, :128]), (to[1][:, :64], None), (to[0].float(), None), (to[0][:6], None)):
        both(r, lambda: r.apply(k, k, pos, out=out))
    got = r.apply(k, k, pos, out=(to[0], None))
    assert got[0] is to[0] and got[1] is not k


def test_results_belong_to_their_stream_and_graph():
    """Native calls on a side stream and in a graph use its stream and its memory."""
    torch.manual_seed(3)
    r = et.Rotary(64)
    x, pos = randn(5, 128), torch.arange(5, dtype=torch.int32, device="cuda:0")
    ref, _ = r.apply(x, None, pos)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        a, _ = r.apply(x, None, pos)
    b, _ = r.apply(x, None, pos, stream=side)
    side.synchronize()
    assert torch.equal(a, ref) and torch.equal(b, ref)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, _ = r.apply(x, None, pos)
    for _ in range(3):
        x.copy_(randn(5, 128))
        g.replay()
        assert torch.equal(out, r.apply(x, None, pos)[0])


def test_errors_of_an_entry_point_carry_its_message():
    c = et.KVCache(4, 16, 2, 64)
    tab, ln = torch.zeros((3, 2), dtype=torch.int32, device="cuda:0"), torch.ones(3, dtype=torch.int32, device="cuda:0")
    with pytest.raises(et.EtError, match="n_heads"):
        c.attend(randn(3, 192), tab, ln, 16)
    with pytest.raises(et.EtError, match="max_len"):
        c.attend(randn(3, 128), tab, ln, 0)
    with pytest.raises(et.EtError, match="aligned"):
        c.append_at(randn(3, 130)[:, 2:], randn(3, 128), torch.zeros(3, dtype=torch.int64, device="cuda:0"))


@pytest.mark.parametrize("rows", [0, 1, 3, 500, 9000])
def test_results_of_a_call_keep_apart(rows):
    """Small results share a piece of memory: aligned, apart, of their own shapes, and each survives the others."""
    d, r = 64, et.Rotary(64)
    g = torch.Generator("cuda:0").manual_seed(rows)
    q, k = (torch.randn((rows, n * d), generator=g, device="cuda:0").to(torch.bfloat16) for n in (9, 3))
    pos = torch.arange(rows, dtype=torch.int32, device="cuda:0")
    want = r.apply(q, None, pos)[0], r.apply(k, None, pos)[0]
    a, b = r.apply(q, k, pos)
    assert a.shape == q.shape and b.shape == k.shape and a.is_contiguous() and b.is_contiguous() and a.data_ptr() % 128 == b.data_ptr() % 128 == 0
    assert not a.requires_grad and a._base is None and a.dtype is torch.bfloat16
    keep = a.clone()
    b.zero_()
    del b
    filler = [torch.full((64, d), 7.0, dtype=torch.bfloat16, device="cuda:0") for _ in range(64)]
    assert torch.equal(a, keep) and torch.equal(a, want[0])
    a, b = r.apply(q, k, pos)
    del a, filler
    assert torch.equal(b, want[1]) and torch.equal(b + b, want[1] + want[1])
    pool = et.PagePool(700, 16)
    table = torch.full((1, 700), -1, dtype=torch.int32, device="cuda:0")
    old, new = torch.zeros(1, dtype=torch.int32, device="cuda:0"), torch.full((1,), rows, dtype=torch.int32, device="cuda:0")
    cu, positions, slots = pool.resize(table, old, new, rows)
    assert cu.dtype is positions.dtype is torch.int32 and slots.dtype is torch.int64
    assert cu.tolist() == [0, rows] and torch.equal(positions, pos) and torch.equal(slots, pos.long())
    positions.fill_(-5)
    assert cu.tolist() == [0, rows] and torch.equal(slots, pos.long())
