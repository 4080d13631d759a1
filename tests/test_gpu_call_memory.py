"""Tensors whose address torch withholds (as it does for those that stand for others in a trace): the binding's calls raise torch's error, with and without the native part, and go on."""
import pytest
import torch

import paper_2605_30010_amd as et

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("native", [True, False])
def test_tensors_without_an_address_are_an_error(native):
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda:0")
    cache, pool, rotary = et.KVCache(8, 16, 2, 64), et.PagePool(8, 16), et.Rotary(64)
    if not native:
        cache._calls = pool._calls = rotary._calls = None
    cache.data.zero_()
    rows, table, one, new = torch.ones((3, 128), dtype=torch.bfloat16, device="cuda:0"), ints(0, 1, 2).view(3, 1), ints(1, 1, 1), ints(2, 1, 1)
    slots, cu = torch.arange(3, device="cuda:0"), ints(0, 1, 2, 3)
    made = [(lambda k, v, t, n, c: cache.append(k, v, t, n, c), (rows, rows, table, one, cu)), (lambda k, v, s: cache.append_at(k, v, s), (rows, rows, slots)),
            (lambda t, n, c: cache.read(t, n, c, 3), (table, one, cu)), (lambda q, t, n: cache.attend(q, t, n, 16), (rows, table, one)),
            (lambda t, n, m: pool.resize(t, n, m, 1), (table, one, new)), (lambda q, k, p: rotary.apply(q, k, p), (rows, rows, one))]
    for call, args in made:
        for i in range(len(args)):
            gone = args[i].clone()
            torch._C._set_throw_on_mutable_data_ptr(gone)
            with pytest.raises(RuntimeError, match="data pointer"):
                call(*args[:i], gone, *args[i + 1:])
    torch.cuda.synchronize()
    assert not cache.data.any() and pool.state.tolist() == [0, 8, 0, 0]
    for call, args in made:
        call(*args)
    torch.cuda.synchronize()
    assert cache.data.any()
