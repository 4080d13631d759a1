"""The binding's native part with a stream that is no number: Python's error, and the next call is as ever."""
import pytest
import torch

import paper_2605_30010_amd as et

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", ["x", None, 1.5, 2 ** 70])
def test_a_stream_that_is_none_is_an_error(bad):
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda:0")
    cache, pool, rotary = et.KVCache(8, 16, 2, 64), et.PagePool(8, 16), et.Rotary(64)
    cache.data.zero_()
    x, table, one, new = torch.ones((3, 128), dtype=torch.bfloat16, device="cuda:0"), ints(0, 1, 2).view(3, 1), ints(1, 1, 1), ints(2, 1, 1)
    slots, cu = torch.arange(3, device="cuda:0"), ints(0, 1, 2, 3)
    native, at = cache._calls, cache._index
    made = [lambda s: native.append(cache._at, at, x, x, table, one, cu, s), lambda s: native.append_at(cache._at, at, x, x, slots, s),
            lambda s: native.read(cache._at, at, table, one, cu, 3, s), lambda s: native.attend(cache._at, at, x, table, one, 16, 0, 0.125, s),
            lambda s: native.resize(pool._at, at, pool.state, pool.state, table, one, new, 1, s),
            lambda s: native.rotate(rotary._at, at, x, x, one, None, None, False, s)]
    for call in made:
        with pytest.raises((TypeError, OverflowError)):
            call(bad)
    torch.cuda.synchronize()
    assert not cache.data.any() and pool.state.tolist() == [0, 8, 0, 0]          # nothing ran
    for call in made:
        got = call(torch.cuda.current_stream().cuda_stream)
        assert got is not None and (type(got) is not int or got == 0)
    torch.cuda.synchronize()
    assert cache.data.any()
