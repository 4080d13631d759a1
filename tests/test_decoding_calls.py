"""The binding's calls of a decoding step without a GPU: devices, streams, and its native part's answers to what is not plain."""
import numpy as np
import pytest
import torch

import paper_2605_30010_amd as et
from paper_2605_30010_amd import binding as B


class _Device:
    """Stands in for torch.cuda.device and torch.cuda.stream: notes what is current."""
    current, log = 0, []

    def __init__(self, to):
        self.to = to

    def __enter__(self):
        self.was, _Device.current = _Device.current, self.to
        _Device.log.append(self.to)

    def __exit__(self, *_):
        _Device.current = self.was


class _Lib:
    """Notes under which device each entry point is called, and with which stream (its last argument)."""
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, _Device.current, args[-1]))
            return 64 if name.endswith("bytes") else 0
        return call


META = torch.device("meta")


def empty(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device=META)


@pytest.mark.parametrize("current", [0, None])
def test_calls_run_on_their_device_and_its_stream(monkeypatch, current):
    """On another device than the current one: allocation and launch happen with its device current, on that device's stream; a stream of a
    third device is refused.  (Tensors without memory stand for the other device, index None.)"""
    cache, pool, rotary = (object.__new__(c) for c in (et.KVCache, et.PagePool, et.Rotary))
    lib = _Lib()
    cache.device, cache.head_dim, cache.n_kv_heads, cache._width, cache._cache, cache._lib = META, 64, 2, 128, None, lib
    pool.device, pool.ring, pool.state, pool._pool, pool._lib = META, empty(4, dtype=torch.int32), empty(4, dtype=torch.int32), None, lib
    rotary.device, rotary.head_dim, rotary._rotary, rotary._lib = META, 64, None, lib
    monkeypatch.setattr(B, "_current_device", lambda: _Device.current)
    monkeypatch.setattr(torch.cuda, "device", lambda d: _Device(d.index))
    monkeypatch.setattr(torch.cuda, "stream", lambda s: _Device(s.device.index))
    monkeypatch.setattr(B, "_raw_stream", lambda d: ("stream of", d))
    _Device.current, _Device.log = current, []
    x, ints = empty(3, 128), empty(3, dtype=torch.int32)
    table, slots = empty(3, 2, dtype=torch.int32), empty(3, dtype=torch.int64)

    class Stream:
        device, cuda_stream = META, 5

    class Other:
        device, cuda_stream = torch.device("cpu"), 6

    made = [lambda **k: cache.append_at(x, x, slots, **k), lambda **k: pool.resize(table, ints, ints, 3, **k), lambda **k: rotary.apply(x, x, ints, **k),
            lambda **k: rotary.apply(x, None, ints, transpose=True, **k)]
    for extra in ({}, {"stream": Stream()}):
        lib.calls.clear()
        _Device.log.clear()
        for call in made:
            call(**extra)
        assert [k[0] for k in lib.calls] == ["et_kv_append_slots", "et_kv_resize", "et_rotary_apply", "et_rotary_apply"]
        assert all(k[1] is None and k[2] == ("stream of", None) for k in lib.calls)
        assert _Device.current == current and len(_Device.log) == (4 if extra or current == 0 else 0)
    for call in made:
        with pytest.raises(ValueError):
            call(stream=Other())


def test_the_native_part_leaves_what_is_not_plain_to_the_rest():
    """Host tensors, other types, None, numbers, lists: None comes back, nothing is called."""
    et.load_library()
    calls = B._calls
    cache = B._KvCache(data_dev=4096, n_pages=8, page_size=16, n_kv_heads=2, head_dim=64, format=0)
    pool, rotary = B._KvPool(4096, 8, 16), B._Rotary(4096, 64, 64, 0, 1.0)
    import ctypes as C
    at = C.addressof
    x, ints, table = torch.zeros((3, 128), dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32), torch.zeros((3, 2), dtype=torch.int32)
    cu, slots = torch.zeros(4, dtype=torch.int32), torch.zeros(3, dtype=torch.int64)
    good = {"append": (at(cache), 0, x, x, table, ints, cu, 0), "append_at": (at(cache), 0, x, x, slots, 0), "read": (at(cache), 0, table, ints, cu, 3, 0),
            "attend": (at(cache), 0, x, table, ints, 16, 0, 0.1, 0), "resize": (at(pool), 0, cu, cu, table, ints, ints, 3, 0),
            "rotate": (at(rotary), 0, x, x, ints, None, None, False, 0)}
    odd = [None, 3, "x", [1, 2], np.zeros(3), x.float(), x.t(), x[0], torch.zeros(()), torch.zeros((2, 2)).to_sparse()]
    for name, args in good.items():
        for device in (0, -1, 7):
            assert getattr(calls, name)(args[0], device, *args[2:]) is None
        for i in range(2, len(args) - 1):
            for o in odd:
                assert getattr(calls, name)(*args[:i], o, *args[i + 1:]) is None, (name, i)


def test_the_native_part_says_what_is_missing(tmp_path):
    et.load_library()
    with pytest.raises(ImportError):
        B._calls.bind(str(tmp_path / "absent.so"))
    B._calls.bind(B._LIB_PATH)
