"""What the paged cache's calls hand to the library, and what they refuse, without a GPU."""
import pytest
import torch

import paper_2605_30010_amd as et
from paper_2605_30010_amd import binding as B


class _Lib:
    """Notes the calls of the entry points."""
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 64 if name.endswith("bytes") else 0
        return call


META = torch.device("meta")


@pytest.fixture
def cache(monkeypatch):
    """A cache of two heads of 64 whose tensors have no memory."""
    c = object.__new__(et.KVCache)
    c.device, c.fmt, c.head_dim, c.n_kv_heads, c._width, c._scale, c._cache, c._lib = META, "bf16", 64, 2, 128, 0.125, None, _Lib()
    monkeypatch.setattr(B, "_current_device", lambda: None)
    monkeypatch.setattr(B, "_raw_stream", lambda d: 0)
    return c


def ints(*shape):
    return torch.empty(shape, dtype=torch.int32, device=META)


def rows(n, width=128):
    return torch.empty((n, width), dtype=torch.bfloat16, device=META)


def test_read_of_row_ranges_takes_all_rows_of_out_or_asks_for_their_number(cache):
    """The row ranges are on the device: their end is the caller's to say, and never taken to be one row for each sequence."""
    tab, lens, cu = ints(3, 2), ints(3), ints(4)
    asked = lambda: cache._lib.calls[-1][1][3]
    k, v = cache.read(tab, lens, cu, out=(rows(40), rows(40)))
    assert asked() == 40 and k.shape == v.shape == (40, 128)
    cache.read(tab, lens, cu, out=(rows(40), rows(41)))
    assert asked() == 40
    cache.read(tab, lens, cu, 7, out=(rows(40), rows(40)))
    assert asked() == 7
    k, v = cache.read(tab, lens, cu, 7)
    assert asked() == 7 and k.shape == v.shape == (7, 128)
    k, v = cache.read(tab, lens)
    assert asked() == 3 and k.shape == v.shape == (3, 128)
    cache.read(tab, lens, out=(rows(40), rows(40)))
    assert asked() == 3
    n = len(cache._lib.calls)
    with pytest.raises(ValueError, match="rows"):
        cache.read(tab, lens, cu)
    with pytest.raises(ValueError, match="rows"):
        cache.read(tab, lens, cu, out=(rows(40), rows(39)))
    assert len(cache._lib.calls) == n


@pytest.mark.parametrize("max_len,window", [(2 ** 31, 0), (2 ** 32 + 16, 2 ** 32 + 5), (2 ** 63 - 1, 2 ** 31), (10 ** 30, 2 ** 32), (600, 7), (16, 0)])
def test_bounds_and_windows_past_32_bits_are_bounds_and_windows(cache, max_len, window):
    """No length reaches 2^31: a larger bound or window is the same as the largest, and not its low bits."""
    cache.attend(rows(3, 256), ints(3, 2), ints(3), max_len, window=window)
    name, args = cache._lib.calls[-1]
    assert name == "et_attention_paged" and args[5:7] == (min(max_len, 2 ** 31 - 1), min(window, 2 ** 31 - 1))
    asked = [a for n, a in cache._lib.calls if n == "et_attention_paged_workspace_bytes"]
    assert all(a[3:5] == args[5:7] for a in asked) and len(asked) == (max_len > 512)
