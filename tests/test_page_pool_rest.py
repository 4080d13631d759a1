"""Rows behind the last sequence's, without a GPU: what is refused, and which of the two ways the binding asks for."""
import ctypes as C

import pytest
import torch

import paper_2605_30010_amd as et
from paper_2605_30010_amd import binding as B
from tests.test_page_pool import FAKE, call


@pytest.mark.parametrize("keep", [-1, 2, 2 ** 31 - 1])
def test_refused(keep):
    assert call(pool=dict(keep_rest=keep)) == -1 and "keep_rest" in et.et_last_error()


class _Lib:
    def et_kv_resize_workspace_bytes(self, n):
        return 0

    def et_kv_resize(self, pool, *_):
        self.keep = pool.keep_rest
        return 0


def test_only_rows_of_out_are_kept(monkeypatch):
    """Results that the binding makes have no place behind the last row; `out` keeps what it has."""
    meta = lambda *shape, dtype=torch.int32: torch.empty(shape, dtype=dtype, device="meta")
    monkeypatch.setattr(B, "_dev", lambda *_: None)
    pool = et.PagePool(8, 16, ring=meta(8), state=meta(4))
    pool._calls, pool._lib = None, _Lib()
    pool._here = lambda stream: 0
    pool.resize(meta(3, 2), meta(3), meta(3), 5)
    assert pool._lib.keep == 0 and C.cast(pool._at, C.POINTER(B._KvPool)).contents.keep_rest == 0
    pool.resize(meta(3, 2), meta(3), meta(3), 5, out=(meta(4), meta(5), meta(5, dtype=torch.int64)))
    assert pool._lib.keep == 1
