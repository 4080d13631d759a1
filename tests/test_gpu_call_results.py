"""Whose memory the results of a call are."""
import io

import pytest
import torch

import paper_2605_30010_amd as et

pytestmark = pytest.mark.gpu


def ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda:0")


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("rows", [1, 3, 4000])
def test_keys_and_values_read_back_are_tensors_of_their_own(rows, native):
    cache = et.KVCache(300, 16, 2, 64)
    if not native:
        cache._calls = None
    table, cu = torch.arange(300, dtype=torch.int32, device="cuda:0")[None], ints(0, rows)
    x = torch.randn((2, rows, 128), device="cuda:0").to(torch.bfloat16)
    cache.append(x[0], x[1], table, ints(rows), cu)
    k, v = cache.read(table, ints(rows), cu, rows)
    for t, want in ((k, x[0]), (v, x[1])):
        size, at = t.untyped_storage().nbytes(), t.storage_offset()
        assert torch.equal(t, want) and (at, size) == (0, rows * 256)
        f = io.BytesIO()
        torch.save(t, f)
        size = f.tell()
        assert size < rows * 256 + 4096
    k.resize_(4 * rows, 128).fill_(7.0)                                # grows where there is room for it alone
    assert torch.equal(v, x[1])


def test_results_that_share_a_piece_of_memory():
    """As the docstrings of resize and apply have it: one keeps the piece, and with it what it holds, and a clone is on its own."""
    pool, rotary = et.PagePool(8, 16), et.Rotary(64)
    table, x = torch.full((1, 8), -1, dtype=torch.int32, device="cuda:0"), torch.randn((5, 128), device="cuda:0").to(torch.bfloat16)
    cu, positions, slots = pool.resize(table, ints(0), ints(5), 5)
    q, k = rotary.apply(x, x, positions)
    for results in ((cu, positions, slots), (q, k)):
        assert len({t.untyped_storage().data_ptr() for t in results}) == 1
        last, want = results[-1], results[-1].clone()
        size = want.untyped_storage().nbytes()
        assert size == want.numel() * want.element_size()
        del results
        for t in (cu, positions, q):
            t.zero_()
        filler = [torch.full((64,), 9.0, device="cuda:0") for _ in range(64)]
        assert torch.equal(last, want) and len(filler) == 64
