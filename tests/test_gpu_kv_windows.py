"""A window that no sequence fills gives the bits of none."""
import numpy as np
import pytest
import torch

import paper_2605_30010_amd as et
from tests.test_gpu_kv import dev, tables

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["mxfp4", "bf16"])
@pytest.mark.parametrize("kv,heads,lens", [(24, 24, [1000, 33, 900]), (2, 6, [2500, 1, 0]), (2, 2, [2300]), (2, 8, [40, 512])])
def test_windows_up_to_the_largest(fmt, kv, heads, lens):
    g = torch.Generator("cuda:0").manual_seed(1)
    table, n_pages = tables(np.random.default_rng(1), lens, 16)
    cache = et.KVCache(n_pages, 16, kv, 64, fmt=fmt)
    x = torch.randn((sum(lens), 2 * kv * 64), generator=g, device="cuda:0").to(torch.bfloat16)
    q = torch.randn((len(lens), heads * 64), generator=g, device="cuda:0").to(torch.bfloat16)
    args = dev(table), dev(np.array(lens, dtype=np.int32))
    cache.append(x[:, :kv * 64], x[:, kv * 64:], *args, dev(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)))
    none = cache.attend(q, *args, max(lens))
    assert none.any()
    for window in (max(lens), 2 ** 31 - 16, 2 ** 31 - 1, 2 ** 40):
        assert torch.equal(cache.attend(q, *args, max(lens), window=window), none), window
