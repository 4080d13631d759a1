"""Attention over 4 bits: a weight is within 2^-15 of its float32 value in every form of the kernel (four, two and one columns a query head, four
and eight wavefronts, one part and parts that are joined)."""
import math

import numpy as np
import pytest
import torch

import paper_2605_30010_amd as et
from tests.test_gpu_kv import dev, tables

pytestmark = pytest.mark.gpu


def cut(w):
    """Weights as bfloat16 numbers alone: the lower 16 bits of float32 away."""
    return (w.float().view(torch.int32) & -65536).view(torch.float32).double()


# one part by four wavefronts (short; long, more than 256 workgroups), by eight, a window, several parts joined, the same of a single sequence
FORMS = {"short": (16, 2, [400, 512, 77, 1], 0), "long": (32, 8, [600] + [40] * 32, 0), "eight": (16, 24, [1000, 33, 900], 0),
         "window": (64, 24, [1000, 2500, 900, 2000, 1500, 1200, 800, 2050], 1000), "joined": (32, 2, [2500, 1, 1700], 0), "single": (16, 3, [2300], 0)}


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("group,d", [(1, 64), (3, 80), (4, 128), (2, 256), (5, 96), (8, 128), (6, 64), (9, 80), (16, 128), (17, 64)])
def test_weights_keep_sixteen_bits(group, d, form):
    """Keys of 0 and -1, a query head h that looks at dimension h only, and a scale with which -1 weighs 0.504 = (1 + 2^-7 - 2^-13) / 2, of which eight
    bits keep 0.5: all tokens of a head are off in the same direction then.  Values are 2 where the key is -1 and -1 where it is 0, so that dimension h
    of the result all but cancels, and with it the result's own rounding.  Per value: that rounding, 2^-8; weights 2^-15, their exponential
    and the joining factors some roundings of 2^-24 (2^-20 in all); the logits' float32 sums (d products and up to 8 roundings of sums and
    factors, numerator and denominator; 1.45 > log2 e); a sum over up to 2 n weights' halves.  Weights of eight bits are outside in every head of every
    sequence of 64 tokens or more, which is shown on the definition itself."""
    page, kv, lens, window = FORMS[form]
    rng = np.random.default_rng(group + d)
    g = torch.Generator("cuda:0").manual_seed(group + d)
    table, n_pages = tables(rng, lens, page)
    cache = et.KVCache(n_pages, page, kv, d, fmt="mxfp4")
    cache.data.fill_(0xFF)
    rows, heads = sum(lens), torch.arange(group, device="cuda:0")
    bit = torch.randint(0, 2, (rows, kv, d), generator=g, device="cuda:0").double()
    keys, values = -bit, 3 * bit - 1
    q = torch.zeros((len(lens), kv, group, d), dtype=torch.float64, device="cuda:0")
    q[:, :, heads, heads] = 1.0
    scale = -math.log((1 + 2.0 ** -7 - 2.0 ** -13) / 2)
    args = dev(table), dev(np.array(lens, dtype=np.int32))
    k, v = (x.flatten(1).to(torch.bfloat16) for x in (keys, values))
    cu = dev(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32))
    cache.append(k, v, *args, cu)
    back = cache.read(*args, cu, rows)
    assert torch.equal(back[0], k) and torch.equal(back[1], v)        # held exactly
    got = cache.attend(q.to(torch.bfloat16).flatten(1), *args, max(lens), window=window, scale=scale).double().reshape(len(lens), kv, group, d)
    at = 0
    for b, n in enumerate(lens):
        lo = at + (max(0, n - window) if window else 0)
        kb, vb = (x[lo:at + n].transpose(0, 1).contiguous() for x in (keys, values))         # [kv, tokens, d]
        at += n
        logits = q[b] @ kb.transpose(1, 2).contiguous() * scale
        w = torch.exp(logits - logits.amax(-1, keepdim=True))
        total = w.sum(-1, keepdim=True)
        size = logits.abs().amax(-1, keepdim=True)                    # (one product that is not 0)
        ref, mass = w @ vb / total, w @ vb.abs() / total
        tol = 2.0 ** -8 * ref.abs() + (2.0 ** -15 + 2.0 ** -20 + 2 * (d + 8) * 2.0 ** -24 * 1.45 * size + 2 * n * 2.0 ** -24) * mass
        off = (got[b] - ref).abs() - tol
        assert (off <= 0).all(), (b, n, float(off.max()))
        if n >= 64:
            assert ((cut(w) @ vb / total - ref).abs() > tol)[:, heads, heads].all()
