"""The paged key-value cache of the language model behind the encoder: storing the keys and values of new tokens, reading
them back, and the attention of one new token over it.

A cache is `n_pages` pages of `page` tokens each.  A page holds, one key-value head after the other,
    keys [page, head_dim] | values [page, head_dim] | maxima of the key rows [page] | maxima of the value rows [page]
with keys and values in bfloat16 (no maxima then) or in 8 bits: a row x of head_dim values with the largest magnitude m is
held as m (bfloat16, exact) and the codes round(x * Q / m), ties to even, where Q is 127 (int8: whole numbers) or 448 (e4m3:
the 8-bit floats); it stands for code * m / Q.  A sequence is a row of the page table (page numbers, -1 = none) and a length.
"""
import math

import torch

own = False

DEVICE = "cuda" if torch.cuda.is_available() else "cpu"
QMAX = {"int8": 127.0, "e4m3": 448.0}
HEAD_DIMS = (64, 80, 96, 128, 256)
PAGES = (16, 32, 64, 128, 256)

# A decoder of width 3584 (the width that the projector's workloads end in): 28 heads of 128, 4 key-value heads.
LM = dict(heads=28, kv_heads=4, head_dim=128)
# A generic decoder of width 4096: 32 heads of 128, 8 key-value heads.
WIDE = dict(heads=32, kv_heads=8, head_dim=128)


def listed():
    return [
        # the first answer token behind one small frame (196 tokens): launch latency decides
        dict(name="attend_one_frame", op="attend", fmt="bf16", page=16, heads=8, kv_heads=2, head_dim=64, seqs=1, lo=197, hi=197, window=0),
        # one user asks about a 32-frame clip: the 4949 tokens that the paper's layout keeps, and a question
        dict(name="attend_clip", op="attend", fmt="bf16", page=64, **LM, seqs=1, lo=4999, hi=4999, window=0),
        # a batch of such users at every stage, an idle slot (length 0) among them, 8-bit cache
        dict(name="attend_batch_int8", op="attend", fmt="int8", page=64, **LM, seqs=32, lo=0, hi=5309, window=0),
        # one very long video, a single sequence: the split over the length decides
        dict(name="attend_long", op="attend", fmt="bf16", page=256, **WIDE, seqs=1, lo=131072, hi=131072, window=0),
        # a full server: the largest cache that is read
        dict(name="attend_server_e4m3", op="attend", fmt="e4m3", page=128, **WIDE, seqs=64, lo=1000, hi=16384, window=0),
        # one key-value head for all, wide heads, sliding window, small pages
        dict(name="attend_window", op="attend", fmt="bf16", page=32, heads=20, kv_heads=1, head_dim=256, seqs=7, lo=300, hi=9001, window=1024),
        # every head with its own keys and values, an odd head width
        dict(name="attend_own_heads_int8", op="attend", fmt="int8", page=16, heads=32, kv_heads=32, head_dim=80, seqs=5, lo=1, hi=2047, window=0),
        # a decoding step's new tokens, one for each sequence
        dict(name="store_step_e4m3", op="store", fmt="e4m3", page=64, **WIDE, seqs=48, past=3000, new_lo=1, new_hi=1),
        # a clip's prompt in 8 bits, behind a system prompt that is there already
        dict(name="store_clip_int8", op="store", fmt="int8", page=64, **LM, seqs=1, past=37, new_lo=4999, new_hi=4999),
        # prompts of many lengths in one batch, unquantised
        dict(name="store_prompts", op="store", fmt="bf16", page=32, **WIDE, seqs=16, past=100, new_lo=1, new_hi=8191),
        # a short prefix with odd heads is read back
        dict(name="read_prefix_int8", op="read", fmt="int8", page=16, heads=16, kv_heads=16, head_dim=96, seqs=3, lo=0, hi=733),
        # long sequences are read back whole, for another machine or another form
        dict(name="read_long_e4m3", op="read", fmt="e4m3", page=128, **WIDE, seqs=4, lo=30001, hi=65536),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    limit = max(work(c)["bytes"] for c in listed())
    while True:
        case = dict(op=rng.choice(["attend", "attend", "store", "read"]), fmt=rng.choice(["bf16", "e4m3", "int8"]), page=rng.choice(PAGES))
        kv = rng.choice([1, 2, 3, 4, 5, 8, 8, 16])
        case.update(heads=kv * rng.choice([1, 2, 3, 4, 5, 7, 8, 17]), kv_heads=kv, head_dim=rng.choice([64, 80, 96, 128, 128, 128, 256]))
        seqs = _log(rng, 1, 96)
        if case["op"] == "store":
            hi = _log(rng, 1, 8192)
            case.update(seqs=seqs, past=rng.choice([0, _log(rng, 1, 4000)]), new_lo=rng.choice([0, 1, hi]), new_hi=hi)
        else:
            hi = _log(rng, 1, 131072)
            case.update(seqs=seqs, lo=rng.choice([0, 1, hi // 3, hi]), hi=hi)
            if case["op"] == "attend":
                case["window"] = rng.choice([0, 0, 0, _log(rng, 1, 4096)])
        if work(case)["bytes"] <= limit and case["heads"] <= 128:
            return case


# ---------------------------------------------------------------------------------------------- what a case asks for

def spread(lo, hi, n):
    """n lengths from hi down to lo."""
    return [hi - (hi - lo) * i // max(n - 1, 1) for i in range(n)]


def lengths(case):
    """(length of every sequence, how many of its last tokens are new or read)."""
    if case["op"] == "store":
        new = spread(case["new_lo"], case["new_hi"], case["seqs"])
        return [n + p for n, p in zip(new, spread(case["past"] // 2, case["past"], case["seqs"]))], new
    every = spread(case["lo"], case["hi"], case["seqs"])
    return every, every


def element(fmt):
    return 2 if fmt == "bf16" else 1


def work(case):
    every, new = lengths(case)
    kv, d, e = case["kv_heads"], case["head_dim"], element(case["fmt"])
    m = 0 if case["fmt"] == "bf16" else 2
    row = 2.0 * kv * (d * e + m)                                     # keys and values of one token as the cache holds them
    plain = 2.0 * kv * d * 2                                         # the same as bfloat16 rows
    if case["op"] == "attend":
        seen = sum(min(n, case["window"]) if case["window"] else n for n in every)
        q = case["heads"] * d
        return dict(bytes=seen * row + case["seqs"] * q * 4.0, flops=4.0 * seen * q)
    rows = sum(new)
    if case["op"] == "read":
        return dict(bytes=rows * (row + plain), flops=2.0 * rows * kv * d)
    if case["fmt"] == "bf16":
        return dict(bytes=rows * (row + plain), flops=float(rows * kv * d))
    return dict(bytes=rows * 2 * (row + plain), flops=8.0 * rows * kv * d)   # stored, and read back


# ---------------------------------------------------------------------------------------------- the cache in plain form

def layout(case):
    """Byte offsets of keys, values and the two maxima in a head's part of a page, and its size."""
    n, e = case["page"] * case["head_dim"], element(case["fmt"])
    m = 0 if case["fmt"] == "bf16" else 2 * case["page"]
    return 0, n * e, 2 * n * e, 2 * n * e + m, 2 * n * e + 2 * m


def parts(case, data):
    """Views of data [..., kv_heads * head bytes]: keys and values [..., kv_heads, page, head_dim] as bytes or bfloat16, and the
    maxima [..., kv_heads, page] (None, None for bfloat16)."""
    k, v, km, vm, end = layout(case)
    heads = data.unflatten(-1, (case["kv_heads"], end))
    shape, kind = (case["page"], case["head_dim"]), torch.bfloat16 if case["fmt"] == "bf16" else torch.uint8
    keys, values = heads[..., k:v].view(kind).unflatten(-1, shape), heads[..., v:km].view(kind).unflatten(-1, shape)
    if case["fmt"] == "bf16":
        return keys, values, None, None
    return keys, values, heads[..., km:vm].view(torch.bfloat16), heads[..., vm:end].view(torch.bfloat16)


def to_codes(fmt, x):
    """(codes as bytes, maxima) of rows x [..., head_dim] bfloat16."""
    x = x.float()
    top = x.abs().amax(-1, keepdim=True)
    y = x * QMAX[fmt] / torch.where(top > 0, top, torch.ones_like(top))
    codes = torch.round(y).to(torch.int8) if fmt == "int8" else y.to(torch.float8_e4m3fn)
    return codes.view(torch.uint8), top[..., 0].to(torch.bfloat16)


def to_values(fmt, codes, top):
    """float32 values of rows as the cache holds them."""
    if fmt == "bf16":
        return codes.float()
    return codes.view(torch.int8 if fmt == "int8" else torch.float8_e4m3fn).float() * top.float()[..., None] / QMAX[fmt]


def places(case, s):
    """(page, place in the page) of every row of a store or read."""
    row = torch.arange(s["rows"], device=DEVICE)
    seq = torch.searchsorted(s["cu"][1:].long(), row, right=True)
    pos = s["lens"].long()[seq] - s["cu"].long()[seq + 1] + row
    return s["table"].long()[seq, pos // case["page"]], pos % case["page"]


def store_plain(case, s):
    page, at = places(case, s)
    keys, values, key_max, value_max = parts(case, s["data"])
    for_heads = (s["rows"], case["kv_heads"], case["head_dim"])
    k, v = s["k"].reshape(for_heads), s["v"].reshape(for_heads)
    if case["fmt"] == "bf16":
        keys[page, :, at], values[page, :, at] = k, v
    else:
        keys[page, :, at], key_max[page, :, at] = to_codes(case["fmt"], k)
        values[page, :, at], value_max[page, :, at] = to_codes(case["fmt"], v)


def read_plain(case, s):
    page, at = places(case, s)
    keys, values, key_max, value_max = parts(case, s["data"])
    quantised = case["fmt"] != "bf16"
    k = to_values(case["fmt"], keys[page, :, at], key_max[page, :, at] if quantised else None)
    v = to_values(case["fmt"], values[page, :, at], value_max[page, :, at] if quantised else None)
    return k.to(torch.bfloat16).flatten(1), v.to(torch.bfloat16).flatten(1)


def attend_plain(case, s):
    kv, d, group = case["kv_heads"], case["head_dim"], case["heads"] // case["kv_heads"]
    seqs, wide = s["table"].shape
    pages = s["data"][s["table"].long().clamp(min=0)]                               # [seqs, pages, bytes]
    keys, values, key_max, value_max = parts(case, pages)

    def along(x):                                                                  # [seqs, kv, tokens, head_dim]
        return x.transpose(1, 2).reshape(seqs, kv, wide * case["page"], d)

    pos = torch.arange(wide * case["page"], device=DEVICE)
    lens = s["lens"].long()[:, None]
    seen = (pos < lens) & (pos >= lens - case["window"] if case["window"] else pos >= 0)
    seen = (seen & (s["table"].long() >= 0).repeat_interleave(case["page"], 1))[:, None, None]
    k = along(to_values(case["fmt"], keys, key_max))
    logits = s["q"].float().reshape(seqs, kv, group, d) @ k.transpose(2, 3) * (1.0 / math.sqrt(d))
    del k
    logits = torch.where(seen, logits, -math.inf)
    top = logits.amax(-1, keepdim=True)
    p = torch.exp(logits - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    v = torch.where(seen[:, :, 0, :, None], along(to_values(case["fmt"], values, value_max)), 0.0)
    out = p @ v / torch.where(total > 0, total, 1.0)
    return out.to(torch.bfloat16).reshape(seqs, case["heads"] * d)


# ---------------------------------------------------------------------------------------------- inputs

def normal(g, *size):
    return torch.randn(size, generator=g, device=DEVICE)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    every, new = lengths(case)
    order = torch.randperm(len(every), generator=g, device=DEVICE).tolist()
    every, new = [every[i] for i in order], [new[i] for i in order]
    kv, d, page = case["kv_heads"], case["head_dim"], case["page"]
    used = [-(-n // page) for n in every]
    n_pages, wide = sum(used) + 3, max(max(used), 1)                               # some pages are free
    table = torch.full((len(every), wide), -1, dtype=torch.int32)
    free = torch.randperm(n_pages, generator=g, device=DEVICE).int().cpu()
    for i, n in enumerate(used):
        table[i, :n], free = free[:n], free[n:]
    s = dict(case=case, table=table.to(DEVICE), lens=torch.tensor(every, dtype=torch.int32, device=DEVICE), max_len=max(max(every), 1),
             rows=sum(new), cu=torch.tensor([0] + new, device=DEVICE).cumsum(0).int(),
             data=torch.empty((n_pages, kv * layout(case)[-1]), dtype=torch.uint8, device=DEVICE))
    # keys: some channels are much larger than the rest and off zero, as in trained decoders; values are plain
    size, middle = 0.3 + normal(g, kv, 1, d).square(), normal(g, kv, 1, d)
    for first in range(0, n_pages, 256):
        some = s["data"][first:first + 256]
        keys, values, key_max, value_max = parts(case, some)
        for to, top, x in ((keys, key_max, normal(g, *keys.shape) * size + middle), (values, value_max, normal(g, *values.shape))):
            if case["fmt"] == "bf16":
                to.copy_(x)
            else:
                codes, m = to_codes(case["fmt"], x.to(torch.bfloat16))
                to.copy_(codes)
                top.copy_(m)
    rows = case["seqs"] if case["op"] == "attend" else s["rows"]
    if case["op"] != "read":
        # queries, keys and values are columns of one projection's rows; an attending query agrees a little with the keys' middle
        width = case["heads"] * d
        fused = normal(g, rows, width + 2 * kv * d)
        fused[:, :width] *= 0.8
        fused[:, width:width + kv * d] = fused[:, width:width + kv * d] * size.flatten() + middle.flatten()
        fused = fused.to(torch.bfloat16)
        s["q"], s["k"], s["v"] = fused[:, :width], fused[:, width:width + kv * d], fused[:, width + kv * d:]
    if own:
        import paper_2605_30010_amd as et
        s["cache"] = et.KVCache(n_pages, page, kv, d, fmt=case["fmt"], data=s["data"])
    return s


def run(s):
    case = s["case"]
    if own:
        cache = s["cache"]
        if case["op"] == "attend":
            return cache.attend(s["q"], s["table"], s["lens"], s["max_len"], window=case["window"])
        if case["op"] == "store":
            cache.append(s["k"], s["v"], s["table"], s["lens"], s["cu"])
            if case["fmt"] == "bf16":
                return s["data"].view(torch.bfloat16)
        return cache.read(s["table"], s["lens"], s["cu"], s["rows"])
    if case["op"] == "attend":
        return attend_plain(case, s)
    if case["op"] == "store":
        store_plain(case, s)
        if case["fmt"] == "bf16":
            return s["data"].view(torch.bfloat16)
    return read_plain(case, s)


# ---------------------------------------------------------------------------------------------- the same from the definition, in 64 bits

def held(fmt, x):
    """What rows x stand for once they are stored, float64."""
    x = x.double()
    if fmt == "bf16":
        return x
    top = x.abs().amax(-1, keepdim=True)
    top = torch.where(top > 0, top, torch.ones_like(top))
    y = x * QMAX[fmt] / top
    if fmt == "int8":
        return torch.round(y) * top / 127.0
    # three bits behind the leading one, exponents from -6 on; smaller values in steps of 2^-9
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * top / 448.0


def token_rows(case, data, table, positions):
    """Keys and values of one sequence's positions, float64 [tokens, kv_heads, head_dim], byte by byte from the pages."""
    kv, d, fmt = case["kv_heads"], case["head_dim"], case["fmt"]
    k, v, km, vm, end = layout(case)
    e = element(fmt)
    page, at = table[positions // case["page"]].long(), positions % case["page"]
    head = torch.arange(kv, device=DEVICE)[None, :, None] * end
    out = []
    for first, most in ((k, km), (v, vm)):
        where = head + first + at[:, None, None] * (d * e) + torch.arange(d * e, device=DEVICE)
        raw = torch.gather(data[page], 1, where.flatten(1)).unflatten(1, (kv, d * e))
        if fmt == "bf16":
            out.append(raw.view(torch.bfloat16).double())
            continue
        where = head + most + at[:, None, None] * 2 + torch.arange(2, device=DEVICE)
        top = torch.gather(data[page], 1, where.flatten(1)).unflatten(1, (kv, 2)).view(torch.bfloat16).double()
        code = raw.view(torch.int8).double() if fmt == "int8" else raw.view(torch.float8_e4m3fn).double()
        out.append(code * top / QMAX[fmt])
    return out


def exact(case, seed):
    s = prepare(case, seed)
    table, lens, cu = s["table"], s["lens"].tolist(), s["cu"].tolist()
    kv, d = case["kv_heads"], case["head_dim"]
    if case["op"] == "store":
        for_heads = (s["rows"], kv, d)
        k, v = held(case["fmt"], s["k"].reshape(for_heads)), held(case["fmt"], s["v"].reshape(for_heads))
        if case["fmt"] != "bf16":
            return k.flatten(1), v.flatten(1)
        e = 2 * case["page"] * d
        whole = s["data"].view(torch.bfloat16).double()
        inside = torch.arange(d, device=DEVICE)
        for i, n in enumerate(lens):
            first, last = cu[i], cu[i + 1]
            pos = torch.arange(n - (last - first), n, device=DEVICE)
            page, at = table[i][pos // case["page"]].long(), pos % case["page"]
            for h in range(kv):
                where = h * e + at[:, None] * d + inside
                whole[page[:, None], where] = k[first:last, h]
                whole[page[:, None], where + case["page"] * d] = v[first:last, h]
        return whole
    outs = []
    for i, n in enumerate(lens):
        lo = max(0, n - case["window"]) if case.get("window") else 0
        k, v = [], []
        for first in range(lo, n, 2048):                             # (a part of a sequence at a time: pages are gathered whole)
            a, b = token_rows(case, s["data"], table[i], torch.arange(first, min(first + 2048, n), device=DEVICE))
            k.append(a)
            v.append(b)
        k, v = (torch.cat(x) if x else torch.zeros((0, kv, d), dtype=torch.float64, device=DEVICE) for x in (k, v))
        if case["op"] == "read":
            outs.append((k.flatten(1), v.flatten(1)))
            continue
        q = s["q"][i].double().reshape(kv, -1, d)
        logits = torch.matmul(q, k.permute(1, 2, 0).contiguous()) / math.sqrt(d)
        weights = torch.softmax(logits, -1)                          # (no tokens: nothing, and a sum of zero below)
        outs.append(torch.matmul(weights, v.permute(1, 0, 2).contiguous()).reshape(1, -1))
    if case["op"] == "read":
        return torch.cat([k for k, _ in outs]), torch.cat([v for _, v in outs])
    return torch.cat(outs)
