"""Float64 definition of the paged key-value cache: what a row is held as, what it stands for, where a token lies, and the
attention of one new token.  numpy only; shares nothing with the device code."""
import numpy as np

QMAX = {"int8": 127.0, "e4m3": 448.0}


def e4m3_values():
    """The 256 values of the OCP 8-bit float with 4 exponent and 3 fraction bits (bias 7; 0x7F and 0xFF are NaN)."""
    out = np.empty(256)
    for code in range(256):
        sign, e, f = (-1.0 if code & 0x80 else 1.0), code >> 3 & 15, code & 7
        out[code] = sign * (f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))
        if code & 0x7F == 0x7F:
            out[code] = np.nan
    return out


def hold(x, fmt):
    """Rows x [..., d] float64 (bfloat16 values) -> (codes uint8 [..., d], maxima float64 [...]); maxima NaN where a row is not finite."""
    finite = np.isfinite(x).all(-1)
    x = np.where(finite[..., None], x, 0.0)
    m = np.abs(x).max(-1)
    y = x * QMAX[fmt] / np.where(m > 0, m, 1.0)[..., None]
    if fmt == "int8":
        codes = np.rint(y).astype(np.int8).view(np.uint8)
    else:
        grid = e4m3_values()[:127]                                   # the numbers >= 0, ascending with their codes
        a = np.abs(y)
        up = np.clip(np.searchsorted(grid, a), 1, 126)
        low, high = a - grid[up - 1], grid[up] - a
        near = np.where((high < low) | ((high == low) & (up % 2 == 0)), up, up - 1)
        codes = (near + np.where(y < 0, 128, 0)).astype(np.uint8)
    return codes, np.where(finite, m, np.nan)


def stands_for(codes, m, fmt):
    c = codes.view(np.int8).astype(np.float64) if fmt == "int8" else e4m3_values()[codes]
    return c * m[..., None] / QMAX[fmt]


def place(pos, table_row, n_pages, page_size):
    """(page, token of the page), or None."""
    if pos < 0 or pos // page_size >= len(table_row):
        return None
    page = int(table_row[pos // page_size])
    return (page, pos % page_size) if 0 <= page < n_pages else None


def attend_one(q, k, v, scale):
    """q [heads, d], k and v [tokens, kv_heads, d], float64 -> (out [heads, d], sum of weight * |v|, largest sum of |q k| scale)."""
    heads, d = q.shape
    group = heads // k.shape[1] if k.shape[1] else 1
    out, mass, size = np.zeros((heads, d)), np.zeros((heads, d)), np.zeros(heads)
    for h in range(heads):
        kh, vh = k[:, h // group], v[:, h // group]
        if not len(kh):
            continue
        logits = kh @ q[h] * scale
        size[h] = (np.abs(kh) @ np.abs(q[h])).max() * abs(scale)
        top = logits.max()
        if top == -np.inf:
            continue
        w = np.exp(logits - top)
        w /= w.sum()
        out[h], mass[h] = w @ vh, w @ np.abs(vh)
    return out, mass, size


# ---------------------------------------------------------------------------------------------- 4 bits, blocks of 32 with one power of two

MX_GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def mx_blocks(d):
    return -(-d // 32)


def mx_hold(x):
    """Rows x [..., d] float64 (bfloat16 values) -> (codes uint8 [..., d / 2], the even dimension in the low half, exponent bytes uint8
    [..., blocks]); a block with an infinity or a NaN has the byte 255 and codes 0."""
    d = x.shape[-1]
    codes, exps = np.zeros(x.shape, dtype=np.uint8), np.zeros(x.shape[:-1] + (mx_blocks(d),), dtype=np.uint8)
    for i in range(mx_blocks(d)):
        b = x[..., 32 * i:32 * i + 32]
        finite = np.isfinite(b).all(-1)
        b = np.where(finite[..., None], b, 0.0)
        m = np.abs(b).max(-1)
        e = np.floor(np.log2(np.where(m > 0, m, 1.0) / 7.0)) - 1        # the smallest with m <= 7 * 2^e: from below, by comparing
        for _ in range(3):
            e = np.where(m > 7.0 * 2.0 ** e, e + 1, e)
        e = np.clip(np.where(m > 0, e, -125), -125, 125)
        a = np.minimum(np.abs(b) / 2.0 ** e[..., None], 6.0)
        up = np.clip(np.searchsorted(MX_GRID, a), 1, 7)
        low, high = a - MX_GRID[up - 1], MX_GRID[up] - a
        near = np.where((high < low) | ((high == low) & (up % 2 == 0)), up, up - 1)
        codes[..., 32 * i:32 * i + 32] = np.where(finite[..., None], near + 8 * np.signbit(b), 0)
        exps[..., i] = np.where(finite, e + 127, 255)
    return codes[..., 0::2] | codes[..., 1::2] << 4, exps


def mx_stands_for(codes, exps):
    c = np.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[:-1] + (2 * codes.shape[-1],))
    v = np.where(c > 7, -1.0, 1.0) * MX_GRID[c & 7]
    e = np.repeat(exps.astype(np.int64), 32, -1)[..., :c.shape[-1]]
    return np.where(e == 255, np.nan, v * 2.0 ** (e - 127.0))
