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
