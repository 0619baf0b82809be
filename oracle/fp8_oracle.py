"""8-bit floats under power-of-two scales, the 8-bit K/V cache and products of 8-bit matrices, written out as their definitions in float64.

A code has a sign, 4 exponent bits (bias 7) and 3 mantissa bits; 0x7f and 0xff are NaN, the largest value is 448.  A block's scale is 2^e, e
the smallest integer with amax <= 448 * 2^e, cut to [-116, 119], amax its largest finite magnitude; x / 2^e goes to the nearest
code, ties to the even one, magnitudes above 448 to 448, what is not finite to 0x7f.  The attention over cached values is that of
`kv4_oracle.attend`.
"""
from __future__ import annotations

import math

import numpy as np

PAGE = 16
BLOCK = 128
LOWEST, HIGHEST = -116, 119
MAGNITUDES = np.array([c * 2.0 ** -9 if c < 8 else (8 + c % 8) * 2.0 ** (c // 8 - 10) for c in range(127)])


def exponent(amax: float) -> int:
    e = LOWEST
    while e < HIGHEST and amax > math.ldexp(448.0, e):
        e += 1
    return e


def top(x) -> float:
    """Largest finite magnitude, 0 if there is none."""
    x = np.abs(np.asarray(x, np.float64))
    return float(x[np.isfinite(x)].max(initial=0.0))


def encode(x, e):
    """float64 values under 2^e -> codes."""
    x = np.asarray(x, np.float64)
    z = np.minimum(np.abs(np.where(np.isfinite(x), x, 0.0)) * 2.0 ** -float(e), 448.0)
    hi = np.clip(np.searchsorted(MAGNITUDES, z), 1, 126)
    lo = hi - 1
    to_lo, to_hi = z - MAGNITUDES[lo], MAGNITUDES[hi] - z
    code = np.where((to_lo < to_hi) | ((to_lo == to_hi) & (lo % 2 == 0)), lo, hi)
    code = np.where(np.isfinite(x), code | (np.signbit(x).astype(int) << 7), 0x7f)
    return code.astype(np.uint8)


def decode(codes, e):
    codes = np.asarray(codes, np.uint8)
    mag = np.append(MAGNITUDES, np.nan)[codes & 127]
    return np.where(codes & 128, -mag, mag) * np.exp2(np.asarray(e, np.float64))


# ------------------------------------------------------------------------------------------------ the cache
def page_bytes(n_kv: int, hd: int) -> int:
    return n_kv * PAGE * hd + -(-n_kv // 128) * 128


def places(hd: int, v: bool):
    """Where code (token, head_dim index) lies in a block: int [16, hd]."""
    t, d = np.arange(PAGE)[:, None], np.arange(hd)[None, :]
    return d // 4 * 64 + t // 4 * 16 + d % 4 * 4 + t % 4 if v else t * hd + d


def write(pool, page, first, tokens, v):
    """Tokens float64 [n, n_kv, hd] into slots first .. first + n - 1 of a page of pool uint8 [n_pages, page_bytes]."""
    n, n_kv, hd = tokens.shape
    at, own = places(hd, v), pool[page]
    for h in range(n_kv):
        block, x = own[h * PAGE * hd:(h + 1) * PAGE * hd], tokens[:, h].copy()
        x[~np.isfinite(x).all(-1)] = np.nan
        e, codes = exponent(top(x)), np.zeros((PAGE, hd), np.uint8)
        if first > 0:
            old = min(max(int(own[n_kv * PAGE * hd + h]) - 127, LOWEST), HIGHEST)
            e, codes = max(e, old), block[at]
            if e != old:
                codes = encode(decode(codes, old), e)
        codes[first:first + n] = encode(x, e)
        block[at] = codes
        own[n_kv * PAGE * hd + h] = e + 127


def read(pool, page, n_kv, hd, v):
    """float64 [16, n_kv, hd] of a page."""
    own = pool[page]
    return np.stack([decode(own[h * PAGE * hd:(h + 1) * PAGE * hd][places(hd, v)], int(own[n_kv * PAGE * hd + h]) - 127) for h in range(n_kv)], 1)


def write_run(pool, table, start, tokens, v):
    """Tokens of one sequence at positions start, start + 1, ..., page by page; unset pages are passed over."""
    t = 0
    while t < len(tokens):
        page, first = (start + t) // PAGE, (start + t) % PAGE
        n = min(PAGE - first, len(tokens) - t)
        if page < len(table) and 0 <= table[page] < len(pool):
            write(pool, table[page], first, tokens[t:t + n], v)
        t += n


def read_run(pool, table, start, n, n_kv, hd, v):
    pages = np.arange(start // PAGE, -(-(start + n) // PAGE))
    if len(pages) == 0:
        return np.zeros((0, n_kv, hd))
    return np.concatenate([read(pool, table[p], n_kv, hd, v) for p in pages])[start - pages[0] * PAGE:][:n]


# ------------------------------------------------------------------------------------------------ matrices
def quantise(x):
    """float64 [rows, k] -> codes uint8 [rows, k rounded up to 128], scale bytes uint8 [blocks, rows rounded up to 16]."""
    rows, k = x.shape
    blocks = -(-k // BLOCK)
    codes, scales = np.zeros((rows, blocks * BLOCK), np.uint8), np.full((blocks, -(-rows // 16) * 16), 127, np.uint8)
    for r in range(rows):
        for b in range(blocks):
            part = x[r, b * BLOCK:(b + 1) * BLOCK]
            e = exponent(top(part))
            codes[r, b * BLOCK:b * BLOCK + len(part)] = encode(part, e)
            scales[b, r] = e + 127
    return codes, scales


def value(codes, scales, k=None):
    """float64 [rows, k]."""
    e = np.repeat(scales.T[:len(codes)].astype(np.float64) - 127, BLOCK, 1)
    return decode(codes, e)[:, :k]
