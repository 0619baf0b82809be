"""The 4-bit K/V cache and the attention over it, written out as their definitions in float64.

A group of 32 values along head_dim of one token and kv head: scale 2^e, e the smallest integer with max|x| <= 7 * 2^e, cut to
[-126, 125], and every x / 2^e to the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6 with its sign, ties to the even code.  A group with an
infinity or a NaN is all NaN.
"""
from __future__ import annotations

import math

import numpy as np

GROUP = 32
PAGE = 16
MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def block_bytes(hd: int) -> int:
    return 8 * hd + hd // 2


def quantise(x):
    """float64 [..., hd] -> codes uint8 [..., hd] (0..15) and scale bytes uint8 [..., hd / 32]."""
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, GROUP)
    codes = np.zeros(g.shape, np.uint8)
    scales = np.zeros(g.shape[:-1], np.uint8)
    top = np.max(np.abs(g), -1)
    for at in np.ndindex(*top.shape):
        t = top[at]
        if not math.isfinite(t):
            scales[at] = 255
            continue
        e = -126
        while e < 125 and t > math.ldexp(7.0, e):
            e += 1
        scales[at] = e + 127
    fine = scales != 255
    z = np.where(fine[..., None], g, 0.0) * np.exp2(127.0 - scales.astype(np.float64))[..., None]
    far = np.abs(np.abs(z)[..., None] - MAGNITUDES)          # distance to each magnitude; ties: the even code
    best = far.min(-1, keepdims=True)
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])
    codes[...] = order[np.argmax((far == best)[..., order], -1)]
    codes = np.where(fine[..., None], codes | (np.signbit(g).astype(np.uint8) << 3), 0).astype(np.uint8)
    return codes.reshape(x.shape), scales


def value(codes, scales):
    """The inverse, float64 [..., hd]."""
    g = codes.reshape(*codes.shape[:-1], -1, GROUP)
    v = np.where(g & 8, -1.0, 1.0) * MAGNITUDES[g & 7] * np.exp2(scales.astype(np.float64) - 127.0)[..., None]
    return np.where((scales == 255)[..., None], np.nan, v).reshape(codes.shape)


def put(k_pool, v_pool, page, off, k_codes, k_scales, v_codes, v_scales):
    """Writes one token ([n_kv, hd] codes, [n_kv, hd / 32] scales) into pools uint8 [n_pages, n_kv, block]."""
    hd = k_codes.shape[-1]
    pack = lambda c: (c[..., 0::2] | (c[..., 1::2] << 4)).astype(np.uint8)
    k, v, cut = pack(k_codes), pack(v_codes), 8 * hd
    k_pool[page, :, off * hd // 2:(off + 1) * hd // 2] = k
    k_pool[page, :, cut + off * (hd // GROUP):cut + (off + 1) * (hd // GROUP)] = k_scales
    for c in range(hd // 8):
        v_pool[page, :, (c * PAGE + off) * 4:(c * PAGE + off) * 4 + 4] = v[:, 4 * c:4 * c + 4]
    for g in range(hd // GROUP):
        v_pool[page, :, cut + g * PAGE + off] = v_scales[:, g]


def take(k_pool, v_pool, page, off):
    """The values of one token: two float64 [n_kv, hd]."""
    n_kv, hd = k_pool.shape[1], k_pool.shape[2] * 2 // 17
    cut = 8 * hd
    spread = lambda b: np.stack([b & 15, b >> 4], -1).reshape(n_kv, hd)
    k = spread(k_pool[page, :, off * hd // 2:(off + 1) * hd // 2])
    ks = k_pool[page, :, cut + off * (hd // GROUP):cut + (off + 1) * (hd // GROUP)]
    v = spread(np.concatenate([v_pool[page, :, (c * PAGE + off) * 4:(c * PAGE + off) * 4 + 4] for c in range(hd // 8)], -1))
    vs = np.stack([v_pool[page, :, cut + g * PAGE + off] for g in range(hd // GROUP)], -1)
    return value(k, ks), value(v, vs)


def attend(q, k, v, prefix):
    """q [L, n_q, hd] against cached keys and values [prefix + L, n_kv, hd], row t seeing keys <= prefix + t.  Returns the
    output and, element by element, sum p|v| / sum p (what a rounding of the weights is multiplied with).  Values that a row does
    not see do not reach it, NaN included."""
    L, n_q, hd = q.shape
    group = n_q // k.shape[1]
    out, spread = np.zeros((L, n_q, hd)), np.zeros((L, n_q, hd))
    sees = np.arange(prefix + L)[None, :] <= prefix + np.arange(L)[:, None]
    for h in range(n_q):
        kk, vv = k[:, h // group], v[:, h // group]
        with np.errstate(invalid="ignore"):
            s = np.where(sees, q[:, h] @ np.nan_to_num(kk).T / math.sqrt(hd), -np.inf)
            bad_k = np.isnan(kk).any(-1)
            p = np.exp(s - s.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
        clean = np.nan_to_num(vv)
        out[:, h], spread[:, h] = p @ clean, p @ np.abs(clean)
        out[:, h][(sees & bad_k).any(-1)] = np.nan
        out[:, h][(sees.astype(float) @ np.isnan(vv)) > 0] = np.nan
    return out, spread
