"""Blocks of few bits, by definition: e4m3 and e2m1 elements with power-of-two scales,
the linear of e4m3 operands, and a paged KV cache in 4 bits (fp64, NumPy).

The formats are the public ones: e4m3 (bias 7, largest 448, 0x7f and 0xff NaN, no
infinities) and e2m1 (bias 1, largest 6).  Scales are 2^e with the least e in a range
that brings a block's largest magnitude to 448 or less, of e2m1 to 7 or less.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK, GROUP = 128, 32
LOWEST, HIGHEST = -100, {"e4m3": 120, "e2m1": 125}
MOST = {"e4m3": 448.0, "e2m1": 7.0}


def _decode(bits, exp_bits, frac_bits, bias):
    sign = -1.0 if bits >> (exp_bits + frac_bits) & 1 else 1.0
    e, f = bits >> frac_bits & ((1 << exp_bits) - 1), bits & ((1 << frac_bits) - 1)
    size = 1 << frac_bits
    return sign * (f / size * 2.0 ** (1 - bias) if e == 0 else (1 + f / size) * 2.0 ** (e - bias))


#: the value of each code
E4M3 = np.array([math.nan if c & 127 == 127 else _decode(c, 4, 3, 7) for c in range(256)])
E2M1 = np.array([_decode(c, 2, 1, 1) for c in range(16)])
VALUES = {"e4m3": E4M3, "e2m1": E2M1}


def encode(x, kind):
    """The codes nearest to x, ties to the even code, saturated."""
    x = np.asarray(x, np.float64)
    pos = VALUES[kind][:127 if kind == "e4m3" else 8]
    hi = np.clip(np.searchsorted(pos, np.abs(x)), 1, len(pos) - 1)
    lo = hi - 1
    below, above = np.abs(x) - pos[lo], pos[hi] - np.abs(x)
    code = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    return code + np.where(np.signbit(x), len(VALUES[kind]) // 2, 0)


def exponent(most, kind):
    """The least e in range with most <= MOST 2^e, else the highest."""
    e = LOWEST
    while e < HIGHEST[kind] and most > MOST[kind] * 2.0 ** e:
        e += 1
    return e


def quantize_fp8(x):
    """x [M, K] -> (e4m3 values [M, K], scales [ceil(K / 128), M]); NaN scales for blocks that are not finite."""
    x = np.asarray(x, np.float64)
    M, K = x.shape
    values, scales = np.zeros((M, K)), np.zeros((-(-K // BLOCK), M))
    for m in range(M):
        for b in range(scales.shape[0]):
            block = x[m, b * BLOCK:(b + 1) * BLOCK]
            if not np.isfinite(block).all():
                scales[b, m] = math.nan
                continue
            scales[b, m] = 2.0 ** exponent(np.abs(block).max(), "e4m3")
            values[m, b * BLOCK:(b + 1) * BLOCK] = E4M3[encode(block / scales[b, m], "e4m3")]
    return values, scales


def linear_fp8(x, x_scales, w, w_scales, bias=None):
    """x [M, K] and w [N, K]: the values of e4m3 elements."""
    y = np.zeros((x.shape[0], w.shape[0]))
    for b in range(x_scales.shape[0]):
        k = slice(b * BLOCK, (b + 1) * BLOCK)
        rows = np.repeat(w_scales[:, b], BLOCK)[:w.shape[0]]
        y += (x[:, k] @ w[:, k].T) * np.outer(x_scales[b], rows)
    return y if bias is None else y + bias


def cached(x):
    """What a cache in 4 bits holds for heads x [..., D]."""
    x = np.asarray(x, np.float64)
    out = np.empty(x.shape)
    for at in np.ndindex(*x.shape[:-1]):
        for g in range(0, x.shape[-1], GROUP):
            block = x[at][g:g + GROUP]
            if not np.isfinite(block).all():
                out[at][g:g + GROUP] = math.nan
                continue
            scale = 2.0 ** exponent(np.abs(block).max(), "e2m1")
            out[at][g:g + GROUP] = E2M1[encode(block / scale, "e2m1")] * scale
    return out


def pack(x):
    """Pages [nb, block_size, Hkv, D] of numbers -> bytes [nb, Hkv, block_size, D / 2 + D / 32]."""
    x = np.asarray(x, np.float64)
    nb, bs, H, D = x.shape
    out = np.zeros((nb, H, bs * (D // 2 + D // GROUP)), np.uint8)
    for p, r, h in np.ndindex(nb, bs, H):
        for g in range(D // GROUP):
            block = x[p, r, h, g * GROUP:(g + 1) * GROUP]
            e, codes = 128, np.zeros(GROUP, np.int64)
            if np.isfinite(block).all():
                e = exponent(np.abs(block).max(), "e2m1")
                codes = encode(block / 2.0 ** e, "e2m1")
            at = r * (D // 2) + g * GROUP // 2
            out[p, h, at:at + GROUP // 2] = codes[0::2] | codes[1::2] << 4
            out[p, h, bs * (D // 2) + g * bs + r] = e + 127
    return out.reshape(nb, H, bs, D // 2 + D // GROUP)


def unpack(pages):
    """The numbers that such bytes stand for, [nb, block_size, Hkv, D]."""
    nb, H, bs, row = pages.shape
    D = row * 32 // 17
    flat = pages.reshape(nb, H, -1).astype(np.int64)
    codes = flat[..., :bs * D // 2].reshape(nb, H, bs, D // 2)
    e = flat[..., bs * D // 2:].reshape(nb, H, D // GROUP, bs)
    x = np.stack([E2M1[codes & 15], E2M1[codes >> 4]], -1).reshape(nb, H, bs, D // GROUP, GROUP)
    scale = np.where(e == 255, math.nan, np.ldexp(1.0, np.minimum(e, 254) - 127)).swapaxes(2, 3)
    return (x * scale[..., None]).reshape(nb, H, bs, D).swapaxes(1, 2)
