"""fp64 definitions of the attention path's further operators (test
infrastructure only): norms of the query and key heads with the rotation, the
tables of a step, and attention with score modifiers and masks.

Each is the definition written out, row by row; none shares a formula with the
kernels' way of computing it.
"""
from __future__ import annotations

import math

import numpy as np


def _f64(a) -> np.ndarray:
    return np.asarray(a, dtype=np.float64)


# -------------------------------------------------------- rotation and norm --
def rope_frequencies(rot, theta, scaling="none", factor=1.0, low=1.0, high=4.0, original_len=8192):
    """(frequencies [rot / 2], magnitude).  A frequency that turns `high` times or
    more over the original length stays, one that turns `low` times or fewer is
    divided by the factor; between, "bands" mixes by the turns, "ramp" by the
    pair's index."""
    out, mag = [], 1.0
    if scaling == "ramp":
        mag = 0.1 * math.log(factor) + 1.0

        def index(turns):  # theta^(-2 i / rot) = 2 pi turns / original_len, solved for i
            return -rot / 2 * math.log(2 * math.pi * turns / original_len) / math.log(theta)

        lo, hi = max(0, math.floor(index(high))), min(rot - 1, math.ceil(index(low)))
    for i in range(rot // 2):
        f = theta ** (-2.0 * i / rot)
        turns = original_len * f / (2 * math.pi)
        if scaling == "none":
            w = 0.0
        elif scaling == "linear":
            w = 1.0
        elif scaling == "bands":
            w = min(1.0, max(0.0, (high - turns) / (high - low)))
        else:
            w = min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
        out.append(w * f / factor + (1.0 - w) * f)
    return np.array(out), mag


def qk_norm_rope(x, w, eps, positions, freq, interleaved, magnitude=1.0) -> np.ndarray:
    """x [T, H, D]: each head normed (w not None), then its first 2 len(freq) elements
    turned pair by pair."""
    y = _f64(x).copy()
    T, H, D = y.shape
    if w is not None:
        y = y / np.sqrt(np.mean(y * y, axis=-1, keepdims=True) + eps) * _f64(w)
    n = 0 if freq is None else len(freq)
    out = y.copy()
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        t = _f64(positions) * float(freq[i])
        c, s = magnitude * np.cos(t)[:, None], magnitude * np.sin(t)[:, None]
        out[:, :, a] = y[:, :, a] * c - y[:, :, b] * s
        out[:, :, b] = y[:, :, b] * c + y[:, :, a] * s
    return out


# ------------------------------------------------------------- step tables --
def block_tables(context_lens, new_lens, table, free_blocks, free_begin, block_size, max_tokens):
    """(cu_seqlens, positions, slots, kv_lens, free_next, table): token by token,
    page by page."""
    B, cols = np.asarray(table).shape
    table = np.array(table, np.int64)
    cu, positions, slots, kv = [0], [0] * max_tokens, [-1] * max_tokens, []
    at = int(free_begin)
    for b in range(B):
        have, new = max(0, int(context_lens[b])), max(0, int(new_lens[b]))
        new = min(new, max_tokens - cu[-1])
        end = min(have + new, cols * block_size)
        kv.append(end)
        first_page = min(-(-have // block_size), cols)
        for j in range(first_page, -(-end // block_size)):
            table[b, j] = free_blocks[at] if 0 <= at < len(free_blocks) else -1
            at += 1
        for i in range(new):
            p, t = have + i, cu[-1] + i
            positions[t] = p
            j = p // block_size
            if j < cols and table[b, j] >= 0:
                slot = int(table[b, j]) * block_size + p % block_size
                slots[t] = slot if slot < 2 ** 31 else -1
        cu.append(cu[-1] + new)
    return cu, positions, slots, kv, at, table


# ---------------------------------------------- attention with modifiers ----
def _row(q, k, v, scale, i, keys, softcap, slope):
    """One output row: query q at position i over the visible positions `keys`."""
    if len(keys) == 0:
        return np.zeros(v.shape[-1])
    s = scale * (_f64(k)[keys] @ _f64(q))
    if softcap > 0:
        s = softcap * np.tanh(s / softcap)
    s = s - slope * np.abs(i - np.asarray(keys, np.float64))
    p = np.exp(s - s.max())
    return (p / p.sum()) @ _f64(v)[keys]


def visible(i, n, causal, window, prefix, start):
    """Positions of [0, n) that the query at i sees."""
    j = np.arange(n)
    own = j >= start
    if causal:
        own &= j <= i
    if window > 0:
        own &= np.abs(i - j) < window
    return np.nonzero(own | (j < prefix))[0]


def attn_prefill_mod(q, k, v, cu_seqlens, scale, causal=True, softcap=0.0, slopes=None, window=0, prefix_lens=None,
                     doc_starts=None, rows=None) -> np.ndarray:
    """q [T, Hq, D], k and v [T, Hkv, D].  rows: (token, head) pairs to compute,
    [len(rows), D]; all of them, [T, Hq, D], if None."""
    T, Hq, D = q.shape
    group = Hq // k.shape[1]
    cu = np.asarray(cu_seqlens, np.int64)
    every = rows is None
    rows = [(t, h) for t in range(int(cu[-1])) for h in range(Hq)] if every else rows
    out = np.zeros((len(rows), D))
    for r, (t, h) in enumerate(rows):
        b = int(np.searchsorted(cu, t, side="right")) - 1
        s0, n = int(cu[b]), int(cu[b + 1] - cu[b])
        prefix = 0 if prefix_lens is None else int(prefix_lens[b])
        start = 0 if doc_starts is None else int(doc_starts[t])
        keys = visible(t - s0, n, causal, window, prefix, start)
        out[r] = _row(q[t, h], k[s0:s0 + n, h // group], v[s0:s0 + n, h // group], scale, t - s0, keys, softcap,
                      0.0 if slopes is None else float(slopes[h]))
    return out.reshape(T, Hq, D) if every else out


def attn_decode_mod(q, k_cache, v_cache, block_table, context_lens, scale, softcap=0.0, slopes=None, window=0,
                    prefix_lens=None, doc_starts=None) -> np.ndarray:
    """q [B, Hq, D], caches [num_blocks, block_size, Hkv, D]; keys of a page outside
    the cache are not there."""
    B, Hq, D = q.shape
    nb, bs, Hkv, _ = k_cache.shape
    out = np.zeros((B, Hq, D))
    for b in range(B):
        n = min(max(int(context_lens[b]), 0), block_table.shape[1] * bs)
        prefix = 0 if prefix_lens is None else int(prefix_lens[b])
        start = 0 if doc_starts is None else int(doc_starts[b])
        keys = visible(n - 1, n, True, window, prefix, start)
        page = np.asarray(block_table[b], np.int64)[keys // bs]
        ok = (page >= 0) & (page < nb)
        page, off, pos = page[ok], (keys % bs)[ok], keys[ok]
        for h in range(Hq):
            k, v = _f64(k_cache[page, off, h // (Hq // Hkv)]), _f64(v_cache[page, off, h // (Hq // Hkv)])
            if len(pos) == 0:
                continue
            s = scale * (k @ _f64(q[b, h]))
            if softcap > 0:
                s = softcap * np.tanh(s / softcap)
            s = s - (0.0 if slopes is None else float(slopes[h])) * (n - 1 - pos)
            p = np.exp(s - s.max())
            out[b, h] = (p / p.sum()) @ v
    return out
