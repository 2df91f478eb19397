"""GPU decode attention over a 4-bit cache, on the plan for batches: equal ranges of the whole batch's
key tiles, several sequences a workgroup, for each number of KV heads a workgroup, of either head
size and type, planned in every workgroup (up to 512 sequences) and before the launch.

Sequences share the pages of a small cache.  The tolerance is test_gpu_fp4's.
"""
import math

import numpy as np
import pytest

from oracle import narrow, step
from parity_util import cuda, f64, gen, say
from test_gpu_attn_mods import counted, decode_rules, i32, near, on_gpu
from test_gpu_fp4 import ops, tolerance, u8  # noqa: F401

pytestmark = pytest.mark.gpu

# (Hq, Hkv, D, page): 8, 4, 2 and 1 KV heads a workgroup (1, 2, 4 and 8 waves a head)
LAYOUTS = [(16, 8, 128, 16), (16, 8, 64, 64), (8, 4, 128, 64), (8, 4, 64, 16), (6, 2, 128, 16), (3, 3, 64, 16), (5, 1, 128, 64)]


def check(ops, dtype, ctx, Hq, Hkv, D, bs, rules, max_ctx=None):
    import torch
    B, n, nb = len(ctx), max(ctx), 120
    rng = np.random.default_rng([B, n, Hkv, D, bs])
    caches = []
    for _ in range(2):
        flat = rng.integers(0, 256, size=(nb, Hkv, bs * (D // 2 + D // 32))).astype(np.uint8)
        flat[:, :, bs * D // 2:] = rng.integers(124, 129, size=(nb, Hkv, bs * D // 32))
        flat[0, :, bs * D // 2:] = 255  # page 0, which lies behind every sequence's last, is NaN
        caches.append(flat.reshape(nb, Hkv, bs, D // 2 + D // 32))
    table = rng.integers(1, nb, size=(B, -(-n // bs) + 1)).astype(np.int32)
    for b, c in enumerate(ctx):
        table[b, -(-c // bs):] = 0
    q = gen(B, "q", (B, Hq, D), dtype, 1.5)
    table[B // 3, 1::5], table[B // 2, 2::7] = -1, nb  # (pages that are not there)
    scale = 1.0 / math.sqrt(D)
    values = [narrow.unpack(c) for c in caches]
    dev = [u8(c) for c in caches]
    for kw in rules:
        say(f"attn_decode_fp4 {dtype} B={B} {sum(ctx)} keys, most {n}, Hq={Hq} Hkv={Hkv} D={D} bs={bs} {sorted(kw)}")
        out = torch.full((B, Hq, D), float("nan"), dtype=q.dtype, device="cuda")
        args = cuda(q), *dev, i32(table), i32(ctx), max_ctx or n, scale
        ops.opscale_attn_decode_fp4(*args, out=out, **on_gpu(kw))
        again = ops.opscale_attn_decode_fp4(*args, **on_gpu(kw))
        torch.cuda.synchronize()
        assert torch.equal(out, again), "two runs differ"
        ref, weighted = (step.attn_decode_mod(f64(q), values[0], v, table, ctx, scale, **kw)
                         for v in (values[1], np.abs(values[1])))
        dot = scale * np.abs(f64(q)).sum(-1).max() * np.nanmax(np.abs(values[0]))
        near(f64(out.cpu()), ref, tolerance(ref, weighted, dtype, D, n, dot, kw.get("softcap"), counted(kw, n)), "decode")


def lengths(B, seed):
    """Sequences of no keys, of a tile or two, of some tiles, and one over several windows of page ids."""
    rng = np.random.default_rng([seed, B])
    ctx = np.where(rng.random(B) < 0.2, rng.integers(100, 700, B), rng.integers(0, 70, B))
    ctx[[0, B // 3 + 1, B - 1]], ctx[B // 3], ctx[B // 2] = 0, 700, 5000 + int(rng.integers(0, 100))
    return [int(n) for n in ctx]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D,bs", LAYOUTS)
@pytest.mark.parametrize("B", [100, 513])
def test_equal_ranges(ops, dtype, B, Hq, Hkv, D, bs):
    ctx = lengths(B, D)
    check(ops, dtype, ctx, Hq, Hkv, D, bs, [decode_rules("all" if B == 100 else "prefix_window", ctx, Hq), {}])


@pytest.mark.parametrize("Hq,Hkv,D,bs", LAYOUTS)
def test_long_ranges(ops, Hq, Hkv, D, bs):
    """Ranges of fifteen tiles and more, over windows of page ids and from one sequence into the next (the lengths
    told as short, so that as many workgroups as two a sequence take them)."""
    ctx = [1500, 0, 1, 4000, 40, 0, 1200, 33] * 17
    kw = dict(window=900, prefix_lens=np.array([1100, 0, 1, 40, 0, 0, 1200, 7] * 17), softcap=30.0)
    check(ops, "bf16", ctx, Hq, Hkv, D, bs, [{}, kw], max_ctx=16)
