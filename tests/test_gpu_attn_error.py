"""GPU attention with score modifiers, element by element within the bounds that
attn_error derives (their own checks: test_attn_error.py)."""
import math

import numpy as np
import pytest

from attn_error import row
from oracle import step
from parity_util import cuda, f64, gen, say
from test_gpu_attn_mods import f32, i32, on_gpu, ops, paged, slopes_of  # noqa: F401

pytestmark = pytest.mark.gpu


def within(got, want, bound, what):
    assert np.isfinite(got).all(), f"{what}: not finite"
    r = np.abs(got - want) / bound
    say(f"  {what}: {r.max():.3f} of the bound")
    assert r.max() <= 1.0, f"{what}: {r.max():.3f} of the bound at {np.unravel_index(r.argmax(), r.shape)}"


# The modifiers of a call: (cap, slopes, window, prefix)
RULES = {"none": (0.0, False, 0, 0), "cap": (5.0, False, 0, 0), "cap50": (50.0, False, 0, 0), "bias": (0.0, True, 0, 0),
         "cap_bias": (30.0, True, 0, 0), "window": (0.0, False, 20, 0), "prefix_window": (50.0, True, 24, 9)}


def _modifiers(name, Hq, B):
    cap, bias, window, prefix = RULES[name]
    kw = dict(softcap=cap, window=window)
    if bias:
        kw["slopes"] = slopes_of(Hq)
    if prefix:
        kw["prefix_lens"] = np.full(B, prefix)
    return kw


def _keys(kw, i, n, causal=True):
    prefix = 0 if kw.get("prefix_lens") is None else int(kw["prefix_lens"][0])
    return step.visible(i, n, causal, kw["window"], prefix, 0)


# ----------------------------------------------------------------- decode ---
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", RULES)
@pytest.mark.parametrize("D", [64, 128])
def test_decode(ops, dtype, name, D):
    """bf16: the probabilities reach V in 16 bits."""
    import torch
    ctx, Hq, Hkv, bs, scale = [1, 2, 5, 33, 70, 150, 400], 8, 2, 16, 1 / math.sqrt(D)
    kw = _modifiers(name, Hq, len(ctx))
    say(f"attn_decode_mod {dtype} D={D} {name}")
    for std in (0.3, 1.5):
        table, kc, vc = paged(91, ctx, Hkv, D, bs, dtype, std=std)
        q = gen(91, "q", (len(ctx), Hq, D), dtype, std)
        got = ops.opscale_attn_decode_mod(cuda(q), cuda(kc), cuda(vc), i32(table), i32(ctx), max(ctx), scale, **on_gpu(kw))
        torch.cuda.synchronize()
        want, bound = np.zeros((2, len(ctx), Hq, D))
        for b, n in enumerate(ctx):
            keys = _keys(kw, n - 1, n)
            for h in range(Hq):
                k, v = (f64(c)[table[b, keys // bs], keys % bs, h // (Hq // Hkv)] for c in (kc, vc))
                want[b, h], bound[b, h] = row(f64(q)[b, h], k, v, n - 1, keys, scale, kw["softcap"],
                                              float(kw["slopes"][h]) if "slopes" in kw else 0.0, dtype, pieces=2)
        within(f64(got.cpu()), want, bound, f"std {std}")
