"""The attention half of a layer on e4m3 operands and a cache in 4 bits, as a serving step runs it:
a batch of prompts, the cache read back, then decode steps from one graph.  Each operator's result is
compared with its definition on the operands that it was given: what is exact, exactly, the rest
within the bounds of test_gpu_fp8 and test_gpu_fp4."""
import math

import numpy as np
import pytest

from oracle import narrow, step
from parity_util import cuda, f64, gen, say
from test_gpu_attn_mods import i32, near, ops  # noqa: F401
from test_gpu_fp4 import slots_of, tolerance
from test_gpu_fp8 import operands, reference

pytestmark = pytest.mark.gpu
H, HQ, HKV, D, BS, EPS = 528, 8, 2, 64, 16, 1e-6  # a K block of 16 behind four of 128


class Half:
    """Weights, caches and tables of the half, on the GPU."""

    def __init__(self, ops, ctx, cols, spare, dtype):
        import torch
        self.ops, self.dtype = ops, torch.bfloat16 if dtype == "bf16" else torch.float32
        B = len(ctx)
        nb = B * cols + 3
        self.free = np.random.default_rng(5).permutation(nb - spare).astype(np.int32)
        self.d = dict(ctx=i32(ctx), table=i32(np.full((B, cols), -1)), begin=i32([0]))
        self.free_d = i32(self.free)
        self.kc = torch.full((nb, HKV, BS, D // 2 + D // 32), 255, dtype=torch.uint8, device="cuda")
        self.vc = self.kc.clone()
        e4 = lambda a: torch.from_numpy(a).cuda().view(torch.float8_e4m3fn)  # noqa: E731
        self.w = [operands(1, N, K, 31 + N)[2:] for N, K in (((HQ + 2 * HKV) * D, H), (H, HQ * D))]
        self.wd = [(e4(c), cuda(torch.from_numpy(s * np.float32(2.0 ** -3)))) for c, s in self.w]
        self.w = [(c, s * np.float32(2.0 ** -3)) for c, s in self.w]
        self.norm = cuda(gen(3, "q", (H,), dtype))
        self.freq, self.mag = ops.opscale_rope_frequencies(D // 2, 10000.0, device="cuda")

    def tables(self, new, tokens):
        d = self.d
        return self.ops.opscale_block_tables(d["ctx"], new, d["table"], self.free_d, d["begin"], BS, tokens)

    def run(self, x, new, longest, decode):
        """Every operand and result, for the checks."""
        o, d = self.ops, self.d
        T = x.shape[0]
        cu, pos, slots, kv, begin = self.tables(new, T)
        h = o.opscale_rmsnorm(x, self.norm, eps=EPS)
        h8, hs = o.opscale_quantize_fp8(h)
        qkv = o.opscale_linear_fp8(h8, hs, *self.wd[0], dtype=self.dtype)
        raw = qkv.clone()
        q, k, v = qkv.view(T, HQ + 2 * HKV, D).split([HQ, HKV, HKV], 1)
        o.opscale_qk_norm_rope(q, k, pos, self.freq, magnitude=self.mag)
        o.opscale_kv_write_fp4(k, v, self.kc, self.vc, slots)
        if decode:
            attn = o.opscale_attn_decode_fp4(q, self.kc, self.vc, d["table"], kv, longest, D ** -0.5, softcap=30.0,
                                             window=60)
        else:
            attn = o.opscale_attn_prefill(q, k, v, cu, longest, D ** -0.5)
        a8, scales = o.opscale_quantize_fp8(attn.view(T, HQ * D))
        y = o.opscale_linear_fp8(a8, scales, *self.wd[1], dtype=self.dtype)
        d["ctx"].copy_(kv)
        d["begin"].copy_(begin)
        return dict(cu=cu, slots=slots, kv=kv, h=h, h8=h8, hs=hs, raw=raw, q=q, k=k, v=v, attn=attn, a8=a8, scales=scales, y=y)


def check(half, r, dtype, T, decode):
    """T: the tokens that are there; the rest of a batch is padding."""
    import torch
    torch.cuda.synchronize()
    host = {n: t.cpu() for n, t in r.items()}
    for x, q8, s, out, (wc, ws) in (("h", "h8", "hs", "raw", half.w[0]), ("attn", "a8", "scales", "y", half.w[1])):
        a = f64(host[x]).reshape(host[x].shape[0], -1)[:T]
        values, scales = narrow.quantize_fp8(a)
        codes = host[q8].view(torch.uint8).numpy()[:T]
        assert np.array_equal(narrow.E4M3[codes], values)
        assert np.array_equal(f64(host[s])[:, :T], scales)
        want, off = reference(codes, scales.astype(np.float32), wc, ws, None, dtype)
        worst = (np.abs(f64(host[out])[:T] - want) / off).max()
        say(f"  {out}: {worst:.3f} of the bound")
        assert worst <= 1.0
    # the cache holds the tokens' rows
    at = host["slots"].numpy()[:T]
    kp, vp = narrow.unpack(half.kc.cpu().numpy()), narrow.unpack(half.vc.cpu().numpy())
    for pages, rows in ((kp, host["k"]), (vp, host["v"])):
        assert np.array_equal(pages[at // BS, at % BS], narrow.cached(f64(rows)[:T]))
    if decode:
        table, kv, q = half.d["table"].cpu().numpy(), host["kv"].numpy(), f64(host["q"])
        kw = dict(softcap=30.0, window=60)
        ref, weighted = (step.attn_decode_mod(q, kp, p, table, kv, D ** -0.5, **kw) for p in (vp, np.abs(vp)))
        dot = D ** -0.5 * np.abs(q).sum(-1).max() * np.nanmax(np.abs(kp))
        near(f64(host["attn"]), ref, tolerance(ref, weighted, dtype, D, int(kv.max()), dot, 30.0, 0.0), "decode")
    return kp, vp


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompts_then_decode_in_a_graph(ops, dtype):
    import torch
    say(f"narrow step {dtype}")
    lens = [37, 0, 5, 80]
    B, T, pad = len(lens), sum(lens), 3
    half = Half(ops, [0] * B, 6, 2, dtype)
    r = half.run(cuda(gen(41, "x", (T + pad, H), dtype)), i32(lens), max(lens), False)
    kp, vp = check(half, r, dtype, T, False)
    table = half.d["table"].cpu().numpy()
    assert np.array_equal(r["slots"].cpu().numpy(), np.r_[slots_of(table, lens, BS), [-1] * pad])

    # what a later chunk of the prompts would read, from key 3 on
    first = [3, 0, 3, 3]
    cu = np.r_[0, np.cumsum(np.maximum(np.array(lens) - first, 0))]
    k, v = ops.opscale_kv_read_fp4(half.kc, half.vc, half.d["table"], i32(cu), int(cu[-1]) + 2, i32(first), dtype=half.dtype)
    at = slots_of(table, lens, BS, first)
    for pages, got in ((kp, k), (vp, v)):
        assert np.array_equal(f64(got.cpu())[:cu[-1]], pages[at // BS, at % BS])

    # decode: one token a sequence (the empty one starts), the step in a graph
    x, one = cuda(gen(42, "x", (B, H), dtype)), i32([1] * B)
    half.run(x, one, 96, True)
    state = [*half.d.values(), half.kc, half.vc]
    before = [t.clone() for t in state]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = half.run(x, one, 96, True)
    for i in range(4):
        x.copy_(gen(43 + i, "x", (B, H), dtype))
        eager = half.run(x, one, 96, True)
        torch.cuda.synchronize()
        after = [t.clone() for t in state]
        for t, b in zip(state, before):
            t.copy_(b)
        g.replay()
        torch.cuda.synchronize()
        for n in out:
            assert torch.equal(out[n].view(torch.uint8), eager[n].view(torch.uint8)), f"step {i}: {n}"
        for t, a in zip(state, after):
            assert torch.equal(t, a), f"step {i}"
        check(half, out, dtype, B, True)
        before = after
    assert half.d["ctx"].tolist() == [n + 5 for n in lens]
