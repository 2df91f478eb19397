"""A decoder layer with head norms, its own rotation and attention modifiers, run
as a serving loop runs it: a step's tables from the requests' lengths, the prompts
through the layer, then decode steps, eager and as one replayed graph.

Each stage is held to its 64-bit definition on the inputs that the GPU gave it:
projections, norms and rotation at the layer's tolerance, attention at that of its own
tests (its derivation stands there)."""
import math

import numpy as np
import pytest

import workloads as wl
from oracle import step
from parity_util import assert_close, cuda, f64, gen, say
from test_gpu_attn_mods import counted, near, slopes_of, tolerance

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    import torch
    assert torch.cuda.is_available()
    import paper_2608_13499_amd as ops
    ops.load()
    return ops


def i32(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def _weights(seed, shape, dtype, norms):
    H, Hq, Hkv, D, F = shape.hidden, shape.n_q_heads, shape.n_kv_heads, shape.head_dim, shape.ffn
    w = {"w_norm1": gen(seed, "w_norm", (H,), dtype, std=0.02, mean=1.0),
         "w_qkv": gen(seed, "w_qkv", ((Hq + 2 * Hkv) * D, H), dtype, std=0.06),
         "w_o": gen(seed, "w_o", (H, Hq * D), dtype, std=0.02),
         "w_norm2": gen(seed, "bias", (H,), dtype, std=0.02, mean=1.0),
         "w_gate_up": gen(seed, "w_gate_up", (2 * F, H), dtype, std=0.02),
         "w_down": gen(seed, "w_down", (H, F), dtype, std=0.02)}
    if norms:
        w["w_q_norm"] = gen(seed, "x", (D,), dtype, std=0.1, mean=1.0)
        w["w_k_norm"] = gen(seed, "v", (D,), dtype, std=0.1, mean=1.0)
    return w


class Loop:
    """What a serving loop holds: weights, cache, page tables and lengths."""

    def __init__(self, ops, dtype, shape, norms, scaling, rot, lens, bs, steps, sharing, seed=91):
        import torch
        self.ops, self.dtype, self.shape, self.bs, self.seed = ops, dtype, shape, bs, seed
        B, Hkv, D = len(lens), shape.n_kv_heads, shape.head_dim
        self.wh = _weights(seed, shape, dtype, norms)
        self.w = {n: cuda(t) for n, t in self.wh.items()}
        self.w["inv_freq"] = ops.opscale_rope_frequencies(rot, shape.rope_theta, scaling, 4.0, 1.0, 32.0, 4096)[0].cuda()
        self.freq = self.w["inv_freq"].cpu().numpy()
        self.cols = -(-(max(lens) + steps) // bs)
        nb = int(sum(-(-(n + steps) // bs) for n in lens)) + 3
        self.kc, self.vc = (cuda(gen(seed, t, (nb, bs, Hkv, D), dtype)) for t in ("k_cache", "v_cache"))
        self.free = i32(np.random.default_rng(seed).permutation(nb))
        self.begin = i32([0])
        self.ctx = i32([0] * B)
        self.table = torch.full((B, self.cols), -1, dtype=torch.int32, device="cuda")
        self.max_ctx = max(lens) + steps
        self.rules = {}
        if sharing:
            self.rules = {"slopes": torch.from_numpy(slopes_of(shape.n_q_heads)).cuda(),
                          "prefix_lens": i32([min(n, 3) for n in lens])}
        modded = sharing or shape.softcap or shape.window
        size = ops.opscale_attn_decode_mod_workspace_size if modded else ops.opscale_attn_decode_workspace_size
        self.ws = torch.empty(max(size(B, shape.n_q_heads, D, self.max_ctx), 16), dtype=torch.uint8, device="cuda")

    def tables(self, new, tokens):
        out = self.ops.opscale_block_tables(self.ctx, new, self.table, self.free, self.begin, self.bs, tokens)
        self.ctx.copy_(out[3])
        self.begin.copy_(out[4])
        return out

    def prefill(self, x, res, new, tokens, longest):
        from paper_2608_13499_amd.layer import prefill_layer
        cu, pos, slots, _, _ = self.tables(new, tokens)
        return prefill_layer(self.shape, self.w, x, res, pos, cu, longest, self.kc, self.vc, slots, rules=self.rules)

    def decode(self, x, res, one):
        from paper_2608_13499_amd.layer import decode_layer
        _, pos, slots, kv, _ = self.tables(one, x.shape[0])
        return decode_layer(self.shape, self.w, x, res, pos, slots, self.kc, self.vc, self.table, kv, self.max_ctx,
                            self.ws, rules=self.rules)

    def check_heads(self, out, pos, what):
        """q, k and v of `out` from its h1."""
        s = self.shape
        Hq, Hkv, D = s.n_q_heads, s.n_kv_heads, s.head_dim
        ref = f64(out["h1"].cpu()) @ f64(self.wh["w_qkv"]).T
        got = f64(out["qkv"].cpu())
        T = len(got)
        ref, got = ref.reshape(T, -1, D), got.reshape(T, -1, D)
        for name, a, b, w in (("q", 0, Hq, "w_q_norm"), ("k", Hq, Hq + Hkv, "w_k_norm")):
            g = f64(self.wh[w]) if w in self.wh else None
            want = step.qk_norm_rope(ref[:, a:b], g, s.head_eps, pos, self.freq, s.rope_interleaved,
                                     np.float32(s.rope_magnitude))
            assert_close(got[:, a:b], want, self.dtype, f"{what} {name}")
        assert_close(got[:, Hq + Hkv:], ref[:, Hq + Hkv:], self.dtype, f"{what} v")
        return got[:, :Hq], got[:, Hq:Hq + Hkv], got[:, Hq + Hkv:]

    def attention_args(self):
        kw = {n: t.cpu().numpy() for n, t in self.rules.items()}
        return dict(kw, softcap=self.shape.softcap, window=self.shape.window)

    def tolerance(self, ref, weighted, q, k, n):
        kw, s = self.attention_args(), self.shape
        scale = 1.0 / math.sqrt(s.head_dim)
        dot = scale * float((np.abs(q).max((0, 1)) * np.abs(k).reshape(-1, s.head_dim).max(0)).sum())
        return tolerance(ref, weighted, self.dtype, s.head_dim, n, dot, s.softcap, counted(kw, n))

    def close_rest(self, out, what):
        assert_close(f64(out["o"].cpu()), f64(out["attn"].cpu()).reshape(len(out["o"]), -1) @ f64(self.wh["w_o"]).T,
                     self.dtype, f"{what} o")
        assert np.isfinite(f64(out["y"].cpu())).all()


CASES = {
    # a capped, windowed layer with head norms
    "cap_window": dict(dtype="bf16", kw=dict(softcap=20.0, window=40), norms=True, scaling="none", rot=128, sharing=False,
                       dims=(512, 8, 2, 128, 1024), lens=[200, 31, 97, 5, 64], bs=16),
    # a partial, interleaved, stretched rotation, slopes and a common prefix; seven query heads a KV head
    "bias_prefix": dict(dtype="bf16", kw=dict(rope_interleaved=True, rope_magnitude=1.1), norms=False, scaling="ramp",
                        rot=32, sharing=True, dims=(256, 14, 2, 64, 512), lens=[64, 130, 1], bs=4),
    "f32": dict(dtype="f32", kw=dict(softcap=5.0), norms=True, scaling="bands", rot=64, sharing=True,
                dims=(256, 6, 3, 64, 512), lens=[33, 70, 1], bs=16),
    # head norms alone, before the plain attention
    "plain_attention": dict(dtype="bf16", kw=dict(), norms=True, scaling="linear", rot=64, sharing=False,
                            dims=(256, 4, 4, 64, 512), lens=[64, 130], bs=1),
}


def _loop(ops, name, steps):
    from paper_2608_13499_amd.layer import LayerShape
    c = CASES[name]
    return c, Loop(ops, c["dtype"], LayerShape(*c["dims"], 1e-5, 10000.0, **c["kw"]), c["norms"], c["scaling"], c["rot"],
                   c["lens"], c["bs"], steps, c["sharing"])


@pytest.mark.parametrize("name,pad", [(n, 0) for n in CASES] + [("cap_window", 23), ("bias_prefix", 1), ("f32", 100)])
def test_prompts_then_steps(ops, name, pad):
    """pad: tokens past the last prompt's, as a step of a fixed size has them (NaN here)."""
    import torch
    c, loop = _loop(ops, name, steps=3)
    say(f"layer with rules: {name}, {pad} tokens of padding")
    s, lens, dtype = loop.shape, c["lens"], c["dtype"]
    T, B, scale = sum(lens), len(lens), 1.0 / math.sqrt(s.head_dim)
    cu = wl.cu_seqlens(np.asarray(lens))
    pos = np.concatenate([np.arange(n) for n in lens])
    x = gen(loop.seed, "x", (T, s.hidden), dtype)
    padded = torch.cat([x, torch.full((pad, s.hidden), float("nan"), dtype=x.dtype)])
    out = loop.prefill(cuda(padded), None, i32(lens), T + pad, max(lens))
    torch.cuda.synchronize()
    out = {n: t[:T] for n, t in out.items()}
    q, k, v = loop.check_heads(out, pos, "prefill")
    kw = loop.attention_args()
    ref, weighted = (step.attn_prefill_mod(q, k, t, cu, scale, True, **kw) for t in (v, np.abs(v)))
    near(f64(out["attn"].cpu()), ref, loop.tolerance(ref, weighted, q, k, max(lens)), "prefill attention")
    loop.close_rest(out, "prefill")

    one, ctx = i32([1] * B), np.asarray(lens)
    for n in range(3):
        ctx = ctx + 1
        xd, rd = (cuda(gen(loop.seed + 1 + n, t, (B, s.hidden), dtype)) for t in ("x", "attn_out"))
        out = loop.decode(xd, rd, one)
        torch.cuda.synchronize()
        assert loop.ctx.tolist() == ctx.tolist()
        q, k1, v1 = loop.check_heads(out, ctx - 1, f"step {n}")
        table, kc, vc = loop.table.cpu().numpy(), f64(loop.kc.cpu()), f64(loop.vc.cpu())
        at = table[np.arange(B), (ctx - 1) // loop.bs], (ctx - 1) % loop.bs
        assert np.array_equal(kc[at], k1) and np.array_equal(vc[at], v1), "the step's keys and values in the cache"
        used = [p for b in range(B) for p in table[b, :-(-ctx[b] // loop.bs)]]
        assert min(used) >= 0 and len(set(used)) == len(used), "a page of two requests"
        ref, weighted = (step.attn_decode_mod(q, kc, t, table, ctx, scale, **kw) for t in (vc, np.abs(vc)))
        near(f64(out["attn"].cpu()), ref, loop.tolerance(ref, weighted, q, kc, max(ctx)), f"step {n} attention")
        loop.close_rest(out, f"step {n}")
    # the prompts' keys and values have stayed in their pages
    for b, n in enumerate(lens):
        j = np.arange(n)
        assert np.array_equal(kc[table[b, j // loop.bs], j % loop.bs], k[cu[b]:cu[b + 1]])
        assert np.array_equal(vc[table[b, j // loop.bs], j % loop.bs], v[cu[b]:cu[b + 1]])


@pytest.mark.parametrize("name", CASES)
def test_steps_as_a_graph(ops, name):
    """A captured decode step, replayed as the lengths and page tables grow, against
    the eager loop on a cache of its own."""
    import torch
    steps = 4
    c, eager = _loop(ops, name, steps + 1)
    _, graph = _loop(ops, name, steps + 1)
    say(f"layer with rules as a graph: {name}")
    s, lens, dtype = eager.shape, c["lens"], c["dtype"]
    T, B = sum(lens), len(lens)
    x, one = cuda(gen(eager.seed, "x", (T, s.hidden), dtype)), i32([1] * B)
    for loop in (eager, graph):
        loop.prefill(x, None, i32(lens), T, max(lens))
    ins = [[cuda(gen(5 + n, t, (B, s.hidden), dtype)) for t in ("x", "attn_out")] for n in range(steps + 1)]
    xs, rs = (t.clone() for t in ins[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # the first step, and every kernel's first launch
        first = graph.decode(xs, rs.clone(), one)["y"].clone()
    torch.cuda.current_stream().wait_stream(side)
    want = [{n: t.clone() for n, t in eager.decode(a, b.clone(), one).items()} for a, b in ins]
    assert torch.equal(first, want[0]["y"])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = graph.decode(xs, rs, one)
    for n in range(1, steps + 1):
        xs.copy_(ins[n][0])
        rs.copy_(ins[n][1])
        g.replay()
        torch.cuda.synchronize()
        for key in ("qkv", "attn", "y", "residual"):
            assert torch.equal(got[key], want[n][key]), f"replay {n}: {key}"
        assert graph.ctx.tolist() == [m + n + 1 for m in lens]
    assert torch.equal(graph.table, eager.table)
    assert torch.equal(graph.kc, eager.kc) and torch.equal(graph.vc, eager.vc)


def test_two_loops_on_two_streams(ops):
    """Loops that run at once on streams of their own give what each gives alone."""
    import torch
    say("two loops on two streams")
    names, steps = ("cap_window", "bias_prefix", "f32"), 3

    def run(loop, c, stream, out):
        T, B = sum(c["lens"]), len(c["lens"])
        with torch.cuda.stream(stream):
            x = cuda(gen(7, "x", (T, loop.shape.hidden), c["dtype"]))
            out.append(loop.prefill(x, None, i32(c["lens"]), T, max(c["lens"]))["y"])
            yield
            for n in range(steps):
                xd, rd = (cuda(gen(8 + n, t, (B, loop.shape.hidden), c["dtype"])) for t in ("x", "attn_out"))
                out.append(loop.decode(xd, rd, i32([1] * B))["y"])
                yield

    alone, together = [], []
    for name in names:
        c, loop = _loop(ops, name, steps)
        out = []
        for _ in run(loop, c, torch.cuda.current_stream(), out):
            torch.cuda.synchronize()
        alone.append((out, loop))
    live = []
    for name in names:
        c, loop = _loop(ops, name, steps)
        out, stream = [], torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        together.append((out, loop))
        live.append(run(loop, c, stream, out))
    for _ in range(steps + 1):
        for it in live:
            next(it)
    torch.cuda.synchronize()
    for (a, la), (b, lb) in zip(alone, together):
        assert all(torch.equal(x, y) for x, y in zip(a, b)) and len(a) == len(b) == steps + 1
        assert torch.equal(la.kc, lb.kc) and torch.equal(la.vc, lb.vc) and torch.equal(la.table, lb.table)


def test_refuses_norms_without_frequencies(ops):
    import torch
    from paper_2608_13499_amd.layer import LayerShape, prefill_layer
    shape = LayerShape(256, 4, 4, 64, 512)
    w = {n: cuda(t) for n, t in _weights(1, shape, "bf16", True).items()}
    x = torch.zeros(4, 256, dtype=torch.bfloat16, device="cuda")
    cache = torch.zeros(1, 16, 4, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ops.OpscaleError, match="inv_freq"):
        prefill_layer(shape, w, x, None, i32(range(4)), i32([0, 4]), 4, cache, cache.clone(), i32(range(4)))
