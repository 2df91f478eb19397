"""GPU parity of the head norms with rotation and cache write, and of a step's
tables, against the 64-bit definitions in oracle.step.

Tolerances, by counting roundings (u = 2^-24, a half step of fp32):
  * fp32 heads: the sum of squares is 16 fused steps and up to 4 additions (20 u,
    halved by the root), the division, epsilon, root (2 u) and two products 6 u; sine and
    cosine 4 u of 1 each (the angle's rounding at pi is 2 u, the functions 1 u, the magnitude
    1 u), two products and an addition 3 u: below 32 u of the pair's length;
  * bf16: half a step of the result (2^-8 relative) beside those.
"""
import numpy as np
import pytest

import workloads as wl
from oracle import step
from parity_util import cuda, f64, gen, say, torch_dtype

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


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


# ----------------------------------------------------------- qk_norm_rope ---
def _heads_ok(got, ref, scale, dtype, what):
    """|got - ref| <= 32 u of the pair's length (bounded by the head's largest
    element), and half a bf16 step of the value."""
    got, ref = f64(got.cpu()), np.asarray(ref)
    tol = 32 * U * 1.5 * np.abs(scale).max(-1, keepdims=True) + (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0.0)
    bad = np.abs(got - ref) > tol + 1e-38
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.abs(got - ref).max():.3e}"


def _run_heads(ops, dtype, T, Hq, Hkv, D, rot, norm, inter, scaling="none", in_place=True, cache=0, maxpos=131072,
               seed=51, stream=None):
    import torch
    say(f"qk_norm_rope {dtype} T={T} Hq={Hq} Hkv={Hkv} D={D} rot={rot} norm={norm} inter={inter} {scaling} "
        f"in_place={in_place} cache={cache}")
    rng = np.random.default_rng([seed, T, D])
    W = (Hq + 2 * Hkv) * D
    qkv = gen(seed, "q", (T, W + 16), dtype)  # 16 more columns: a stride of its own
    cols = qkv[:, :W]
    q0, k0, v0 = (t.reshape(T, -1, D) for t in (cols[:, :Hq * D], cols[:, Hq * D:(Hq + Hkv) * D], cols[:, (Hq + Hkv) * D:]))
    pos = rng.integers(0, maxpos, T).astype(np.int32)
    pos[:1] = 0
    wq, wk = (gen(seed, tag, (D,), dtype, 0.3, 1.0) for tag in ("w_norm", "bias"))
    freq = mag = None
    kw = {}
    mag = 1.0
    if rot:
        kw["inv_freq"], mag = ops.opscale_rope_frequencies(rot, 10000.0, scaling, 4.0, 1.0, 32.0, 4096)
        freq = kw["inv_freq"].cpu().numpy()
        kw.update(positions=i32(pos), magnitude=mag)
    if norm:
        kw.update(q_weight=cuda(wq), k_weight=cuda(wk))
    dev = cuda(qkv)
    q, k, v = (dev[:, a:b].unflatten(1, (-1, D)) for a, b in ((0, Hq * D), (Hq * D, (Hq + Hkv) * D), ((Hq + Hkv) * D, W)))
    if cache:
        nb = T // cache + 2
        kc0, vc0 = gen(seed, "k_cache", (nb, cache, Hkv, D), dtype), gen(seed, "v_cache", (nb, cache, Hkv, D), dtype)
        slots = rng.permutation(nb * cache)[:T].astype(np.int64)
        if T > 3:
            slots[1], slots[2], slots[3] = -1, nb * cache, -2 ** 31  # padding: skipped
        kc, vc = cuda(kc0), cuda(vc0)
        kw.update(v=v, k_cache=kc, v_cache=vc, slot_mapping=i32(slots))
    if not in_place:
        out = torch.full((T, (Hq + Hkv) * D), 7.0, dtype=dev.dtype, device="cuda")
        kw.update(q_out=out[:, :Hq * D].unflatten(1, (-1, D)), k_out=out[:, Hq * D:].unflatten(1, (-1, D)))
    gq, gk = ops.opscale_qk_norm_rope(q, k, eps=1e-3, interleaved=inter, stream=stream, **kw)
    torch.cuda.synchronize()
    for got, x0, w, name in ((gq, q0, wq, "q"), (gk, k0, wk, "k")):
        x = f64(x0)
        ref = step.qk_norm_rope(x, f64(w) if norm else None, 1e-3, pos, freq, inter, np.float32(mag))
        normed = step.qk_norm_rope(x, f64(w) if norm else None, 1e-3, pos, None, inter)
        _heads_ok(got, ref, normed * mag, dtype, name)
    after = dev.cpu()
    if in_place:
        assert torch.equal(after[:, (Hq + Hkv) * D:], qkv[:, (Hq + Hkv) * D:]), "v or the columns after it were touched"
    else:
        assert torch.equal(after, qkv), "an input was touched"
    if cache:
        rk, rv = kc0.clone().view(-1, Hkv, D), vc0.clone().view(-1, Hkv, D)
        for t, s in enumerate(slots):
            if 0 <= s < nb * cache:
                rk[s], rv[s] = gk[t].cpu(), v0[t]
        assert torch.equal(kc.cpu().view(-1, Hkv, D), rk), "k cache"
        assert torch.equal(vc.cpu().view(-1, Hkv, D), rv), "v cache"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D,rot", [(128, 128), (128, 64), (128, 16), (64, 64), (64, 32), (256, 256), (256, 64), (96, 96),
                                   (96, 48), (80, 32), (32, 32), (32, 16), (144, 128), (240, 240)])
def test_qk_norm_rope_layouts(ops, dtype, inter, D, rot):
    _run_heads(ops, dtype, 5, 6, 2, D, rot, True, inter, cache=4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,Hq,Hkv", [(1, 1, 1), (1, 32, 8), (2, 71, 1), (7, 28, 4), (33, 64, 64), (1021, 3, 1),
                                      (1024, 5, 5), (1027, 8, 2), (2051, 12, 4),
                                      (4099, 2, 2), (8201, 2, 1)])
def test_qk_norm_rope_sizes(ops, dtype, T, Hq, Hkv):
    _run_heads(ops, dtype, T, Hq, Hkv, 64, 64, T % 2 == 1, False, "ramp", in_place=T % 3 == 0, cache=16)


@pytest.mark.parametrize("norm,rot,cache,in_place", [(True, 0, 0, True), (False, 128, 0, False), (False, 0, 8, False),
                                                     (True, 128, 0, False), (False, 0, 0, False), (True, 0, 8, True)])
def test_qk_norm_rope_steps(ops, norm, rot, cache, in_place):
    """Each step by itself and the pairs of them."""
    _run_heads(ops, "bf16", 19, 8, 2, 128, rot, norm, False, "bands", in_place, cache)


def test_qk_norm_rope_equals_rope_and_cache_write(ops):
    """The plain rotation and the cache write give what their own operators give,
    to a rounding; a row of zeros is normed to zeros."""
    import torch
    T, Hq, Hkv, D = 37, 8, 2, 128
    qkv = cuda(gen(52, "q", (T, (Hq + 2 * Hkv) * D), "bf16"))
    split = lambda x: (x[:, :Hq * D].unflatten(1, (-1, D)), x[:, Hq * D:(Hq + Hkv) * D].unflatten(1, (-1, D)),
                       x[:, (Hq + Hkv) * D:].unflatten(1, (-1, D)))
    pos, slots = i32(np.arange(T) * 211), i32(np.random.default_rng(0).permutation(64)[:T])
    a, b = qkv.clone(), qkv.clone()
    caches = [torch.zeros(4, 16, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    q, k, v = split(a)
    ops.opscale_rope(q, k, pos, 500000.0)
    ops.opscale_reshape_and_cache(k, v, caches[0], caches[1], slots)
    q, k, v = split(b)
    f, m = ops.opscale_rope_frequencies(D, 500000.0)
    ops.opscale_qk_norm_rope(q, k, pos, f, magnitude=m, v=v, k_cache=caches[2], v_cache=caches[3], slot_mapping=slots)
    torch.cuda.synchronize()
    # the frequencies agree to 1e-13: the fp32 angles to a step, the results to a bf16 step at its border
    d = (a.float() - b.float()).abs()
    assert bool((d <= 2.0 ** -7 * a.float().abs() + 1e-6).all())
    assert torch.equal(caches[1], caches[3])
    assert torch.equal(b[:, (Hq + Hkv) * D:], qkv[:, (Hq + Hkv) * D:])
    z = torch.zeros(2, 4, D, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(D, dtype=torch.bfloat16, device="cuda")
    y, _ = ops.opscale_qk_norm_rope(z, z.clone(), q_weight=w, k_weight=w)
    assert bool((y == 0).all())


def test_qk_norm_rope_streams_and_graph(ops):
    """On a stream of the caller's, and replayed from a graph between eager calls."""
    import torch
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    _run_heads(ops, "bf16", 65, 8, 2, 128, 128, True, False, cache=16, stream=s)
    T, H, D = 130, 8, 128
    x = cuda(gen(53, "q", (T, 2 * H, D), "bf16"))
    q, k = x[:, :H], x[:, H:]
    qo, ko = torch.empty(T, H, D, dtype=x.dtype, device="cuda"), torch.empty(T, H, D, dtype=x.dtype, device="cuda")
    f, m = ops.opscale_rope_frequencies(D, 10000.0, "ramp", 8.0, 1.0, 32.0, 4096)
    w = cuda(gen(53, "w_norm", (D,), "bf16", 0.1, 1.0))
    pos = i32(np.arange(T))
    call = lambda a, b: ops.opscale_qk_norm_rope(q, k, pos, f, w, w, magnitude=m, q_out=a, k_out=b)
    call(qo, ko)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(qo, ko)
    for i in range(3):
        x.copy_(gen(54 + i, "q", (T, 2 * H, D), "bf16"))
        pos.add_(i * 1000)
        qo.zero_(), ko.zero_()
        g.replay()
        torch.cuda.synchronize()
        eq, ek = call(torch.empty_like(qo), torch.empty_like(ko))
        torch.cuda.synchronize()
        assert torch.equal(qo, eq) and torch.equal(ko, ek), i


def test_qk_norm_rope_refuses_tensors(ops):
    import torch
    q = torch.zeros(4, 8, 128, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(4, 2, 128, dtype=torch.bfloat16, device="cuda")
    f, _ = ops.opscale_rope_frequencies(128, 1e4)
    pos = i32(np.arange(4))
    w = torch.ones(128, dtype=torch.bfloat16, device="cuda")
    kc = torch.zeros(2, 4, 2, 128, dtype=torch.bfloat16, device="cuda")
    good = dict(q=q, k=k, positions=pos, inv_freq=f)
    ops.opscale_qk_norm_rope(**good)
    for bad in (dict(q=q.half()), dict(q=q.cpu()), dict(k=k.float()), dict(k=k[:3]), dict(q=q.transpose(0, 1)),
                dict(positions=None), dict(positions=pos.long()), dict(positions=pos[:3]), dict(positions=pos.cpu()),
                dict(inv_freq=f.float()), dict(inv_freq=f.cpu()), dict(q_weight=w), dict(q_weight=w, k_weight=w[:64]),
                dict(q_weight=w.float(), k_weight=w), dict(k_cache=kc, v_cache=kc.clone(), v=k),
                dict(k_cache=kc, v=k, slot_mapping=pos), dict(k_cache=kc, v_cache=kc.float(), v=k, slot_mapping=pos),
                dict(k_cache=kc, v_cache=kc, v=k, slot_mapping=pos), dict(q_out=q[:3]), dict(k_out=q), dict(q_out=k)):
        with pytest.raises(ops.OpscaleError):
            ops.opscale_qk_norm_rope(**dict(good, **bad))
    torch.cuda.synchronize()
    assert not q.any() and not kc.any()


# ----------------------------------------------------------- block_tables ---
def _tables(ops, ctx, new, block, max_tokens, cols=None, short=0, begin=3, stream=None, seed=0):
    import torch
    ctx, new = np.asarray(ctx, np.int64), np.asarray(new, np.int64)
    B = len(ctx)
    say(f"block_tables B={B} tokens={new.clip(0).sum()} block={block} max_tokens={max_tokens} cols={cols} short={short}")
    rng = np.random.default_rng(seed)
    have = -(-ctx.clip(0) // block)
    want = -(-(ctx.clip(0) + new.clip(0)) // block) - have
    cols = int((have + want).max(initial=1)) + 1 if cols is None else cols
    ids = rng.permutation(int(have.sum() + want.sum()) + 8).astype(np.int32)
    table = np.full((B, cols), -7, np.int32)  # (left as they were)
    at = 0
    for b in range(B):
        n = min(int(have[b]), cols)
        table[b, :n] = ids[at:at + n]
        at += n
    free = ids[at:][:begin + int(want.sum()) - short]
    td = i32(table)
    out = ops.opscale_block_tables(i32(ctx), i32(new), td, i32(free), i32([begin]), block, max_tokens, stream=stream)
    torch.cuda.synchronize()
    ref = step.block_tables(ctx, new, table, free, begin, block, max_tokens)
    for got, want_, name in zip((*out, td), ref, ("cu_seqlens", "positions", "slots", "kv_lens", "free_next", "table")):
        np.testing.assert_array_equal(got.cpu().numpy().reshape(np.shape(want_)), want_, err_msg=name)
    return out, td


@pytest.mark.parametrize("block", [1, 4, 16, 256, 1024])
@pytest.mark.parametrize("ctx,new,max_tokens", [
    ([0], [1], 1), ([0], [0], 4), ([15], [1], 1), ([16], [1], 8), ([7], [300], 300), ([0, 0, 0], [0, 0, 0], 0),
    ([5, 0, 31, 16], [3, 17, 0, 1], 64), ([5, 0, 31, 16], [3, 17, 0, 1], 20), ([5, 0, 31, 16], [3, 17, 0, 1], 3),
    ([-3, 9], [4, -1], 9), ([100] * 5, [33] * 5, 150)])
def test_block_tables_small(ops, block, ctx, new, max_tokens):
    _tables(ops, ctx, new, block, max_tokens)


@pytest.mark.parametrize("B", [255, 256, 257, 512, 1000, 4099])
def test_block_tables_many_requests(ops, B):
    rng = np.random.default_rng(B)
    ctx = rng.integers(0, 900, B)
    _tables(ops, ctx, np.ones(B, np.int64), 16, B)                 # a decode step
    new = np.where(rng.random(B) < 0.2, 0, rng.integers(1, 60, B))
    total = int(new.sum())
    _tables(ops, ctx, new, 16, total + 77)                         # padded
    _tables(ops, ctx, new, 16, total // 2)                         # cut inside
    _tables(ops, ctx, new, 16, int(new[:256].sum()))               # cut at a group's border
    _tables(ops, ctx, new, 16, total, short=total // 32)           # the free list ends early


def test_block_tables_long_and_skewed(ops):
    _tables(ops, [0], [200_001], 16, 200_064)
    new = np.ones(700, np.int64)
    new[3] = 150_000
    _tables(ops, np.zeros(700), new, 64, int(new.sum()) + 5)


def test_block_tables_narrow_rows_and_bad_pages(ops):
    """Tokens past the row's pages, a free list that is empty or starts elsewhere,
    and page ids that are negative or too large for a slot."""
    import torch
    _tables(ops, [30, 0, 64, 70], [10, 100, 1, 3], 16, 120, cols=4)
    _tables(ops, [3, 0], [2, 9], 4, 16, short=4, begin=0)
    for begin in (-5, 2 ** 31 - 1):
        table = i32([[5, -1, -1]])
        out = ops.opscale_block_tables(i32([4]), i32([6]), table, i32([1, 2, 3]), i32([begin]), 4, 6)
        ref = step.block_tables([4], [6], [[5, -1, -1]], [1, 2, 3], begin, 4, 6)
        np.testing.assert_array_equal(out[2].cpu().numpy(), ref[2])
        assert int(out[4]) == min(ref[4], 2 ** 31 - 1) and table.cpu().tolist() == ref[5].tolist()
    table = i32([[-9, 2 ** 31 - 1]])
    out = ops.opscale_block_tables(i32([3]), i32([3]), table, torch.empty(0, dtype=torch.int32, device="cuda"), i32([0]), 4, 6)
    assert out[2].cpu().tolist() == [-1] * 6
    assert out[0].cpu().tolist() == [0, 3] and out[1].cpu().tolist() == [3, 4, 5, 0, 0, 0]


def test_block_tables_no_requests(ops):
    import torch
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    out = ops.opscale_block_tables(e, e, e.view(0, 4), i32([1]), i32([7]), 16, 5)
    assert [t.cpu().tolist() for t in out] == [[0], [0] * 5, [-1] * 5, [], [7]]


def test_block_tables_step_after_step_in_a_graph(ops):
    """A decode loop from one graph: lengths and the free list's place go round on
    the GPU; every step equals the definition's."""
    import torch
    B, block, cols = 37, 4, 12
    rng = np.random.default_rng(1)
    ctx = rng.integers(0, 20, B)
    new = rng.integers(0, 3, B)
    ids = rng.permutation(1000).astype(np.int32)
    table = np.full((B, cols), -1, np.int32)
    at = 0
    for b in range(B):
        n = -(-int(ctx[b]) // block)
        table[b, :n] = ids[at:at + n]
        at += n
    free = ids[at:]
    d = dict(ctx=i32(ctx), new=i32(new), table=i32(table), free=i32(free), begin=i32([0]))
    mt = 2 * B
    out = [torch.empty(n, dtype=torch.int32, device="cuda") for n in (B + 1, mt, mt, B, 1)]
    call = lambda: ops.opscale_block_tables(d["ctx"], d["new"], d["table"], d["free"], d["begin"], block, mt, out=out)
    call()
    torch.cuda.synchronize()
    d["table"].copy_(i32(table))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
        d["ctx"].copy_(out[3])
        d["begin"].copy_(out[4])
    rctx, rtable, rbegin = ctx, table, 0
    for i in range(6):
        g.replay()
        torch.cuda.synchronize()
        cu, pos, slots, kv, rbegin, rtable = step.block_tables(rctx, new, rtable, free, rbegin, block, mt)
        for got, ref in zip((*out, d["table"]), (cu, pos, slots, kv, [rbegin], rtable)):
            np.testing.assert_array_equal(got.cpu().numpy(), ref, err_msg=f"step {i}")
        rctx = kv


def test_block_tables_refuses_tensors(ops):
    e = dict(context_lens=i32([1, 2]), new_lens=i32([1, 1]), block_table=i32([[0, 1], [2, 3]]), free_blocks=i32([4]),
             free_begin=i32([0]), block_size=16, max_tokens=4)
    ops.opscale_block_tables(**e)
    for bad in (dict(context_lens=i32([1])), dict(new_lens=e["new_lens"].long()), dict(free_blocks=e["free_blocks"].cpu()),
                dict(free_begin=i32([0, 1])), dict(block_size=12), dict(block_table=i32([[0, 1, 2], [3, 4, 5]])[:, :2]),
                dict(out=(e["new_lens"],) * 5), dict(max_tokens=-1, out=None)):
        with pytest.raises((ops.OpscaleError, RuntimeError)):
            ops.opscale_block_tables(**dict(e, **bad))


# --------------------------------------------- timing and profiles of a step ---
def test_work_and_profiles(ops):
    """Timed calls and profiles count the work of the definition, in closed form."""
    import torch
    flush = torch.zeros(1 << 20, dtype=torch.float32, device="cuda")
    B, Hq, Hkv, D, bs, new, kept = 6, 8, 2, 64, 16, 40, 50
    ctx, fresh = i32([kept] * B), i32([new] * B)
    table, free, begin = i32(np.full((B, 8), -1)), i32(range(64)), i32([0])
    out, t = ops.opscale_block_tables(ctx, fresh, table, free, begin, bs, B * new, timed=True)
    pages = B * (-(-(kept + new) // bs) - -(-kept // bs))
    assert t.alg_flops == 0 and t.alg_bytes == 4 * (4 * B + 3 + 2 * B * new + 2 * pages)
    p = ops.opscale_op_profile(ops.desc_block_tables(ctx, fresh, table, free, begin, bs, B * new, out), 1, 3, flush)
    assert (p.alg_flops, p.alg_bytes) == (0, t.alg_bytes) and p.us_median > 0
    assert int(out[4]) == pages

    # a prompt of its own for each: the tokens, norms, a rotation of half the head, the cache
    T = B * new
    pos, slots, cu = i32(list(range(new)) * B), i32(np.random.default_rng(0).permutation(T)), i32(np.arange(B + 1) * new)
    g = torch.Generator(device="cuda").manual_seed(5)
    q, k, v = (torch.randn(T, h, D, device="cuda", generator=g).bfloat16() for h in (Hq, Hkv, Hkv))
    kc, vc = (torch.zeros(T // bs, bs, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    w, (f, m) = torch.ones(D, dtype=torch.bfloat16, device="cuda"), ops.opscale_rope_frequencies(D // 2, 1e4)
    kw = dict(positions=pos, inv_freq=f, q_weight=w, k_weight=w, magnitude=m, v=v, k_cache=kc, v_cache=vc,
              slot_mapping=slots, q_out=torch.empty_like(q), k_out=torch.empty_like(k))
    (q1, k1), t = ops.opscale_qk_norm_rope(q, k, timed=True, **kw)
    heads = T * (Hq + Hkv)
    weights = 2 * 2 * D + 4 * (D // 2)  # two gains, and D / 4 frequencies of 8 bytes
    assert t.alg_flops == 4 * heads * D + 3 * heads * (D // 2)
    assert t.alg_bytes == 2 * (2 * heads * D + 3 * T * Hkv * D) + weights + 8 * T
    p = ops.opscale_op_profile(ops.desc_qk_norm_rope(q, k, **kw), 1, 3, flush)
    assert (p.alg_flops, p.alg_bytes) == (t.alg_flops, t.alg_bytes)
    assert (p.weight_bytes, p.io_bytes) == (weights, 2 * (heads + T * Hkv) * D)

    # prefill: a window of 10, the first 4 keys seen by all
    seen = sum(len(step.visible(i, new, True, 10, 4, 0)) for i in range(new))
    rules = dict(softcap=5.0, window=10, prefix_lens=i32([4] * B), doc_starts=i32([0] * T),
                 slopes=torch.ones(Hq, device="cuda"))
    o, t = ops.opscale_attn_prefill_mod(q1, k1, v, cu, new, 0.1, True, timed=True, **rules)
    assert t.alg_flops == 4 * D * Hq * B * seen
    p = ops.opscale_op_profile(ops.desc_attn_prefill_mod(q1, k1, v, torch.empty_like(o), cu, new, 0.1, True, **rules), 1,
                               3, flush)
    assert (p.alg_flops, p.alg_bytes) == (t.alg_flops, t.alg_bytes) and p.us_median > 0

    # decode: the same window and prefix over 40 keys
    tab, lens = i32(np.arange(18).reshape(B, 3) % (T // bs)), i32([new] * B)
    q1, rules["doc_starts"] = q1[:B].contiguous(), i32([0] * B)
    o, t = ops.opscale_attn_decode_mod(q1, kc, vc, tab, lens, new, 0.1, timed=True, **rules)
    assert t.alg_flops == 4 * D * Hq * B * 14
    o2 = torch.zeros_like(o)
    ws = torch.empty(ops.opscale_attn_decode_mod_workspace_size(B, Hq, D, new), dtype=torch.uint8, device="cuda")
    p = ops.opscale_op_profile(ops.desc_attn_decode_mod(q1, kc, vc, tab, lens, o2, new, 0.1, ws, **rules), 1, 3, flush)
    assert (p.alg_flops, p.alg_bytes) == (t.alg_flops, t.alg_bytes)
    assert torch.equal(o, o2)
