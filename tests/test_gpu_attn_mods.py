"""GPU parity of attention with score modifiers and masks, prefill and paged
decode, against the 64-bit definitions in oracle.step.

Tolerance.  With p the probabilities and A = sum p |v| / sum p of an output element
(the oracle's result with |v| for v):
  * bf16: a probability is rounded to bf16 for its product with V and not for the
    sum (2^-8 A), the result once (2^-8 |o|);
  * a score's error e changes its probability by the factor 1 +- e, the quotient by
    2 e A at most.  e counts, in u = 2^-24: the products' sum, D roundings of
    scale |q| . |k| at worst; the cap's 5.5e-7 (10 u) and 6 roundings of the capped
    score; the bias's 10 roundings of slope |i - j|, for the keys that count (a
    score 30 below its row's largest does not);
  * the sums over n keys, n u A each at worst.
"""
import math

import numpy as np
import pytest

import workloads as wl
from oracle import step
from parity_util import cuda, f64, gen, say

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


def f32(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()


def tolerance(ref, weighted, dtype, D, n, dot, cap, bias):
    """dot: the largest scale |q| . |k|; bias: the largest slope |i - j| that counts."""
    e = D * U * dot + (16 * U * min(cap, dot) if cap else 2 * U * dot) + 10 * U * bias
    tol = (2 * e + 2 * (n + 64) * U) * weighted
    return tol + (2.0 ** -8 * (weighted + np.abs(ref)) if dtype == "bf16" else 2 * U * np.abs(ref)) + 1e-30


def near(got, ref, tol, what):
    got = np.asarray(got, np.float64)
    assert np.isfinite(got).all(), f"{what}: not finite at {np.argwhere(~np.isfinite(got))[:4].tolist()}"
    r = np.abs(got - ref) / tol
    say(f"  {what}: {r.max():.3f} of the tolerance")
    assert r.max() <= 1.0, f"{what}: {r.max():.3f} of the tolerance at {np.unravel_index(r.argmax(), r.shape)}"


def slopes_of(H):
    return np.float32(2.0 ** (-8.0 * (1 + np.arange(H)) / H))


def rules(name, lens, Hq, seed=0):
    """Named modifiers of a batch: (arguments of the oracle, causal)."""
    rng = np.random.default_rng([seed, len(lens), int(np.sum(lens))])
    n = int(max(lens, default=1))
    starts = []
    for L in lens:
        s = np.zeros(L, np.int64)
        for c in sorted(rng.integers(0, L + 1, 3)):
            s[c:] = c
        if L > 4:
            s[L - 2:] = [L, 10 * L]  # padding: past the prompt
        starts.append(s)
    starts = np.concatenate(starts) if lens else np.zeros(0, np.int64)
    prefix = np.array([rng.integers(-1, L + 3) for L in lens])
    return {
        "none": (dict(), True),
        "cap": (dict(softcap=5.0), True),
        "cap_wide": (dict(softcap=1000.0), True),
        "bias": (dict(slopes=slopes_of(Hq)), True),
        "cap_bias": (dict(softcap=8.0, slopes=slopes_of(Hq)), True),
        "window1": (dict(window=1), True),
        "window": (dict(window=max(1, n // 5), softcap=5.0), True),
        "window_all": (dict(window=2 ** 31 - 1), True),
        "prefix": (dict(prefix_lens=prefix, softcap=5.0), True),
        "prefix_bias": (dict(prefix_lens=prefix, slopes=slopes_of(Hq)), True),
        "docs": (dict(doc_starts=starts, slopes=slopes_of(Hq)), True),
        "docs_prefix_window": (dict(doc_starts=starts, prefix_lens=prefix, window=max(1, n // 3), softcap=5.0,
                                    slopes=slopes_of(Hq)), True),
        "open": (dict(softcap=5.0), False),
        "open_window_bias": (dict(window=max(1, n // 6), slopes=slopes_of(Hq)), False),
        "open_docs_prefix": (dict(doc_starts=starts, prefix_lens=prefix), False),
    }[name]


RULES = ["none", "cap", "cap_wide", "bias", "cap_bias", "window1", "window", "window_all", "prefix", "prefix_bias",
         "docs", "docs_prefix_window", "open", "open_window_bias", "open_docs_prefix"]


def on_gpu(kw):
    d = dict(kw)
    for n in ("prefix_lens", "doc_starts"):
        if d.get(n) is not None:
            d[n] = i32(d[n])
    if d.get("slopes") is not None:
        d["slopes"] = f32(d["slopes"])
    return d


def heads(seed, T, Hq, Hkv, D, dtype, std=1.5):
    """A packed QKV tensor and its views."""
    qkv = gen(seed, "q", (T, (Hq + 2 * Hkv) * D), dtype, std)
    return qkv, [qkv[:, a * D:b * D].unflatten(1, (-1, D)) for a, b in
                 ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv))]


def counted(kw, n):
    """The largest slope * distance whose key can count against one 30 higher."""
    s = kw.get("slopes")
    return 0.0 if s is None else float(min(n * np.max(s), 30 + n * np.max(s)))


def check_prefill(ops, dtype, lens, Hq, Hkv, D, name, seed=61, rows=None, stream=None, std=1.5):
    import torch
    kw, causal = rules(name, lens, Hq, seed) if isinstance(name, str) else name
    say(f"attn_prefill_mod {dtype} lens={lens if len(lens) < 9 else len(lens)} Hq={Hq} Hkv={Hkv} D={D} {name}")
    T, cu = int(np.sum(lens)), wl.cu_seqlens(lens)
    qkv, views = heads(seed, T, Hq, Hkv, D, dtype, std)
    dev = cuda(qkv)
    q, k, v = (dev[:, a * D:b * D].unflatten(1, (-1, D)) for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
    scale = 1.0 / math.sqrt(D)
    out = torch.full((T, Hq, D), float("nan"), dtype=dev.dtype, device="cuda")
    ops.opscale_attn_prefill_mod(q, k, v, i32(cu), max(1, max(lens)), scale, causal, out=out, stream=stream, **on_gpu(kw))
    torch.cuda.synchronize()
    qh, kh, vh = (f64(t) for t in views)
    if rows is not None:
        rng = np.random.default_rng(seed)
        rows = [(int(t), int(h)) for t, h in zip(np.r_[0, T - 1, rng.integers(0, T, rows)], rng.integers(0, Hq, rows + 2))]
    ref, weighted = (step.attn_prefill_mod(qh, kh, x, cu, scale, causal, rows=rows, **kw) for x in (vh, np.abs(vh)))
    got = f64(out.cpu())
    got = got if rows is None else np.stack([got[t, h] for t, h in rows])
    n = max(lens)
    dot = scale * np.abs(qh).sum(-1).max() * np.abs(kh).max() if T else 0.0
    near(got, ref, tolerance(ref, weighted, dtype, D, n, dot, kw.get("softcap"), counted(kw, n)), str(name)[:40])
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", RULES)
def test_prefill_rules(ops, dtype, name):
    check_prefill(ops, dtype, [150, 0, 1, 67, 33], 8, 2, 128, name)
    check_prefill(ops, dtype, [97, 40], 6, 6, 64, name)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 193, 300])
def test_prefill_lengths(ops, dtype, L):
    for name in ("cap", "docs_prefix_window", "open_window_bias"):
        check_prefill(ops, dtype, [L], 4, 1, 64, name)


@pytest.mark.parametrize("Hq,Hkv,D", [(1, 1, 64), (3, 1, 128), (7, 1, 128), (28, 4, 64), (12, 6, 128), (16, 2, 64),
                                      (24, 2, 128), (71, 1, 64)])
def test_prefill_head_layouts(ops, Hq, Hkv, D):
    for name in ("cap", "docs_prefix_window"):
        check_prefill(ops, "bf16", [70, 5, 129], Hq, Hkv, D, name, rows=200)


@pytest.mark.parametrize("schedule", [0, 1])
@pytest.mark.parametrize("name", ["window", "prefix_bias", "docs_prefix_window", "open_docs_prefix"])
def test_prefill_schedules(ops, tune, schedule, name):
    tune(prefill_schedule=schedule)
    for lens in ([300, 1], [130, 130], [65], [5, 0, 700, 64, 31]):
        check_prefill(ops, "bf16", lens, 8, 2, 128, name, rows=300)


def test_prefill_many_prompts_and_long_ones(ops):
    rng = np.random.default_rng(5)
    check_prefill(ops, "bf16", [int(x) for x in rng.integers(0, 9, 1500)], 4, 2, 64, "cap_bias", rows=300)
    check_prefill(ops, "f32", [int(x) for x in rng.integers(0, 40, 300)], 4, 2, 64, "docs_prefix_window", rows=300)
    check_prefill(ops, "bf16", [5000, 2300], 8, 2, 128, "window", rows=60)
    check_prefill(ops, "bf16", [4099], 8, 8, 128, "docs_prefix_window", rows=60)
    check_prefill(ops, "f32", [2100], 4, 1, 128, "prefix_bias", rows=60)


@pytest.mark.parametrize("cap", [1e-3, 0.5, 30.0, 50.0, 1e6])
def test_prefill_caps(ops, cap):
    """Scores far past the cap, within half of it (the polynomial) and at its end."""
    for std in (0.3, 1.5, 4.0, 30.0):
        check_prefill(ops, "bf16", [200, 77], 4, 2, 64, (dict(softcap=cap), True), std=std, rows=200)


def test_prefill_without_modifiers_is_the_plain_operator(ops):
    import torch
    lens, Hq, Hkv, D = [333, 64, 1], 8, 2, 128
    x, views = heads(62, sum(lens), Hq, Hkv, D, "bf16")
    qkv = cuda(x)
    q, k, v = (qkv[:, a * D:b * D].unflatten(1, (-1, D)) for a, b in ((0, 8), (8, 10), (10, 12)))
    cu = wl.cu_seqlens(lens)
    qh, kh, vh = (f64(t) for t in views)
    for causal in (True, False):
        a = ops.opscale_attn_prefill(q, k, v, i32(cu), 333, 0.09, causal)
        b = ops.opscale_attn_prefill_mod(q, k, v, i32(cu), 333, 0.09, causal)
        torch.cuda.synchronize()
        # (the two may add the keys up in another order: each is held to the definition)
        ref, weighted = (step.attn_prefill_mod(qh, kh, t, cu, 0.09, causal) for t in (vh, np.abs(vh)))
        tol = tolerance(ref, weighted, "bf16", D, 333, 0.09 * np.abs(qh).sum(-1).max() * np.abs(kh).max(), None, 0.0)
        near(f64(a.cpu()), ref, tol, "plain")
        near(f64(b.cpu()), ref, tol, "without modifiers")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_prefill_masked_infinities_and_nan(ops, dtype, D):
    """K and V rows that hold infinities and NaN reach the queries that see them and
    no other."""
    import torch
    lens, Hq, Hkv = [300, 90], 4, 2
    T, cu = sum(lens), wl.cu_seqlens(lens)
    qkv, _ = heads(63, T, Hq, Hkv, D, dtype)
    starts = np.concatenate([np.r_[np.zeros(100), np.full(190, 100), np.full(10, 300)], np.r_[np.zeros(80), np.full(10, 90)]])
    bad = qkv.clone()
    kcol, vcol = slice(Hq * D, (Hq + Hkv) * D), slice((Hq + Hkv) * D, None)
    rng = np.random.default_rng(0)
    for t in (*range(290, 300), *range(380, 390)):  # the padding: seen by none
        bad[t, kcol] = float(rng.choice([np.inf, -np.inf, np.nan]))
        bad[t, vcol] = float(rng.choice([np.inf, -np.inf, np.nan]))
    bad[120, (Hq + Hkv) * D + 3] = float("inf")   # seen from 120 on in the document at 100 (KV head 0)
    bad[130, (Hq + Hkv) * D + 3] = float("-inf")
    bad[200, (Hq + Hkv) * D + 7] = float("nan")
    dev = cuda(bad)
    q, k, v = (dev[:, a * D:b * D].unflatten(1, (-1, D)) for a, b in ((0, 4), (4, 6), (6, 8)))
    for extra in (dict(), dict(softcap=9.0), dict(slopes=slopes_of(Hq)), dict(softcap=9.0, slopes=slopes_of(Hq))):
        say(f"masked infinities {dtype} D={D} {list(extra)}")
        kw = dict(extra, doc_starts=starts)
        got = ops.opscale_attn_prefill_mod(q, k, v, i32(cu), 300, 0.1, True, **on_gpu(kw))
        torch.cuda.synchronize()
        got = f64(got.cpu())
        assert (got[290:300] == 0).all() and (got[380:] == 0).all()
        head0 = got[:, :2]
        assert (head0[120:130, :, 3] == np.inf).all() and not np.isfinite(head0[130:290, :, 3]).any()
        assert np.isnan(head0[200:290, :, 7]).all()
        hit = np.zeros(got.shape, bool)
        hit[120:290, :2, 3] = hit[200:290, :2, 7] = True
        qh, kh, vh = (f64(t) for t in (qkv[:, :4 * D].unflatten(1, (-1, D)), qkv[:, kcol].unflatten(1, (-1, D)),
                                       qkv[:, vcol].unflatten(1, (-1, D))))
        ref, weighted = (step.attn_prefill_mod(qh, kh, x, cu, 0.1, True, **kw) for x in (vh, np.abs(vh)))
        dot = 0.1 * np.abs(qh).sum(-1).max() * np.abs(kh).max()
        tol = tolerance(ref, weighted, dtype, D, 300, dot, extra.get("softcap"), counted(extra, 300))
        near(np.where(hit, ref, got), ref, tol, "the others")


@pytest.mark.parametrize("schedule", [0, 1])
@pytest.mark.parametrize("name,D", [("window", 128), ("docs", 64), ("docs_prefix_window", 128), ("open_window_bias", 64),
                                    ("cap", 64)])
def test_prefill_special_values_stay_with_their_queries(ops, tune, schedule, name, D):
    """An infinity and a NaN in V, in several prompts and tiles: the queries that see them get
    them in those columns, every other element what it is with zeros in their place."""
    import torch
    tune(prefill_schedule=schedule)
    lens, Hq, Hkv = [150, 1, 333, 64, 20], 4, 2
    say(f"attn_prefill_mod: special values, {name} D={D} schedule={schedule}")
    kw, causal = rules(name, lens, Hq)
    cu, T = wl.cu_seqlens(lens), sum(lens)
    x = gen(68, "q", (T, (Hq + 2 * Hkv) * D), "bf16", 1.5)
    at = [(70, 0, 3, float("inf")), (149, 1, 0, float("nan")), (151, 0, D - 1, float("-inf")), (151 + 63, 1, 5, float("nan")),
          (151 + 200, 0, 17, float("inf")), (151 + 332, 1, 40, float("nan")), (T - 84, 0, 9, float("-inf"))]

    def run(values):
        y = x.clone()
        for t, g, d, val in values:
            y[t, (Hq + Hkv + g) * D + d] = val
        dev = cuda(y)
        q, k, w = (dev[:, a * D:b * D].unflatten(1, (-1, D)) for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
        out = ops.opscale_attn_prefill_mod(q, k, w, i32(cu), max(lens), 1 / math.sqrt(D), causal, **on_gpu(kw))
        torch.cuda.synchronize()
        return f64(out.cpu())

    clean, got = run([(t, g, d, 0.0) for t, g, d, _ in at]), run(at)
    want = clean.copy()
    for t, g, d, val in at:
        b = int(np.searchsorted(cu, t, side="right")) - 1
        for i in range(lens[b]):
            row = int(cu[b]) + i
            prefix = 0 if kw.get("prefix_lens") is None else int(kw["prefix_lens"][b])
            start = 0 if kw.get("doc_starts") is None else int(kw["doc_starts"][row])
            if t - cu[b] in step.visible(i, lens[b], causal, kw.get("window", 0), prefix, start):
                want[row, g * (Hq // Hkv):(g + 1) * (Hq // Hkv), d] = val
    assert np.isfinite(clean).all() and not np.isfinite(want).all()
    np.testing.assert_array_equal(got, want)


def test_prefill_offsets_past_32_bits(ops):
    """Token rows 2^17 elements apart: 5 GB from the first to the last."""
    import torch
    T, Hq, Hkv, D, stride = 20000, 4, 2, 64, 1 << 17
    say("attn_prefill_mod: rows 2^17 elements apart")
    buf = torch.zeros((T - 1) * stride + (Hq + 2 * Hkv) * D, dtype=torch.bfloat16, device="cuda")
    rows = buf.as_strided((T, (Hq + 2 * Hkv) * D), (stride, 1))
    g = torch.Generator(device="cuda").manual_seed(3)
    rows.copy_(torch.empty(rows.shape, dtype=torch.float32, device="cuda").normal_(0, 1.5, generator=g))
    lens = [100] * 200
    cu = wl.cu_seqlens(lens)
    q, k, v = (rows[:, a * D:b * D].unflatten(1, (-1, D)) for a, b in ((0, 4), (4, 6), (6, 8)))
    out = ops.opscale_attn_prefill_mod(q, k, v, i32(cu), 100, 0.125, True, softcap=6.0, window=70)
    dense = [t.contiguous() for t in (q, k, v)]
    near_out = ops.opscale_attn_prefill_mod(*dense, i32(cu), 100, 0.125, True, softcap=6.0, window=70)
    torch.cuda.synchronize()
    assert torch.equal(out, near_out)
    pick = [(T - 1, 3), (T - 50, 0), (0, 1), (T // 2, 2)]
    ref = step.attn_prefill_mod(*(f64(t.cpu()) for t in dense), cu, 0.125, True, softcap=6.0, window=70, rows=pick)
    got = f64(out.cpu())
    for (t, h), r in zip(pick, ref):
        assert np.abs(got[t, h] - r).max() <= 2.0 ** -6 * np.abs(r).max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefill_prompts_past_one_grid(ops, dtype):
    """More prompts than a launch has workgroups, nearly all of them empty."""
    import torch
    B, D = (1 << 24) + 300, 64
    say(f"attn_prefill_mod {dtype}: {B} prompts")
    lens = np.zeros(B, np.int64)
    at = [0, 1, 5000, (1 << 24) - 2, (1 << 24) - 1, 1 << 24, B - 1]
    lens[at] = [3, 40, 1, 33, 65, 70, 7]
    cu, T = wl.cu_seqlens(lens), int(lens.sum())
    x = gen(63, "q", (T, 3 * D), dtype, 1.5)
    q, k, v = (cuda(x)[:, i * D:(i + 1) * D].unflatten(1, (1, D)) for i in range(3))
    prefix = np.zeros(B, np.int64)
    prefix[at] = [2, 0, 1, 20, 64, 1, 7]
    kw = dict(softcap=5.0, window=9)
    out = ops.opscale_attn_prefill_mod(q, k, v, i32(cu), 70, 0.125, True, prefix_lens=i32(prefix), **kw)
    torch.cuda.synchronize()
    few = wl.cu_seqlens(lens[at])
    qh, kh, vh = (f64(x)[:, i * D:(i + 1) * D].reshape(T, 1, D) for i in range(3))
    kw["prefix_lens"] = prefix[at]
    ref, weighted = (step.attn_prefill_mod(qh, kh, t, few, 0.125, True, **kw) for t in (vh, np.abs(vh)))
    dot = 0.125 * np.abs(qh).sum(-1).max() * np.abs(kh).max()
    near(f64(out.cpu()), ref, tolerance(ref, weighted, dtype, D, 70, dot, 5.0, 0.0), "prompts past one grid")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,pad", [([3, 1, 9], 5), ([3, 0], 60), ([70, 33], 200), ([300, 2, 40], 1), ([0, 0], 20)])
def test_prefill_padded_batch(ops, dtype, lens, pad):
    """Tokens past the last prompt: NaN there, in documents and in o, reach and lose nothing."""
    import torch
    Hq, Hkv, D, n = 4, 2, 64, sum(lens)
    say(f"attn_prefill_mod {dtype}: {lens} and {pad} tokens of padding")
    x = gen(67, "q", (n + pad, (Hq + 2 * Hkv) * D), dtype, 1.5)
    x[n:] = float("nan")
    dev = cuda(x)
    q, k, v = (dev[:, a * D:b * D].unflatten(1, (-1, D)) for a, b in ((0, 4), (4, 6), (6, 8)))
    starts = np.zeros(n + pad, np.int64)
    kw = dict(softcap=5.0, slopes=slopes_of(Hq), doc_starts=starts)
    for causal in (True, False):
        out = torch.full((n + pad, Hq, D), 7.0, dtype=dev.dtype, device="cuda")
        ops.opscale_attn_prefill_mod(q, k, v, i32(wl.cu_seqlens(lens)), max(1, max(lens)), 0.125, causal, out=out, **on_gpu(kw))
        torch.cuda.synchronize()
        assert bool((out[n:] == 7.0).all())
        if n == 0:
            continue
        qh, kh, vh = (f64(x[:n])[:, a * D:b * D].reshape(n, -1, D) for a, b in ((0, 4), (4, 6), (6, 8)))
        ref, weighted = (step.attn_prefill_mod(qh, kh, t, wl.cu_seqlens(lens), 0.125, causal, **kw) for t in (vh, np.abs(vh)))
        dot = 0.125 * np.abs(qh).sum(-1).max() * np.abs(kh).max()
        near(f64(out[:n].cpu()), ref, tolerance(ref, weighted, dtype, D, max(lens), dot, 5.0, counted(kw, max(lens))),
             f"padded, causal {causal}")


def test_prefill_streams_and_graph(ops):
    import torch
    lens, Hq, Hkv, D = [200, 33, 64], 8, 2, 128
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    check_prefill(ops, "bf16", lens, Hq, Hkv, D, "docs_prefix_window", stream=s, rows=100)
    kw, causal = rules("docs_prefix_window", lens, Hq)
    d = on_gpu(kw)
    x = cuda(heads(64, sum(lens), Hq, Hkv, D, "bf16")[0])
    q, k, v = (x[:, a * D:b * D].unflatten(1, (-1, D)) for a, b in ((0, 8), (8, 10), (10, 12)))
    cu, out = i32(wl.cu_seqlens(lens)), torch.empty(sum(lens), Hq, D, dtype=x.dtype, device="cuda")
    call = lambda o: ops.opscale_attn_prefill_mod(q, k, v, cu, 200, 0.09, causal, out=o, **d)
    call(out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(out)
    for i in range(3):
        x.copy_(heads(65 + i, sum(lens), Hq, Hkv, D, "bf16")[0])
        d["prefix_lens"].fill_(10 * i)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, call(torch.empty_like(out))), i


def test_prefill_refuses_tensors(ops):
    import torch
    q = torch.zeros(8, 4, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(8, 2, 64, dtype=torch.bfloat16, device="cuda")
    good = dict(q=q, k=k, v=k.clone(), cu_seqlens=i32([0, 8]), max_seqlen=8, scale=0.1)
    ops.opscale_attn_prefill_mod(**good)
    for bad in (dict(q=q.half()), dict(k=k.float()), dict(v=k.cpu()), dict(cu_seqlens=i32([0, 8]).long()),
                dict(softcap=-1.0), dict(softcap=float("inf")), dict(softcap=float("nan")), dict(window=-1),
                dict(window=1 << 31), dict(slopes=f32([1, 2, 3])), dict(slopes=f32([1, 2, 3, 4]).double()),
                dict(prefix_lens=i32([1, 2])), dict(prefix_lens=i32([1]).long()), dict(doc_starts=i32([0] * 7)),
                dict(doc_starts=torch.zeros(8, dtype=torch.int32)), dict(out=q), dict(out=torch.zeros_like(q).float()),
                dict(v=k[:4]), dict(scale=0.0)):
        with pytest.raises(ops.OpscaleError):
            ops.opscale_attn_prefill_mod(**dict(good, **bad))


# ----------------------------------------------------------------- decode ---
def paged(seed, ctx, Hkv, D, bs, dtype, holes=False, std=1.5):
    ctx = np.asarray(ctx, np.int64)
    table, nb = wl.paged_cache_layout(np.maximum(ctx, 1), bs, wl.rng_for(seed, "block_table"), extra_blocks=3)
    kc, vc = gen(seed, "k_cache", (nb, bs, Hkv, D), dtype, std), gen(seed, "v_cache", (nb, bs, Hkv, D), dtype)
    if holes:
        flat = table.reshape(-1)
        flat[::7], flat[3::11] = -1, nb
    return table.astype(np.int32), kc, vc


def check_decode(ops, dtype, ctx, Hq, Hkv, D, bs, kw, seed=71, holes=False, stream=None, max_ctx=None, std=1.5):
    import torch
    say(f"attn_decode_mod {dtype} B={len(ctx)} max={max(ctx)} Hq={Hq} Hkv={Hkv} D={D} bs={bs} {sorted(kw)} holes={holes}")
    table, kc, vc = paged(seed, ctx, Hkv, D, bs, dtype, holes, std)
    B = len(ctx)
    x = gen(seed, "q", (B, (Hq + 4) * D), dtype, std)  # a stride of its own
    dev = cuda(x)
    q = dev[:, :Hq * D].unflatten(1, (-1, D))
    n = max(1, max(ctx))
    scale = 1.0 / math.sqrt(D)
    out = torch.full((B, Hq, D), float("nan"), dtype=dev.dtype, device="cuda")
    ops.opscale_attn_decode_mod(q, cuda(kc), cuda(vc), i32(table), i32(ctx), max_ctx or n, scale, out=out, stream=stream,
                                **on_gpu(kw))
    torch.cuda.synchronize()
    qh, kh, vh = f64(x)[:, :Hq * D].reshape(B, Hq, D), f64(kc), f64(vc)
    ref, weighted = (step.attn_decode_mod(qh, kh, v, table, ctx, scale, **kw) for v in (vh, np.abs(vh)))
    dot = scale * np.abs(qh).sum(-1).max() * np.abs(kh).max()
    near(f64(out.cpu()), ref, tolerance(ref, weighted, dtype, D, n, dot, kw.get("softcap"), counted(kw, n)), "decode")
    return out


def decode_rules(name, ctx, Hq):
    rng = np.random.default_rng(len(ctx))
    n = int(max(ctx))
    starts = np.array([rng.integers(-2, max(1, c) + 2) for c in ctx])
    prefix = np.array([rng.integers(-1, c + 3) for c in ctx])
    return {
        "none": dict(), "cap": dict(softcap=5.0), "bias": dict(slopes=slopes_of(Hq)), "window1": dict(window=1),
        "window": dict(window=max(1, n // 4), softcap=5.0), "window_all": dict(window=2 ** 31 - 1),
        "prefix_window": dict(prefix_lens=prefix, window=max(1, n // 5)),
        "docs": dict(doc_starts=starts, slopes=slopes_of(Hq)),
        "all": dict(doc_starts=starts, prefix_lens=prefix, window=max(1, n // 3), softcap=5.0, slopes=slopes_of(Hq)),
        "nothing": dict(doc_starts=np.full(len(ctx), n + 5)),
    }[name]


DECODE_RULES = ["none", "cap", "bias", "window1", "window", "window_all", "prefix_window", "docs", "all", "nothing"]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", DECODE_RULES)
def test_decode_rules(ops, dtype, name):
    for ctx, Hq, Hkv, D, bs in (([700, 1, 0, 33, 64, 129], 16, 8, 128, 16), ([515, 31, 97], 6, 2, 64, 4)):
        check_decode(ops, dtype, ctx, Hq, Hkv, D, bs, decode_rules(name, ctx, Hq))
        check_decode(ops, dtype, ctx, Hq, Hkv, D, bs, decode_rules(name, ctx, Hq), holes=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 511, 512, 513, 1025])
def test_decode_lengths(ops, dtype, n):
    for name in ("cap", "all"):
        check_decode(ops, dtype, [n], 8, 1, 128, 16, decode_rules(name, [n], 8))


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 1), (7, 1), (15, 1), (16, 1), (17, 1), (32, 2), (71, 1), (28, 4), (40, 8),
                                    (9, 3), (12, 12), (24, 12), (10, 5), (48, 16), (64, 2)])
@pytest.mark.parametrize("D", [64, 128])
def test_decode_head_layouts(ops, Hq, Hkv, D):
    ctx = [300, 5, 77]
    check_decode(ops, "bf16", ctx, Hq, Hkv, D, 16, decode_rules("all", ctx, Hq))
    check_decode(ops, "bf16", ctx, Hq, Hkv, D, 16, decode_rules("cap", ctx, Hq))


@pytest.mark.parametrize("bs", [1, 2, 64, 256, 1024])
def test_decode_block_sizes(ops, bs):
    ctx = [1100, 600, 3]
    check_decode(ops, "bf16", ctx, 8, 2, 128, bs, decode_rules("all", ctx, 8))
    check_decode(ops, "f32", ctx, 8, 2, 64, bs, decode_rules("prefix_window", ctx, 8))


@pytest.mark.parametrize("B", [1, 64, 511, 512, 513, 1300])
def test_decode_batches(ops, B):
    rng = np.random.default_rng(B)
    ctx = [int(x) for x in rng.integers(0, 200, B)]
    ctx[0] = 900
    check_decode(ops, "bf16", ctx, 4, 2, 64, 16, decode_rules("all", ctx, 4))
    check_decode(ops, "bf16", ctx, 4, 2, 64, 16, decode_rules("prefix_window", ctx, 4), max_ctx=16)


def test_decode_long(ops):
    ctx = [20000, 9000]
    check_decode(ops, "bf16", ctx, 8, 4, 128, 16, dict(window=4096, prefix_lens=np.array([100, 0]), softcap=30.0))
    check_decode(ops, "bf16", ctx, 8, 1, 64, 64, dict(slopes=slopes_of(8)))
    check_decode(ops, "f32", [5000], 4, 1, 128, 16, dict(softcap=30.0))


@pytest.mark.parametrize("cap", [1e-3, 0.5, 50.0, 1e6])
def test_decode_caps(ops, cap):
    for std in (0.3, 4.0, 20.0):
        check_decode(ops, "bf16", [300, 40], 8, 2, 128, 16, dict(softcap=cap), std=std)


@pytest.mark.parametrize("Hq,Hkv", [(8, 8), (12, 3), (6, 6), (24, 12), (20, 5)])
def test_decode_without_modifiers_is_the_plain_operator(ops, Hq, Hkv):
    """Also for numbers of KV heads that are no power of two."""
    import torch
    ctx = [700, 1, 0, 90]
    table, kc, vc = paged(72, ctx, Hkv, 128, 16, "bf16")
    q = cuda(gen(72, "q", (4, Hq, 128), "bf16"))
    args = (q, cuda(kc), cuda(vc), i32(table), i32(ctx), 700, 0.09)
    a, b = ops.opscale_attn_decode(*args), ops.opscale_attn_decode_mod(*args)
    torch.cuda.synchronize()
    # (the two split the keys differently: each is held to the definition)
    qh, kh = f64(q.cpu()), f64(kc)
    ref, weighted = (step.attn_decode_mod(qh, kh, v, table, ctx, 0.09) for v in (f64(vc), np.abs(f64(vc))))
    tol = tolerance(ref, weighted, "bf16", 128, 700, 0.09 * np.abs(qh).sum(-1).max() * np.abs(kh).max(), None, 0.0)
    near(f64(a.cpu()), ref, tol, "plain")
    near(f64(b.cpu()), ref, tol, "without modifiers")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_masked_infinities_and_nan(ops, dtype):
    """What lies in masked rows, in rows past the length and in pages that are not
    there reaches no output; a query's NaN reaches its own head only."""
    import torch
    ctx, Hq, Hkv, D, bs = [300, 90, 40], 8, 2, 128, 16
    kw = dict(window=50, prefix_lens=np.array([20, 5, 0]), softcap=9.0)
    table, kc, vc = paged(73, ctx, Hkv, D, bs, dtype)
    table[2, 1] = -1
    q0 = gen(73, "q", (3, Hq, D), dtype, 1.5)
    seen = np.zeros((kc.shape[0], bs), bool)
    for b, n in enumerate(ctx):
        for j in step.visible(n - 1, n, True, 50, int(kw["prefix_lens"][b]), 0):
            if table[b, j // bs] >= 0:
                seen[table[b, j // bs], j % bs] = True
    kb, vb = kc.clone(), vc.clone()
    rng = np.random.default_rng(0)
    for p, o in np.argwhere(~seen):
        kb[p, o] = float(rng.choice([np.inf, -np.inf, np.nan]))
        vb[p, o] = float(rng.choice([np.inf, -np.inf, np.nan]))
    q = q0.clone()
    q[1, 0] = float("nan")
    say(f"decode: masked infinities {dtype}")
    got = ops.opscale_attn_decode_mod(cuda(q), cuda(kb), cuda(vb), i32(table), i32(ctx), 300, 0.1, **on_gpu(kw))
    torch.cuda.synchronize()
    got = f64(got.cpu())
    assert np.isnan(got[1, 0]).all()
    ref, weighted = (step.attn_decode_mod(f64(q0), f64(kc), v, table, ctx, 0.1, **kw) for v in (f64(vc), np.abs(f64(vc))))
    got[1, 0] = ref[1, 0]
    dot = 0.1 * np.abs(f64(q0)).sum(-1).max() * np.abs(f64(kc)).max()
    near(got, ref, tolerance(ref, weighted, dtype, D, 300, dot, 9.0, 0.0), "the others")


def test_decode_cache_past_32_bits(ops):
    """A cache of more than 2^31 elements, its last pages used."""
    import torch
    nb, bs, Hkv, D, Hq = (1 << 31) // (16 * 8 * 128) + 64, 16, 8, 128, 16
    say("attn_decode_mod: a cache past 2^31 elements")
    kc = torch.zeros(nb, bs, Hkv, D, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    ctx = [1000, 600]
    table = np.stack([nb - 1 - np.arange(64), np.r_[nb // 2 + np.arange(38), np.zeros(26)]]).astype(np.int32)
    used = np.unique(table)
    small_k, small_v = (gen(74, t, (len(used), bs, Hkv, D), "bf16", 1.5) for t in ("k_cache", "v_cache"))
    at = torch.from_numpy(used).long().cuda()
    kc[at], vc[at] = cuda(small_k), cuda(small_v)
    q = gen(74, "q", (2, Hq, D), "bf16", 1.5)
    kw = dict(softcap=20.0, window=700)
    got = ops.opscale_attn_decode_mod(cuda(q), kc, vc, i32(table), i32(ctx), 1000, 0.08, **on_gpu(kw))
    ref = ops.opscale_attn_decode_mod(cuda(q), cuda(small_k), cuda(small_v), i32(np.searchsorted(used, table)), i32(ctx),
                                      1000, 0.08, **on_gpu(kw))
    torch.cuda.synchronize()
    assert torch.equal(got, ref) and bool(got.abs().sum() > 0)


def test_decode_streams_workspaces_and_graph(ops):
    import torch
    ctx, Hq, Hkv, D = [300, 64, 5, 0], 8, 2, 128
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    check_decode(ops, "bf16", ctx, Hq, Hkv, D, 16, decode_rules("all", ctx, Hq), stream=s)
    table, kc, vc = paged(75, ctx, Hkv, D, 16, "bf16")
    kc, vc, table, lens = cuda(kc), cuda(vc), i32(table), i32(ctx)
    q, out = cuda(gen(75, "q", (4, Hq, D), "bf16")), torch.empty(4, Hq, D, dtype=torch.bfloat16, device="cuda")
    d = on_gpu(decode_rules("all", ctx, Hq))
    ws = torch.full((ops.opscale_attn_decode_mod_workspace_size(4, Hq, D, 300),), 255, dtype=torch.uint8, device="cuda")
    call = lambda o, w=None: ops.opscale_attn_decode_mod(q, kc, vc, table, lens, 300, 0.09, workspace=w, out=o, **d)
    call(out, ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(out, ws)
    for i in range(4):
        q.copy_(gen(76 + i, "q", (4, Hq, D), "bf16"))
        lens.copy_(i32([300 - 90 * i, 64 - i, 5, i]))
        out.fill_(float("nan"))
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, call(torch.empty_like(out))), i


def test_decode_refuses_tensors(ops):
    import torch
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    kc = torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16, device="cuda")
    good = dict(q=q, k_cache=kc, v_cache=kc.clone(), block_table=i32([[0, 1], [2, 3]]), context_lens=i32([20, 3]),
                max_context_len=20, scale=0.1)
    ops.opscale_attn_decode_mod(**good)
    small = torch.zeros(16, dtype=torch.uint8, device="cuda")
    for bad in (dict(q=q.float()), dict(q=q.cpu()), dict(k_cache=kc.float()), dict(v_cache=kc[:3]),
                dict(block_table=i32([[0, 1]])), dict(block_table=i32([0, 1, 2, 3])), dict(context_lens=i32([1])),
                dict(context_lens=i32([1, 2]).long()), dict(workspace=small), dict(softcap=-1.0), dict(window=-3),
                dict(slopes=f32([1, 2])), dict(prefix_lens=i32([1])), dict(doc_starts=i32([1, 2, 3])), dict(out=q),
                dict(out=torch.zeros(2, 4, 32, dtype=q.dtype, device="cuda")), dict(max_context_len=0), dict(scale=-1.0)):
        with pytest.raises(ops.OpscaleError):
            ops.opscale_attn_decode_mod(**dict(good, **bad))
