"""GPU attention with score modifiers, element by element within the bounds that
attn_error derives (their own checks: test_attn_error.py)."""
import math

import numpy as np
import pytest

from attn_error import row
from oracle import step
from parity_util import cuda, f64, gen, say
from test_gpu_attn_mods import check_decode, i32, on_gpu, ops, paged, slopes_of  # noqa: F401

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


# ---------------------------------------------------------------- prefill ---
def _prefill(ops, x, lens, Hq, Hkv, D, scale, kw, causal=True):
    """The result for packed x [T, (Hq + 2 Hkv) * D], in float64."""
    import torch
    dev = cuda(x)
    q, k, v = (dev[:, a * D:b * D].unflatten(1, (-1, D)) for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
    cu = np.r_[0, np.cumsum(lens)]
    out = ops.opscale_attn_prefill_mod(q, k, v, i32(cu), max(lens), scale, causal, **on_gpu(kw))
    torch.cuda.synchronize()
    return f64(out.cpu())


@pytest.mark.parametrize("name", RULES)
@pytest.mark.parametrize("D", [64, 128])
def test_prefill_equal_rows(ops, name, D):
    """Where every key has the same V, each query that sees one gets it, bit by bit: its
    weights add up to one within the sums' rounding, far below a step of bf16."""
    lens, Hq, Hkv = [1, 2, 90, 300], 8, 2
    kw = _modifiers(name, Hq, len(lens))
    say(f"attn_prefill_mod bf16 D={D} {name}: equal rows of V")
    for std in (0.3, 1.5):
        x = gen(92, "q", (sum(lens), (Hq + 2 * Hkv) * D), "bf16", std)
        x[:, (Hq + Hkv) * D:] = gen(92, "v_cache", (1, Hkv * D), "bf16")
        got = _prefill(ops, x, lens, Hq, Hkv, D, 1 / math.sqrt(D), kw)
        v = f64(x)[:, (Hq + Hkv) * D:].reshape(-1, Hkv, D)
        np.testing.assert_array_equal(got, np.repeat(v, Hq // Hkv, axis=1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", RULES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_prefill(ops, dtype, name, D, causal):
    """bf16: the probabilities reach V in 8 bits, and their sum as they were rounded."""
    lens, Hq, Hkv, scale = [1, 2, 5, 40, 150, 70], 8, 2, 1 / math.sqrt(D)
    kw = _modifiers(name, Hq, len(lens))
    say(f"attn_prefill_mod {dtype} D={D} {name} causal={causal}")
    at = np.r_[0, np.cumsum(lens)]
    rng = np.random.default_rng(7)
    for std in (0.3, 1.5):
        x = gen(93, "q", (sum(lens), (Hq + 2 * Hkv) * D), dtype, std)
        got = _prefill(ops, x, lens, Hq, Hkv, D, scale, kw, causal)
        q, k, v = (f64(x)[:, a * D:b * D].reshape(-1, b - a, D) for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
        rows = [(b, i, int(rng.integers(Hq))) for b, n in enumerate(lens) for i in range(n)]
        want, bound = np.zeros((2, len(rows), D))
        for r, (b, i, h) in enumerate(rows):
            keys = _keys(kw, i, lens[b], causal)
            g = h // (Hq // Hkv)
            want[r], bound[r] = row(q[at[b] + i, h], k[at[b] + keys, g], v[at[b] + keys, g], i, keys, scale, kw["softcap"],
                                    float(kw["slopes"][h]) if "slopes" in kw else 0.0, dtype)
        within(np.stack([got[at[b] + i, h] for b, i, h in rows]), want, bound, f"std {std}")


@pytest.mark.parametrize("window", [1, 16, 200])
@pytest.mark.parametrize("Hq,Hkv", [(8, 8), (14, 2), (4, 1)])
def test_decode_long_prefix_behind_a_short_window(ops, window, Hq, Hkv):
    """Nearly all the keys lie in the prefix, few in the window."""
    ctx = [9000, 40, 7000]
    kw = dict(window=window, prefix_lens=np.array([8500, 40, 0]), softcap=30.0)
    check_decode(ops, "bf16", ctx, Hq, Hkv, 128, 16, kw)
    check_decode(ops, "f32", ctx[:1], Hq, Hkv, 64, 16, dict(kw, prefix_lens=kw["prefix_lens"][:1]))


# ------------------------------------------------------- caps and values at the ends ---
def _held(ops, dtype, x, lens, Hq, Hkv, D, scale, cap, what, every=1):
    """Prefill of packed x, and decode of each prompt's last token over the same keys, within
    the bounds of each element."""
    import torch
    q, k, v = (f64(x)[:, a * D:b * D].reshape(-1, b - a, D) for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
    at, kw = np.r_[0, np.cumsum(lens)], dict(softcap=cap, window=0)
    got = _prefill(ops, x, lens, Hq, Hkv, D, scale, kw)
    rows = [(b, i, h) for b, n in enumerate(lens) for i in range(n - 1, -1, -every) for h in range(Hq)]
    keep = [row(q[at[b] + i, h], k[at[b]:at[b] + i + 1, h * Hkv // Hq], v[at[b]:at[b] + i + 1, h * Hkv // Hq], i,
                np.arange(i + 1), scale, cap, dtype=dtype) for b, i, h in rows]
    want, bound = (np.stack(t) for t in zip(*keep))
    within(np.stack([got[at[b] + i, h] for b, i, h in rows]), want, bound, f"prefill, {what}")
    bs = 16
    pages = [-(-n // bs) for n in lens]
    first = np.r_[0, np.cumsum(pages)]
    table = np.array([[first[b] + min(j, p - 1) for j in range(max(pages))] for b, p in enumerate(pages)])
    shape = (int(first[-1]), bs, Hkv, D)
    kc, vc = (torch.zeros(shape, dtype=x.dtype) for _ in range(2))
    for b, n in enumerate(lens):
        for c, lo in ((kc, Hq), (vc, Hq + Hkv)):
            c.view(-1, Hkv, D)[first[b] * bs:first[b] * bs + n] = x[at[b]:at[b + 1], lo * D:(lo + Hkv) * D].unflatten(1, (-1, D))
    last = x[at[1:] - 1, :Hq * D].unflatten(1, (-1, D)).contiguous()
    got = ops.opscale_attn_decode_mod(cuda(last), cuda(kc), cuda(vc), i32(table), i32(lens), max(lens), scale, softcap=cap)
    torch.cuda.synchronize()
    pick = [r for r, (b, i, h) in enumerate(rows) if i == lens[b] - 1]
    within(f64(got.cpu()).reshape(-1, D), want[pick], bound[pick], f"decode, {what}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap", [1e-44, 1e-30, 1e-12, 1e-9, 1e-8, 1e5, 1e8, 1e12, 1e20, 3e38])
def test_caps_far_from_the_scores(ops, dtype, cap):
    """Some heads' queries are zeros, beside heads whose scores pass any small cap."""
    lens, Hq, Hkv = [70, 1, 130], 8, 2
    say(f"{dtype}: a cap of {cap}")
    for D, scale in ((128, 0.09), (64, 1e-3)):
        x = gen(94, "q", (sum(lens), (Hq + 2 * Hkv) * D), dtype, 1.5)
        x[:, :3 * D] = 0.0
        x[::2, 4 * D:5 * D] = 0.0
        _held(ops, dtype, x, lens, Hq, Hkv, D, scale, float(np.float32(cap)), f"D={D} scale={scale}", every=3)


def _apart(seed, lens, Hq, Hkv, D, far, std_v):
    """Packed bf16 rows whose keys lie along one direction, so that the raw scores of
    every query are about far[j] sqrt(D) for key j of its prompt; V of std_v."""
    x = gen(seed, "q", (sum(lens), (Hq + 2 * Hkv) * D), "bf16", 0.3).float()
    u = gen(seed, "k", (D,), "f32").sign()
    at = 0
    for n in lens:
        x[at:at + n, :Hq * D] += 3.0 * u.repeat(Hq)
        for j in range(n):
            x[at + j, Hq * D:(Hq + Hkv) * D] += far(j) / (3.0 * math.sqrt(D)) * u.repeat(Hkv)
        at += n
    x[:, (Hq + Hkv) * D:] = gen(seed, "v_cache", (sum(lens), Hkv * D), "f32") * std_v
    return x.bfloat16()


@pytest.mark.parametrize("cap", [5.0, 30.0, 50.0, 52.0, 80.0])
@pytest.mark.parametrize("D", [64, 128])
def test_large_and_small_values_behind_a_cap(ops, cap, D):
    """V near the ends of bf16, where scores lie near -cap first and near cap later, and
    where all of them lie near -cap."""
    lens, Hq, Hkv = [200, 1, 70, 300], 4, 2
    for name, far, std_v in (("rising, large V", lambda j: -400.0 if j < 80 else 400.0, 2.0 ** 100),
                             ("rising, V of 2^75", lambda j: -400.0 if j < 80 else 400.0, 2.0 ** 75),
                             ("rising in part, V of 2^100", lambda j: -200.0 + 2 * j, 2.0 ** 100),
                             ("low, small V", lambda j: -400.0, 2.0 ** -100),
                             ("low, V of 2^-50", lambda j: -400.0 + j % 7, 2.0 ** -50),
                             ("low, large V", lambda j: -400.0 + j % 5, 2.0 ** 100)):
        say(f"cap {cap} D={D}: {name}")
        x = _apart(95, lens, Hq, Hkv, D, far, std_v)
        _held(ops, "bf16", x, lens, Hq, Hkv, D, 1 / math.sqrt(D), cap, name, every=7)


@pytest.mark.parametrize("cap", [30.0, 50.0])
def test_large_values_beside_an_infinity(ops, cap):
    """An infinity that only the last query sees leaves the large finite results of the others."""
    lens, Hq, Hkv, D = [200], 4, 2, 128
    say(f"cap {cap}: large V beside an infinity")
    x = _apart(96, lens, Hq, Hkv, D, lambda j: -400.0 if j < 80 else 400.0, 2.0 ** 100)
    bad = x.clone()
    bad[199, (Hq + Hkv) * D + 5] = float("inf")
    kw = dict(softcap=cap, window=0)
    clean, got = (_prefill(ops, y, lens, Hq, Hkv, D, 1 / math.sqrt(D), kw) for y in (x, bad))
    assert np.isfinite(clean).all() and (got[199, :2, 5] == np.inf).all()
    clean[199, :2, 5] = np.inf
    np.testing.assert_array_equal(got, clean)


@pytest.mark.parametrize("lens", [[9, 3, 1, 16], [40, 12], [64], [300] + [4] * 60])
@pytest.mark.parametrize("name", ["cap", "bias", "prefix_window"])
def test_prefill_f32_short_prompts(ops, lens, name):
    """Prompts of a wave a token and head, alone and beside a long one."""
    Hq, Hkv, D, scale = 4, 2, 64, 0.125
    kw = _modifiers(name, Hq, len(lens))
    if "prefix_lens" in kw:
        kw["prefix_lens"] = np.minimum(kw["prefix_lens"], lens)
    say(f"attn_prefill_mod f32 {lens[:5]} {name}")
    at = np.r_[0, np.cumsum(lens)]
    x = gen(97, "q", (sum(lens), (Hq + 2 * Hkv) * D), "f32", 1.5)
    got = _prefill(ops, x, lens, Hq, Hkv, D, scale, kw)
    q, k, v = (f64(x)[:, a * D:b * D].reshape(-1, b - a, D) for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
    rows = [(b, i, h) for b, n in enumerate(lens) for i in range(n) for h in range(Hq)]
    want, bound = np.zeros((2, len(rows), D))
    for r, (b, i, h) in enumerate(rows):
        prefix = int(kw["prefix_lens"][b]) if "prefix_lens" in kw else 0
        keys = step.visible(i, lens[b], True, kw["window"], prefix, 0)
        want[r], bound[r] = row(q[at[b] + i, h], k[at[b] + keys, h // 2], v[at[b] + keys, h // 2], i, keys, scale,
                                kw["softcap"], float(kw["slopes"][h]) if "slopes" in kw else 0.0)
    within(np.stack([got[at[b] + i, h] for b, i, h in rows]), want, bound, "short prompts")
