"""GPU KV cache in 4 bits: rows written and read back bit by bit, and decode attention over
it against the 64-bit definition (oracle.narrow for the values that the cache holds,
oracle.step for attention).

The cache's values are exact in every product.  The tolerance is test_gpu_attn_mods' with
the errors that this kernel has: bf16 probabilities in two pieces (2^-16 A), the sum
unrounded; fp32 queries and probabilities in three pieces (2^-24 of them: one rounding more).
"""
import math

import numpy as np
import pytest

import workloads as wl
from attn_error import row as bounded_row
from oracle import narrow, step
from parity_util import cuda, f64, gen, say, torch_dtype
from test_gpu_attn_error import RULES, _keys, _modifiers, within
from test_gpu_attn_mods import (DECODE_RULES, U, counted, decode_rules, f32, i32, near, on_gpu, ops,  # noqa: F401
                                slopes_of)

pytestmark = pytest.mark.gpu


def u8(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


# --------------------------------------------------------------- write and read ---
def slots_of(table, lens, bs, first=None):
    return np.concatenate([[table[b, j // bs] * bs + j % bs for j in range(0 if first is None else first[b], n)]
                           for b, n in enumerate(lens)] + [[]]).astype(np.int64)


def spread_heads(seed, T, H, D, dtype):
    """Heads of many sizes, group by group."""
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(T, H, D)) * np.repeat(2.0 ** rng.integers(-7, 7, size=(T, H, D // 32)), 32, -1)
    import torch
    return torch.from_numpy(x).to(torch_dtype(dtype))


def read(ops, kc, vc, table, cu, T, first=None, **kw):
    import torch
    k, v = ops.opscale_kv_read_fp4(kc, vc, i32(table), i32(cu), T, None if first is None else i32(first), **kw)
    torch.cuda.synchronize()
    return k, v


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hkv,bs,lens", [(1, 16, [1]), (3, 16, [33, 0, 16, 5]), (8, 64, [70, 3]), (2, 1024, [9, 40])])
def test_write_and_read(ops, dtype, D, Hkv, bs, lens):
    """Every byte of the cache, not only what it reads as; bytes of other slots stay."""
    import torch
    say(f"kv fp4 {dtype} D={D} Hkv={Hkv} bs={bs} lens={lens}")
    table, nb = wl.paged_cache_layout(np.maximum(lens, 1), bs, wl.rng_for(5, "block_table"), extra_blocks=2)
    T = int(sum(lens))
    wide = torch.zeros(T + 3, 2 * Hkv + 1, D, dtype=torch_dtype(dtype), device="cuda")  # K, V and something else in a row
    x = spread_heads(6, T + 3, 2 * Hkv, D, dtype)
    wide[:, :2 * Hkv] = x.cuda()
    slots = slots_of(table, lens, bs)
    padded = np.r_[slots, -1, nb * bs, -7].astype(np.int64)  # padding: written nowhere
    rng = np.random.default_rng(1)
    kc, vc = (rng.integers(0, 256, size=(nb, Hkv, bs, D // 2 + D // 32)).astype(np.uint8) for _ in range(2))
    dk, dv = u8(kc), u8(vc)
    ops.opscale_kv_write_fp4(wide[:, :Hkv], wide[:, Hkv:2 * Hkv], dk, dv, i32(padded))
    torch.cuda.synchronize()
    for cache, dev, heads in ((kc, dk, x[:T, :Hkv]), (vc, dv, x[:T, Hkv:])):
        rows = narrow.pack(f64(heads)[:, None])  # a page of one row a token
        want = cache.reshape(nb, Hkv, -1)
        for t, s in enumerate(slots):
            p, r = divmod(int(s), bs)
            want[p, :, r * (D // 2):(r + 1) * (D // 2)] = rows[t].reshape(Hkv, -1)[:, :D // 2]
            want[p, :, bs * (D // 2) + r + bs * np.arange(D // 32)] = rows[t].reshape(Hkv, -1)[:, D // 2:].T
        assert np.array_equal(dev.cpu().numpy().reshape(nb, Hkv, -1), want)
    cu = np.r_[0, np.cumsum(lens)]
    k, v = read(ops, dk, dv, table, cu, T, dtype=torch_dtype(dtype))
    assert np.array_equal(f64(k.cpu()), narrow.cached(f64(x[:T, :Hkv])))
    assert np.array_equal(f64(v.cpu()), narrow.cached(f64(x[:T, Hkv:])))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_write_values(ops, dtype):
    """Ties, every value, groups next to where the scale doubles, zeros, the smallest and largest
    numbers, infinities and NaN."""
    import torch
    say(f"kv fp4 {dtype}: values")
    vals = np.r_[narrow.E2M1, [.25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -.75, -5, 0.1, 6.9, -3.2, 0, 7, 5.1]]
    groups = [vals, np.zeros(32), -vals]
    for e in (-140, -130, -126, -101, -100, -99, -20, 0, 60, 124, 125):
        for top in (6.0, 6.99, 7.0, 7.01, 7.9):
            groups.append(np.where(np.arange(32) == 30, top, vals * 0.5) * 2.0 ** e)
    for bad in (np.inf, -np.inf, np.nan):
        groups.append(np.where(np.arange(32) == 7, bad, vals))
    while len(groups) % 4:
        groups.append(vals)
    x = torch.from_numpy(np.clip(np.stack(groups), -3.3e38, 3.3e38)).to(torch_dtype(dtype)).view(-1, 1, 128)
    x[torch.from_numpy(~np.isfinite(np.stack(groups).reshape(-1, 1, 128)))] = float("nan")
    x.view(-1)[32 * (len(groups) - 6) + 7] = float("inf")
    T = x.shape[0]
    kc = torch.zeros(4, 1, 16, 68, dtype=torch.uint8, device="cuda")
    vc = torch.zeros_like(kc)
    ops.opscale_kv_write_fp4(x.cuda(), x.cuda(), kc, vc, i32(np.arange(T)))
    for out in ("bf16", "f32"):
        k, v = read(ops, kc, vc, [[0, 1, 2, 3]], [0, T], T, dtype=torch_dtype(out))
        want = narrow.cached(f64(x))
        assert np.array_equal(f64(k.cpu()), want, equal_nan=True) and torch.equal(k.view(torch.int16), v.view(torch.int16))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_read_ranges(ops, dtype):
    """From keys in the middle of pages, past the table, below zero, pages that are not there; rows past
    the last sequence and between the strided ones stay."""
    import torch
    say(f"kv_read_fp4 {dtype}: ranges")
    D, H, bs, nb = 128, 3, 16, 9
    rng = np.random.default_rng(3)
    kc, vc = (rng.integers(0, 256, size=(nb, H, bs, 68)).astype(np.uint8) for _ in range(2))
    for c in (kc, vc):
        c.reshape(nb, H, -1)[:, :, bs * 64:] %= 200  # no scale of infinities' size
    table = np.array([[0, 3, -1, 8], [nb, 1, 2, 7], [5, 5, 6, 4]], np.int32)
    first, cu = [10, 0, 50], [0, 54, 54 + 20, 54 + 20 + 30]
    T = cu[-1] + 4
    buf = torch.full((T, 2 * H + 1, D), 7.0, dtype=torch_dtype(dtype), device="cuda")
    read(ops, u8(kc), u8(vc), table, cu, T, first, k=buf[:, :H], v=buf[:, H:2 * H])
    got = f64(buf.cpu())
    assert (got[cu[-1]:] == 7).all() and (got[:, 2 * H] == 7).all()
    for c, at in ((kc, 0), (vc, H)):
        x = narrow.unpack(c)
        for b in range(3):
            for i in range(cu[b + 1] - cu[b]):
                j = first[b] + i
                page = table[b, j // bs] if j // bs < 4 else -1
                want = x[page, j % bs] if 0 <= page < nb else np.zeros((H, D))
                assert np.array_equal(got[cu[b] + i, at:at + H], want), (b, j)
    k, v = read(ops, u8(kc), u8(vc), table, [0, 5, 5, 5], 5, [-3, 0, 0], dtype=torch_dtype(dtype))
    want = narrow.unpack(kc)[0, :2]
    assert (f64(k.cpu())[:3] == 0).all() and np.array_equal(f64(k.cpu())[3:], want)


@pytest.mark.parametrize("B", [1, 2, 63, 700])
def test_read_batches(ops, B):
    say(f"kv_read_fp4: {B} sequences")
    rng = np.random.default_rng(B)
    lens = rng.integers(0, 40, size=B)
    lens[-1] = 0 if B == 2 else lens[-1]
    nb, H, bs = 60, 5, 16
    kc, vc = (rng.integers(0, 190, size=(nb, H, bs, 34)).astype(np.uint8) for _ in range(2))
    table = rng.integers(0, nb, size=(B, 3)).astype(np.int32)
    cu = np.r_[0, np.cumsum(lens)]
    T = int(cu[-1])
    k, v = read(ops, u8(kc), u8(vc), table, cu, T)
    rows = [(b, j) for b in range(B) for j in range(lens[b])]
    for c, got in ((kc, k), (vc, v)):
        x = narrow.unpack(c)
        want = np.stack([x[table[b, j // bs], j % bs] for b, j in rows]) if rows else np.zeros((0, H, 64))
        assert np.array_equal(f64(got.cpu()), want)


def test_write_and_read_past_32_bits(ops):
    """A cache of more than 2^32 bytes, its last slots written and read."""
    import torch
    H, bs, D = 64, 1024, 128
    nb = (1 << 32) // (H * bs * 68) + 2
    say("kv fp4: a cache past 2^32 bytes")
    kc = torch.empty(nb, H, bs, 68, dtype=torch.uint8, device="cuda")
    vc = torch.empty_like(kc)
    x = spread_heads(9, 40, 2 * H, D, "bf16")
    slots = np.r_[nb * bs - 1 - np.arange(20), (nb - 2) * bs + np.arange(20)]
    d = x.cuda()
    ops.opscale_kv_write_fp4(d[:, :H], d[:, H:], kc, vc, i32(slots))
    k, v = read(ops, kc, vc, [[nb - 1], [nb - 2]], [0, 20, 40], 40, [bs - 20, 0])
    order = np.r_[np.arange(20)[::-1], 20 + np.arange(20)]
    want = narrow.cached(f64(x))[order]
    assert np.array_equal(f64(k.cpu()), want[:, :H]) and np.array_equal(f64(v.cpu()), want[:, H:])


# ------------------------------------------------------------------ attention ---
def tolerance(ref, weighted, dtype, D, n, dot, cap, bias):
    e = (D + (2 if dtype == "f32" else 0)) * U * dot + (16 * U * min(cap, dot) if cap else 2 * U * dot) + 10 * U * bias
    tol = (2 * e + 2 * (n + 64) * U) * weighted
    return tol + (2.0 ** -16 * weighted + 2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 4 * U * np.abs(ref)) + 1e-30


def paged4(seed, ctx, Hkv, D, bs, holes=False, low=124, high=128):
    """(table, K bytes, V bytes): random codes, scales of 2^(low - 127) to 2^(high - 127); what no
    sequence has of the cache is full of NaN."""
    ctx = np.asarray(ctx, np.int64)
    table, nb = wl.paged_cache_layout(np.maximum(ctx, 1), bs, wl.rng_for(seed, "block_table"), extra_blocks=3)
    table = table.astype(np.int32)
    rng = np.random.default_rng([seed, nb, Hkv, D])
    live = np.zeros((nb, bs), bool)
    for b, n in enumerate(ctx):
        for j in range(n):
            live[table[b, j // bs], j % bs] = True
    caches = []
    for _ in range(2):
        flat = rng.integers(0, 256, size=(nb, Hkv, bs * (D // 2 + D // 32))).astype(np.uint8)
        e = rng.integers(low, high + 1, size=(nb, Hkv, D // 32, bs)).astype(np.uint8)
        flat[:, :, bs * D // 2:] = np.where(live[:, None, None], e, 255).reshape(nb, Hkv, -1)
        caches.append(flat.reshape(nb, Hkv, bs, D // 2 + D // 32))
    if holes:
        flat = table.reshape(-1)
        flat[::7], flat[3::11] = -1, nb
    return (table, *caches)


def check_decode(ops, dtype, ctx, Hq, Hkv, D, bs, kw, seed=81, holes=False, stream=None, max_ctx=None, std=1.5):
    import torch
    say(f"attn_decode_fp4 {dtype} B={len(ctx)} max={max(ctx)} Hq={Hq} Hkv={Hkv} D={D} bs={bs} {sorted(kw)} holes={holes}")
    table, kc, vc = paged4(seed, ctx, Hkv, D, bs, holes)
    B = len(ctx)
    x = gen(seed, "q", (B, (Hq + 4) * D), dtype, std)  # a stride of its own
    dev = cuda(x)
    q = dev[:, :Hq * D].unflatten(1, (-1, D))
    n, scale = max(1, max(ctx)), 1.0 / math.sqrt(D)
    out = torch.full((B, Hq, D), float("nan"), dtype=dev.dtype, device="cuda")
    ops.opscale_attn_decode_fp4(q, u8(kc), u8(vc), i32(table), i32(ctx), max_ctx or n, scale, out=out, stream=stream,
                                **on_gpu(kw))
    torch.cuda.synchronize()
    qh, kh, vh = f64(x)[:, :Hq * D].reshape(B, Hq, D), narrow.unpack(kc), narrow.unpack(vc)
    ref, weighted = (step.attn_decode_mod(qh, kh, v, table, ctx, scale, **kw) for v in (vh, np.abs(vh)))
    dot = scale * np.abs(qh).sum(-1).max() * np.nanmax(np.abs(kh))
    near(f64(out.cpu()), ref, tolerance(ref, weighted, dtype, D, n, dot, kw.get("softcap"), counted(kw, n)), "decode")
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", DECODE_RULES)
def test_decode_rules(ops, dtype, name):
    for ctx, Hq, Hkv, D, bs in (([700, 1, 0, 33, 64, 129], 16, 8, 128, 16), ([515, 31, 97], 6, 2, 64, 32)):
        check_decode(ops, dtype, ctx, Hq, Hkv, D, bs, decode_rules(name, ctx, Hq))
        check_decode(ops, dtype, ctx, Hq, Hkv, D, bs, decode_rules(name, ctx, Hq), holes=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 64, 65, 511, 512, 513, 1023, 1025, 2100])
def test_decode_lengths(ops, dtype, n):
    for name in ("cap", "all"):
        check_decode(ops, dtype, [n], 8, 1, 128, 16, decode_rules(name, [n], 8))
    check_decode(ops, dtype, [n, n], 4, 4, 64, 16, {})


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 1), (7, 1), (15, 1), (16, 1), (17, 1), (32, 2), (71, 1), (28, 4), (40, 8),
                                    (9, 3), (12, 12), (24, 12), (10, 5), (48, 16), (64, 2)])
@pytest.mark.parametrize("D", [64, 128])
def test_decode_head_layouts(ops, Hq, Hkv, D):
    ctx = [300, 5, 77]
    for dtype in ("bf16", "f32"):
        check_decode(ops, dtype, ctx, Hq, Hkv, D, 16, decode_rules("all", ctx, Hq))
    check_decode(ops, "bf16", ctx, Hq, Hkv, D, 16, {})


@pytest.mark.parametrize("bs", [16, 64, 256, 1024])
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
    """Windows of page ids one after the other, with and without a prefix."""
    ctx = [20000, 9000]
    check_decode(ops, "bf16", ctx, 8, 4, 128, 16, dict(window=4096, prefix_lens=np.array([1500, 0]), softcap=30.0))
    check_decode(ops, "bf16", ctx, 8, 1, 64, 64, dict(slopes=slopes_of(8)))
    check_decode(ops, "bf16", [30000], 8, 8, 128, 16, {}, max_ctx=64)
    check_decode(ops, "f32", [5000], 4, 1, 128, 16, dict(softcap=30.0))


@pytest.mark.parametrize("Hq,Hkv,D", [(4, 1, 128), (17, 1, 64), (6, 2, 128), (9, 3, 128), (8, 4, 64), (8, 8, 128), (24, 24, 128)])
@pytest.mark.parametrize("name", DECODE_RULES)
def test_decode_split(ops, name, Hq, Hkv, D):
    """Short sequences whose greatest length as told has them split over workgroups, and untold, whole."""
    ctx = [900, 0, 1, 40, 257]
    for max_ctx in (8192, 1024):
        check_decode(ops, "bf16", ctx, Hq, Hkv, D, 16, decode_rules(name, ctx, Hq), max_ctx=max_ctx, holes=True)
        check_decode(ops, "f32", ctx, Hq, Hkv, D, 32, decode_rules(name, ctx, Hq), max_ctx=max_ctx)


@pytest.mark.parametrize("Hkv", [1, 2, 8])
def test_decode_pages_ahead(ops, Hkv):
    """First tiles at every place of a window of 64 page ids, and prefixes that end in every one."""
    for w in (3960, 3991, 4000, 4070, 4100):
        ctx = [8000, 5000, 1100 + w // 8]
        check_decode(ops, "bf16", ctx, 2 * Hkv, Hkv, 64, 16, dict(window=w, prefix_lens=np.array([w % 1500, 1030, 7])))
    check_decode(ops, "bf16", [20000], Hkv, Hkv, 64, 16, {})


@pytest.mark.parametrize("cap", [1e-3, 0.5, 50.0, 1e6])
def test_decode_caps(ops, cap):
    for std in (0.3, 4.0, 20.0):
        check_decode(ops, "bf16", [300, 40], 8, 2, 128, 16, dict(softcap=cap), std=std)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", RULES)
@pytest.mark.parametrize("D", [64, 128])
def test_decode_error(ops, dtype, name, D):
    """Element by element, within the bounds that attn_error derives (16 bits of a probability in bf16)."""
    import torch
    ctx, Hq, Hkv, bs, scale = [1, 2, 5, 33, 70, 150, 400], 8, 2, 16, 1 / math.sqrt(D)
    kw = _modifiers(name, Hq, len(ctx))
    say(f"attn_decode_fp4 {dtype} D={D} {name}")
    for std in (0.3, 1.5):
        table, kc, vc = paged4(91, ctx, Hkv, D, bs)
        q = gen(91, "q", (len(ctx), Hq, D), dtype, std)
        got = ops.opscale_attn_decode_fp4(cuda(q), u8(kc), u8(vc), i32(table), i32(ctx), max(ctx), scale, **on_gpu(kw))
        torch.cuda.synchronize()
        kh, vh = narrow.unpack(kc), narrow.unpack(vc)
        want, bound = np.zeros((2, len(ctx), Hq, D))
        for b, n in enumerate(ctx):
            keys = _keys(kw, n - 1, n)
            page, off = table[b][keys // bs], keys % bs
            for h in range(Hq):
                g = h // (Hq // Hkv)
                want[b, h], bound[b, h] = bounded_row(
                    f64(q)[b, h], kh[page, off, g], vh[page, off, g], n - 1, keys, scale, kw["softcap"],
                    float(kw["slopes"][h]) if "slopes" in kw else 0.0, dtype, pieces=2)
        within(f64(got.cpu()), want, bound, f"std {std}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_masked_nan(ops, dtype):
    """Groups of NaN in masked rows and pages that are not there reach no output; in a row that is seen,
    a K group its head's outputs, a V group its 32 elements; a query's NaN its own head."""
    import torch
    ctx, Hq, Hkv, D, bs = [300, 90, 40], 8, 2, 128, 16
    kw = dict(window=50, prefix_lens=np.array([20, 5, 0]), softcap=9.0)
    table, kc, vc = paged4(83, ctx, Hkv, D, bs)
    table[2, 1] = -1
    seen = np.zeros((kc.shape[0], bs), bool)
    for b, n in enumerate(ctx):
        for j in step.visible(n - 1, n, True, 50, int(kw["prefix_lens"][b]), 0):
            if table[b, j // bs] >= 0:
                seen[table[b, j // bs], j % bs] = True
    kb, vb = kc.copy(), vc.copy()
    for c in (kb, vb):
        s = c.reshape(*c.shape[:2], -1)[:, :, bs * 64:].reshape(-1, Hkv, 4, bs)
        s[np.broadcast_to(~seen[:, None, None], s.shape)] = 255
        c.reshape(*c.shape[:2], -1)[:, :, bs * 64:] = s.reshape(-1, Hkv, 4 * bs)
    q0 = gen(83, "q", (3, Hq, D), dtype, 1.5)
    q = q0.clone()
    q[1, 0] = float("nan")
    say(f"decode fp4: masked NaN {dtype}")
    run = lambda: f64(ops.opscale_attn_decode_fp4(cuda(q), u8(kb), u8(vb), i32(table), i32(ctx), 300, 0.1,  # noqa: E731
                                                  **on_gpu(kw)).cpu())
    got = run()
    assert np.isnan(got[1, 0]).all()
    kh, vh = narrow.unpack(kc), narrow.unpack(vc)
    ref, weighted = (step.attn_decode_mod(f64(q0), kh, v, table, ctx, 0.1, **kw) for v in (vh, np.abs(vh)))
    got[1, 0] = ref[1, 0]
    dot = 0.1 * np.abs(f64(q0)).sum(-1).max() * np.nanmax(np.abs(kh))
    tol = tolerance(ref, weighted, dtype, D, 300, dot, 9.0, 0.0)
    near(got, ref, tol, "the others")
    page, off = table[0, 290 // bs], 290 % bs  # a row that sequence 0 sees
    vb[page, 1].reshape(-1)[bs * 64 + 2 * bs + off] = 255
    got = run()
    assert np.isnan(got[0, 4:, 64:96]).all()
    got[0, 4:, 64:96], got[1, 0] = ref[0, 4:, 64:96], ref[1, 0]
    near(got, ref, tol, "beside a V group of NaN")
    kb[page, 0].reshape(-1)[bs * 64 + 3 * bs + off] = 255
    got = run()
    assert np.isnan(got[0, :4]).all() and np.isfinite(got[0, 4:, :64]).all() and np.isfinite(got[2]).all()


def test_decode_scales_far_apart(ops):
    """Scales from 2^-100 to 2^60, the smallest numbers of the cache among them."""
    import torch
    say("decode fp4: scales far apart")
    ctx, Hq, Hkv, D, bs = [200], 4, 1, 128, 16
    table, kc, vc = paged4(84, ctx, Hkv, D, bs, low=27, high=187)
    kc = paged4(84, ctx, Hkv, D, bs)[1]  # (the same pages, scales near 1)
    q = gen(84, "q", (1, Hq, D), "f32", 1.0)
    got = ops.opscale_attn_decode_fp4(cuda(q), u8(kc), u8(vc), i32(table), i32(ctx), 200, 0.1)
    torch.cuda.synchronize()
    kh, vh = narrow.unpack(kc), narrow.unpack(vc)
    ref, weighted = (step.attn_decode_mod(f64(q), kh, v, table, ctx, 0.1) for v in (vh, np.abs(vh)))
    dot = 0.1 * np.abs(f64(q)).sum(-1).max() * np.nanmax(np.abs(kh))
    near(f64(got.cpu()), ref, tolerance(ref, weighted, "f32", D, 200, dot, None, 0.0), "decode")


def test_decode_cache_past_32_bits(ops):
    """A cache of more than 2^32 bytes, its last pages used."""
    import torch
    bs, Hkv, D, Hq = 16, 8, 128, 16
    nb = (1 << 32) // (bs * Hkv * 68) + 64
    say("attn_decode_fp4: a cache past 2^32 bytes")
    kc = torch.zeros(nb, Hkv, bs, 68, dtype=torch.uint8, device="cuda")
    vc = torch.zeros_like(kc)
    ctx = [1000, 600]
    table = np.stack([nb - 1 - np.arange(64), np.r_[nb // 2 + np.arange(38), np.zeros(26)]]).astype(np.int32)
    used = np.unique(table)
    rng = np.random.default_rng(4)
    small = []
    for _ in range(2):
        flat = rng.integers(0, 256, size=(len(used), Hkv, bs * 68)).astype(np.uint8)
        flat[:, :, bs * 64:] = rng.integers(124, 129, size=(len(used), Hkv, bs * 4))
        small.append(u8(flat.reshape(len(used), Hkv, bs, 68)))
    at = torch.from_numpy(used).long().cuda()
    kc[at], vc[at] = small
    q = cuda(gen(74, "q", (2, Hq, D), "bf16", 1.5))
    kw = dict(softcap=20.0, window=700)
    got = ops.opscale_attn_decode_fp4(q, kc, vc, i32(table), i32(ctx), 1000, 0.08, **kw)
    ref = ops.opscale_attn_decode_fp4(q, *small, i32(np.searchsorted(used, table)), i32(ctx), 1000, 0.08, **kw)
    torch.cuda.synchronize()
    assert torch.equal(got, ref) and bool(got.abs().sum() > 0)


def test_streams_workspaces_and_graph(ops):
    """A step's write and attention, captured, and replayed between eager calls on the same cache."""
    import torch
    say("kv fp4: streams, graph")
    ctx, Hq, Hkv, D, bs = [300, 64, 5, 0], 8, 2, 128, 16
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    check_decode(ops, "bf16", ctx, Hq, Hkv, D, bs, decode_rules("all", ctx, Hq), stream=s)
    table, kc, vc = paged4(85, ctx, Hkv, D, bs)
    kc, vc, lens = u8(kc), u8(vc), i32(ctx)
    slots = i32([table[b, (n - 1) // bs] * bs + (n - 1) % bs if n else -1 for b, n in enumerate(ctx)])
    table = i32(table)
    q, kv = cuda(gen(85, "q", (4, Hq, D), "bf16")), cuda(gen(85, "k", (4, 2 * Hkv, D), "bf16"))
    out = torch.empty(4, Hq, D, dtype=torch.bfloat16, device="cuda")
    d = on_gpu(decode_rules("all", ctx, Hq))
    ws = torch.full((ops.opscale_attn_decode_fp4_workspace_size(4, Hq, D, 300),), 255, dtype=torch.uint8, device="cuda")

    def call(o, w=None):
        ops.opscale_kv_write_fp4(kv[:, :Hkv], kv[:, Hkv:], kc, vc, slots)
        return ops.opscale_attn_decode_fp4(q, kc, vc, table, lens, 300, 0.09, workspace=w, out=o, **d)
    call(out, ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(out, ws)
    for i in range(4):
        q.copy_(gen(76 + i, "q", (4, Hq, D), "bf16"))
        kv.copy_(gen(76 + i, "k", (4, 2 * Hkv, D), "bf16"))
        lens.copy_(i32([300 - 90 * i, 64 - i, 5, i]))
        out.fill_(float("nan"))
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.nan_to_num(9.0), call(torch.empty_like(out)).nan_to_num(9.0)), i


def test_refusals(ops):
    import torch
    say("fp4: refusals")
    bf = dict(dtype=torch.bfloat16, device="cuda")
    q, kv = torch.zeros(2, 4, 64, **bf), torch.zeros(2, 4, 64, **bf)
    kc = torch.zeros(4, 2, 16, 34, dtype=torch.uint8, device="cuda")
    vc = kc.clone()
    good = dict(q=q, k_cache=kc, v_cache=vc, block_table=i32([[0, 1], [2, 3]]), context_lens=i32([20, 3]),
                max_context_len=20, scale=0.1)
    ops.opscale_attn_decode_fp4(**good)
    small = torch.zeros(16, dtype=torch.uint8, device="cuda")
    for bad in (dict(q=q.half()), dict(q=q.cpu()), dict(q=torch.zeros(2, 4, 128, **bf)), dict(k_cache=kc.float()),
                dict(v_cache=vc[:3]), dict(k_cache=kc[..., :33].contiguous()), dict(k_cache=kc[0]),
                dict(k_cache=kc.view(4, 4, 8, 34), v_cache=vc.view(4, 4, 8, 34)),
                dict(block_table=i32([[0, 1]])), dict(context_lens=i32([1, 2]).long()), dict(workspace=small),
                dict(softcap=-1.0), dict(window=-3), dict(slopes=f32([1, 2])), dict(doc_starts=i32([1, 2, 3])),
                dict(out=q), dict(max_context_len=0), dict(scale=0.0)):
        with pytest.raises(ops.OpscaleError):
            ops.opscale_attn_decode_fp4(**dict(good, **bad))
    k, v, slots = kv[:, :2], kv[:, 2:], i32([0, 1])
    ops.opscale_kv_write_fp4(k, v, kc, vc, slots)
    for bad in ((k.half(), v.half(), kc, vc, slots), (k, v.float(), kc, vc, slots), (k[:1], v, kc, vc, slots),
                (k, v.contiguous(), kc, vc, slots), (k, v, kc, kc, slots), (k, v, kc, vc[:2], slots),
                (k, v, kc, vc, slots.long()), (k, v, kc, vc, slots[:1]), (kv[:, :3], kv[:, :3], kc, vc, slots),
                (k, v, kc.cpu(), vc, slots)):
        with pytest.raises(ops.OpscaleError):
            ops.opscale_kv_write_fp4(*bad)
    tab, cu = i32([[0, 1], [2, 3]]), i32([0, 5, 9])
    ops.opscale_kv_read_fp4(kc, vc, tab, cu, 9)
    for kw in (dict(dtype=torch.float16), dict(k=torch.zeros(9, 2, 64, **bf)), dict(first_keys=i32([0])),
               dict(k=torch.zeros(8, 2, 64, **bf), v=torch.zeros(8, 2, 64, **bf))):
        with pytest.raises(ops.OpscaleError):
            ops.opscale_kv_read_fp4(kc, vc, tab, cu, 9, **kw)
    out = torch.zeros(9, 2, 64, **bf)
    with pytest.raises(ops.OpscaleError):
        ops.opscale_kv_read_fp4(kc, vc, tab, cu, 9, k=out, v=out)
    with pytest.raises(ops.OpscaleError):
        ops.opscale_kv_read_fp4(kc, vc, tab, i32([0, 5]), 9)


def test_timing_and_profile(ops):
    import torch
    say("fp4: timing and profile")
    ctx, Hq, Hkv, D, bs = [100, 40], 8, 2, 128, 16
    table, kc, vc = paged4(86, ctx, Hkv, D, bs)
    kc, vc, table, lens = u8(kc), u8(vc), i32(table), i32(ctx)
    q, kv = cuda(gen(86, "q", (2, Hq, D), "bf16")), cuda(gen(86, "k", (2, 2 * Hkv, D), "bf16"))
    k, v, slots = kv[:, :Hkv], kv[:, Hkv:], i32([0, 1])
    t = ops.opscale_kv_write_fp4(k, v, kc, vc, slots, timed=True)
    assert t.elapsed_us > 0 and t.alg_bytes == 2 * 2 * Hkv * (2 * D + 68) + 8
    (rk, rv), t = ops.opscale_kv_read_fp4(kc, vc, table, i32([0, 30, 50]), 50, timed=True)
    assert t.alg_bytes == 2 * 50 * Hkv * (2 * D + 68) + 4 * (50 // 16 + 4)
    o, t = ops.opscale_attn_decode_fp4(q, kc, vc, table, lens, 100, 0.1, timed=True)
    assert t.alg_bytes == 2 * 140 * Hkv * 68 + 2 * 2 * 2 * Hq * D + 4 * (7 + 3 + 2) and t.alg_flops == 4 * Hq * D * 140
    ws = torch.empty(ops.opscale_attn_decode_fp4_workspace_size(2, Hq, D, 100), dtype=torch.uint8, device="cuda")
    for d in (ops.desc_kv_write_fp4(k, v, kc, vc, slots),
              ops.desc_kv_read_fp4(kc, vc, table, i32([0, 30, 50]), rk, rv),
              ops.desc_attn_decode_fp4(q, kc, vc, table, lens, o, 100, 0.1, ws, softcap=5.0)):
        assert ops.opscale_op_profile(d, 1, 3).us_median > 0
