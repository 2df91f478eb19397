"""GPU operators of 8 and 4 bits, called as the other tests do not: tensors past 2^32 bytes, batches in
which no sequence has a key, two calls at once, and streams of a share of the CUs."""
import numpy as np
import pytest

import fp8_plan
from oracle import narrow
from parity_util import cuda, f64, gen, say
from test_gpu_attn_mods import i32
from test_gpu_fp4 import paged4, u8
from test_gpu_fp8 import ops, reference  # noqa: F401
from test_gpu_fp8_paths import codes_on_gpu, scales_of

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------- past 32 bits ---
def test_quantize_past_32_bits(ops):
    """More than 2^32 bytes of x and of q: a block's codes are its elements' wherever it lies."""
    import torch
    M, K = 1 << 16, (1 << 16) + 16
    say(f"quantize_fp8: {M} x {K}")
    x = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    rows = torch.tensor([0, 1, M // 2, M - 5, M - 1], device="cuda")
    x[rows] = cuda(gen(3, "x", (5, K), "bf16"))
    q, s = ops.opscale_quantize_fp8(x)
    q1, s1 = ops.opscale_quantize_fp8(x[rows])
    torch.cuda.synchronize()
    assert torch.equal(q.view(torch.uint8)[rows], q1.view(torch.uint8)) and torch.equal(s[:, rows], s1)
    s[:, rows] = 2.0 ** -100  # (a block of zeros has the lowest scale and zeros for codes)
    assert bool((s == 2.0 ** -100).all())
    q.view(torch.uint8)[rows] = 0
    assert not any(bool(q.view(torch.uint8)[m:m + 4096].any()) for m in range(0, M, 4096))


@pytest.mark.parametrize("M,N,K", [(3, 1 << 19, 8208), (40, 1 << 19, 8208), (150, 1 << 19, 8208)])
def test_weights_past_32_bits(ops, M, N, K):
    import torch
    path = fp8_plan.plan(M, N, K).path
    say(f"linear_fp8 {M} x {N} x {K} ({path}): W of more than 2^32 bytes")
    x, w = codes_on_gpu(M, K, 81, 0), torch.zeros(N, K, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    cols = np.r_[0:128, N // 2:N // 2 + 128, N - 128:N]
    w.view(torch.uint8)[torch.from_numpy(cols).cuda()] = codes_on_gpu(384, K, 82, 0).view(torch.uint8)
    xs, ws = scales_of(M, N, K, 83)
    y = ops.opscale_linear_fp8(x, cuda(torch.from_numpy(xs)), w, cuda(torch.from_numpy(ws)))
    torch.cuda.synchronize()
    rows = np.unique([0, M // 2, M - 1])
    xc = x.view(torch.uint8).cpu().numpy()[rows]
    for n0 in (0, N // 2, N - 128):
        want, off = reference(xc, xs[:, rows], w.view(torch.uint8)[n0:n0 + 128].cpu().numpy(), ws[n0 // 128:n0 // 128 + 1],
                              None, "bf16")
        assert (np.abs(f64(y[torch.from_numpy(rows).cuda(), n0:n0 + 128].cpu()) - want) <= off).all(), n0
    y[:, torch.from_numpy(cols).cuda()] = 0
    assert not bool(y.any())  # (the other columns' weights are zeros)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_results_past_32_bits(ops, dtype):
    """More than 2^32 bytes of y; rows whose x is zeros are the bias."""
    import torch
    from parity_util import torch_dtype
    M, N, K = 70001, 32776, 144
    say(f"linear_fp8 {dtype} {M} x {N} x {K} ({fp8_plan.plan(M, N, K, dtype)})")
    x = torch.zeros(M, K, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    rows = np.r_[0, 1, M // 2, M - 1]
    x.view(torch.uint8)[torch.from_numpy(rows).cuda()] = codes_on_gpu(4, K, 84, 0).view(torch.uint8)
    w, (xs, ws) = codes_on_gpu(N, K, 85, 0), scales_of(M, N, K, 86)
    b = cuda(gen(87, "bias", (N,), dtype, 3.0))
    y = ops.opscale_linear_fp8(x, cuda(torch.from_numpy(xs)), w, cuda(torch.from_numpy(ws)), b, dtype=torch_dtype(dtype))
    torch.cuda.synchronize()
    xc = x.view(torch.uint8)[torch.from_numpy(rows).cuda()].cpu().numpy()
    want, off = reference(xc, xs[:, rows], w.view(torch.uint8).cpu().numpy()[-1032:], ws[-9:], f64(b.cpu())[-1032:], dtype)
    assert (np.abs(f64(y[torch.from_numpy(rows).cuda(), -1032:].cpu()) - want) <= off).all()
    y[torch.from_numpy(rows).cuda()] = b
    for m in range(0, M, 4096):
        assert bool((y[m:m + 4096] == b).all()), m


# ----------------------------------------------------------- empty batches ---
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,told", [(1, 1), (3, 900), (3, 9000), (100, 9000), (513, 9000), (30000, 64)])
def test_decode_of_no_keys(ops, dtype, B, told):
    """Every sequence without a key that its query sees: rows of zeros, on every plan."""
    import torch
    from parity_util import torch_dtype
    say(f"attn_decode_fp4 {dtype}: {B} sequences of no keys, told {told}")
    Hq, Hkv, D = 4, 2, 64
    kc = torch.full((3, Hkv, 16, 34), 255, dtype=torch.uint8, device="cuda")
    q = torch.full((B, Hq, D), float("nan"), dtype=torch_dtype(dtype), device="cuda")
    table = torch.zeros(B, 4, dtype=torch.int32, device="cuda")
    for ctx, kw in ((np.zeros(B), {}), (np.full(B, 50), dict(doc_starts=i32(np.full(B, 50)))),
                    (np.full(B, 50), dict(doc_starts=i32(np.full(B, 60)), window=9))):
        out = torch.full((B, Hq, D), 7.0, dtype=q.dtype, device="cuda")
        ops.opscale_attn_decode_fp4(q, kc, kc.clone(), table, i32(ctx), told, 0.1, out=out, **kw)
        torch.cuda.synchronize()
        assert bool((out == 0).all()), kw


def test_decode_of_one_among_many(ops):
    """The last of 30000 sequences has keys, the first some, the others none."""
    import torch
    B, Hq, Hkv, D, bs = 30000, 4, 2, 64, 16
    say("attn_decode_fp4: 30000 sequences, two with keys")
    ctx = [700, 90]
    table, kc, vc = paged4(95, ctx, Hkv, D, bs)
    q = cuda(gen(95, "q", (B, Hq, D), "bf16", 1.5))
    lens = np.zeros(B)
    lens[[0, B - 1]] = ctx
    wide = torch.full((B, table.shape[1]), -1, dtype=torch.int32, device="cuda")
    wide[[0, B - 1]] = i32(table)
    out = ops.opscale_attn_decode_fp4(q, u8(kc), u8(vc), wide, i32(lens), 700, 0.12)
    want = ops.opscale_attn_decode_fp4(q[[0, B - 1]].contiguous(), u8(kc), u8(vc), i32(table), i32(ctx), 700, 0.12)
    torch.cuda.synchronize()
    # (sums of another order: a few roundings of 2^-24, then one of bf16 each)
    assert bool(((out[[0, B - 1]].double() - want.double()).abs() <= 2.0 ** -7 * want.double().abs() + 1e-5).all())
    assert not bool(out[1:B - 1].any())


# -------------------------------------------------- streams, calls at once ---
def _operands(ops):
    import torch
    M, N, K = 300, 5128, 4112  # tiles, K in ranges
    x, w = codes_on_gpu(M, K, 91, 0), codes_on_gpu(N, K, 92, 0)
    xs, ws = (cuda(torch.from_numpy(a)) for a in scales_of(M, N, K, 93))
    x1, w1 = codes_on_gpu(48, K, 94, 0), codes_on_gpu(N, K, 95, 0)
    xs1, ws1 = (cuda(torch.from_numpy(a)) for a in scales_of(48, N, K, 96))
    ctx = [2000, 300, 1] * 30
    table, kc, vc = paged4(97, ctx, 4, 128, 16)
    q = cuda(gen(97, "q", (90, 8, 128), "bf16", 1.5))
    dec = (q, u8(kc), u8(vc), i32(table), i32(ctx), 2000, 0.09)
    big = cuda(gen(98, "x", (3000, 4112), "bf16"))
    torch.cuda.synchronize()
    return [lambda s: ops.opscale_linear_fp8(x, xs, w, ws, stream=s), lambda s: ops.opscale_linear_fp8(x1, xs1, w1, ws1, stream=s),
            lambda s: ops.opscale_attn_decode_fp4(*dec, stream=s),
            lambda s: ops.opscale_quantize_fp8(big, stream=s)[0].view(torch.uint8)]


def test_calls_at_once(ops):
    """The same calls on two streams at once, many times, with a workspace of each call's own."""
    import torch
    say("operators of 8 and 4 bits: two streams")
    calls = _operands(ops)
    want = [c(None) for c in calls]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for i in range(len(calls)):
            for j, s in enumerate(streams):
                with torch.cuda.stream(s):
                    k = (i + j * 2) % len(calls)
                    got.append((k, calls[k](None)))
    torch.cuda.synchronize()
    for k, y in got:
        assert torch.equal(y, want[k]), k


@pytest.mark.parametrize("cus", [13, 128, 230])
def test_share_of_the_cus(ops, cus):
    import torch
    say(f"operators of 8 and 4 bits on {cus} CUs")
    n, x, il = ops.opscale_cu_layout()[:3]
    calls = _operands(ops)
    want = [c(None) for c in calls]
    torch.cuda.synchronize()
    s = ops.opscale_cu_stream_create(ops.opscale_cu_mask_build(n, x, il, 0, cus))
    try:
        got = [c(s) for c in calls]
        torch.cuda.synchronize()
    finally:
        ops.opscale_cu_stream_destroy(s)
    for k, (a, b) in enumerate(zip(got, want)):
        assert torch.equal(a, b), k


def test_narrow_values_of_a_read_past_the_last_sequence(ops):
    """Rows of k and v behind the last sequence stay, those of sequences without rows are nobody's."""
    import torch
    say("kv_read_fp4: no rows")
    _, kc, vc = paged4(99, [40], 2, 128, 16)
    k, v = (torch.full((20, 2, 128), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ops.opscale_kv_read_fp4(u8(kc), u8(vc), i32([[0, 1, 2]] * 4), i32([0, 0, 3, 3, 3]), 20, i32([9, 1, 0, 0]), k=k, v=v)
    torch.cuda.synchronize()
    for got, c in ((k, kc), (v, vc)):
        assert (got[3:] == 5).all() and np.array_equal(f64(got[:3].cpu()), narrow.unpack(c)[0, 1:4], equal_nan=True)
