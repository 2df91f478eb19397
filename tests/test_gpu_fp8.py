"""GPU activations to e4m3 (bit by bit) and the linear of e4m3 operands, element by element.

What a result may be off by (u = 2^-24):
  * bf16: the matrix instruction cuts each of the eight products of k = 8 i .. 8 i + 7 to 2^-13 of the
    largest of them, G: 8 * 2^-13 sum over groups of G; it adds the sixteen groups of a block, of P
    = sum |products| in all, with at most 16 roundings of 2^-23 P.
  * fp32: four instructions of 32 whole products each, at most 40 roundings of 2^-23 P.
  * both: the scales' product and its product with a block's sum, 2 u P each, and a chain over the blocks
    (and the K splits), a rounding each of at most the whole row's P; the bias one; the result half a
    step, 2^-8 (bf16) or u (fp32) of itself.
"""
import numpy as np
import pytest

from oracle import narrow
from parity_util import cuda, f64, gen, say, torch_dtype

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def ops():
    import paper_2608_13499_amd as o
    o.load()
    return o


# ----------------------------------------------------------------- quantize ---
def check_quantize(ops, x, stream=None):
    """x: a GPU matrix; its codes' values and scales are the definition's."""
    import torch
    q, s = ops.opscale_quantize_fp8(x, stream=stream)
    torch.cuda.synchronize()
    assert q.dtype == torch.float8_e4m3fn and q.shape == x.shape and s.shape == (-(-x.shape[1] // 128), x.shape[0])
    want, scales = narrow.quantize_fp8(f64(x.cpu()))
    assert np.array_equal(f64(s.cpu()), scales, equal_nan=True)
    fine = np.isfinite(np.repeat(scales.T, 128, 1)[:, :x.shape[1]])
    got = q.cpu().double().numpy()
    assert np.array_equal(got[fine], want[fine])
    return q, s


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K", [(1, 16), (1, 4096), (3, 128), (17, 144), (15, 688), (33, 512), (2, 1040), (130, 256)])
def test_quantize(ops, dtype, M, K):
    say(f"quantize_fp8 {dtype} {M} x {K}")
    x = f64(gen(3, "x", (M, K), dtype))
    x *= 2.0 ** np.random.default_rng(K).integers(-9, 9, size=(M, 1))
    import torch
    check_quantize(ops, torch.from_numpy(x).to(torch_dtype(dtype)).cuda())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_values(ops, dtype):
    """Ties, every code's own value, largest magnitudes next to where the scale doubles, zeros, the
    smallest and largest numbers, infinities and NaN in one block of a row."""
    import torch
    say(f"quantize_fp8 {dtype}: values")
    dt = torch_dtype(dtype)
    codes = np.concatenate([narrow.E4M3[:127], -narrow.E4M3[:127], [448.0, 0.0]])
    ties = 0.5 * (narrow.E4M3[:126] + narrow.E4M3[1:127])
    rows = [codes, np.concatenate([ties, [448, 0], -ties, [448, -0.0]]), np.zeros(256)]
    for e in (-140, -130, -126, -110, -99, -40, 3, 90, 110, 118, 119):
        for top in (1.0, 1.74, 1.75, 1.76, 1.99):
            rows.append(np.where(np.arange(256) % 128 == 5, top * 2.0 ** (e + 8), codes * 2.0 ** (e - 1)))
    x = torch.from_numpy(np.clip(np.stack(rows), -3.3e38, 3.3e38)).to(dt)
    bad = x[:4].clone()
    bad[0, 3], bad[1, 200], bad[2, 127], bad[3, 128] = float("nan"), float("inf"), -float("inf"), float("nan")
    check_quantize(ops, torch.cat([x, bad]).cuda())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_strides(ops, dtype):
    """Columns of a wider tensor, on a stream of its own; nothing else is written."""
    import torch
    say(f"quantize_fp8 {dtype}: strided rows")
    wide = cuda(gen(5, "x", (21, 1024), dtype))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    check_quantize(ops, wide[:, 256:256 + 400], stream=s)
    buf = torch.full((2 + 21, 400), 7, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    sc = torch.full((6, 21), -1.0, device="cuda")
    ops.opscale_quantize_fp8(wide[:, :400], q=buf[1:22], scales=sc[1:5])
    torch.cuda.synchronize()
    assert (buf.view(torch.uint8)[[0, 22]] == 7).all() and (sc[[0, 5]] == -1).all() and (sc[1:5] > 0).all()


# ------------------------------------------------------------------- linear ---
def operands(M, N, K, seed, spread=0):
    """e4m3 values and scales: spread 0, normal elements; 1, every code alike (magnitudes over 2^17)."""
    rng = np.random.default_rng([seed, M, N, K])

    def codes(r):
        if spread:
            c = rng.integers(0, 254, size=(r, K))
            return np.where(c >= 127, c + 1, c)
        return narrow.encode(np.clip(rng.normal(size=(r, K)) * 60, -448, 448), "e4m3")
    nkb, nnb = -(-K // 128), -(-N // 128)
    xs = (2.0 ** rng.integers(-6, 2, size=(nkb, M)) * (1 + rng.random((nkb, M)))).astype(np.float32)
    ws = np.exp(0.5 * rng.normal(size=(nnb, nkb))).astype(np.float32) * np.float32(0.01)
    return codes(M).astype(np.uint8), xs, codes(N).astype(np.uint8), ws


def reference(xc, xs, wc, ws, bias, dtype):
    """(result, what it may be off by)."""
    x, w = narrow.E4M3[xc], narrow.E4M3[wc]
    (M, K), N = x.shape, w.shape[0]
    nkb = xs.shape[0]
    off, mass, want = np.zeros((M, N)), np.zeros((M, N)), np.zeros((M, N))
    for b in range(nkb):
        k = slice(b * 128, min(K, (b + 1) * 128))
        f = np.abs(np.outer(xs[b].astype(np.float64), np.repeat(ws[:, b].astype(np.float64), 128)[:N]))
        P = f * (np.abs(x[:, k]) @ np.abs(w[:, k]).T)
        if dtype == "bf16":
            for i in range(k.start, k.stop, 8):
                off += 2.0 ** -10 * f * (np.abs(x[:, None, i:i + 8]) * np.abs(w[None, :, i:i + 8])).max(-1)
            off += 16 * 2 * U * P
        else:
            off += 40 * 2 * U * P
        off += 4 * U * P
        mass += P
        want += np.outer(xs[b].astype(np.float64), np.repeat(ws[:, b].astype(np.float64), 128)[:N]) * (x[:, k] @ w[:, k].T)
    if bias is not None:
        want, mass = want + bias, mass + np.abs(bias)
    off += (nkb + 64 + 1) * U * mass  # (64: more splits than any plan takes)
    return want, off + (2.0 ** -8 if dtype == "bf16" else U) * (np.abs(want) + off) + 1e-30


def check_linear(ops, dtype, M, N, K, bias=False, seed=7, spread=0, workspace=None, stream=None):
    import torch
    say(f"linear_fp8 {dtype} {M} x {N} x {K} bias={bias} spread={spread} workspace={workspace}")
    xc, xs, wc, ws = operands(M, N, K, seed, spread)
    e4 = lambda a: torch.from_numpy(a).cuda().view(torch.float8_e4m3fn)  # noqa: E731
    b = gen(seed, "bias", (N,), dtype, 3.0) if bias else None
    out = torch.full((M + 2, N), float("nan"), dtype=torch_dtype(dtype), device="cuda")
    y = ops.opscale_linear_fp8(e4(xc), cuda(torch.from_numpy(xs)), e4(wc), cuda(torch.from_numpy(ws)),
                               None if b is None else cuda(b), y=out[1:M + 1], workspace=workspace, stream=stream)
    torch.cuda.synchronize()
    assert torch.isnan(out[0]).all() and torch.isnan(out[M + 1]).all(), "rows around y were written"
    want, off = reference(xc, xs, wc, ws, None if b is None else f64(b), dtype)
    got = f64(y.cpu())
    assert np.isfinite(got).all()
    r = np.abs(got - want) / off
    say(f"  {r.max():.3f} of the bound; error {np.linalg.norm(got - want) / np.linalg.norm(want):.2e}")
    assert r.max() <= 1.0, f"{r.max():.3f} of the bound at {np.unravel_index(r.argmax(), r.shape)}"
    return y


# Few outputs; few rows (each count of row blocks, K split and not); tiles (K split and not, edges in M
# and N); K of one short block to many.
SHAPES = [(1, 8, 16), (1, 136, 128), (2, 512, 4096), (16, 96, 144), (33, 264, 1040), (65, 640, 272), (127, 72, 1152),
          (128, 256, 688), (300, 200, 4112),
          (2, 6160, 400), (16, 6152, 2064), (17, 3208, 144), (33, 2072, 1040), (48, 2048, 2576), (65, 1240, 272),
          (128, 792, 688), (127, 776, 2064),
          (129, 704, 128), (130, 712, 400), (200, 520, 1040), (256, 512, 256), (300, 392, 2064), (513, 264, 144)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_linear(ops, dtype, M, N, K):
    check_linear(ops, dtype, M, N, K)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [(5, 200, 656), (40, 2056, 656), (40, 128, 4096), (140, 712, 1040), (258, 392, 400)])
def test_linear_bias_and_spread(ops, dtype, M, N, K):
    check_linear(ops, dtype, M, N, K, bias=True)
    check_linear(ops, dtype, M, N, K, spread=1)
    a = check_linear(ops, dtype, M, N, K, bias=True, spread=1, workspace=False)
    b = check_linear(ops, dtype, M, N, K, bias=True, spread=1, workspace=False)
    assert bool((a == b).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [(1000, 520, 144), (770, 1288, 272), (2, 57344, 128), (4, 4096, 14336), (1023, 4616, 400),
                                   (1000, 3080, 12304), (1023, 8712, 400), (8200, 12296, 400)])
def test_linear_large(ops, dtype, M, N, K):
    """Several tiles of each shape a dimension, several a workgroup; a row or two of wide and of deep weights."""
    import torch
    say(f"linear_fp8 {dtype} {M} x {N} x {K}, sampled")
    xc, xs, wc, ws = operands(M, N, K, 11)
    e4 = lambda a: torch.from_numpy(a).cuda().view(torch.float8_e4m3fn)  # noqa: E731
    y = ops.opscale_linear_fp8(e4(xc), cuda(torch.from_numpy(xs)), e4(wc), cuda(torch.from_numpy(ws)),
                               dtype=torch_dtype(dtype))
    torch.cuda.synchronize()
    got = f64(y.cpu())
    assert np.isfinite(got).all()
    rng = np.random.default_rng(0)
    rows, blocks = np.unique(np.r_[0, M - 1, rng.integers(0, M, 12)]), np.unique(np.r_[0, ws.shape[0] - 1, rng.integers(0, ws.shape[0], 2)])
    for nb in blocks:
        n = slice(nb * 128, min(N, (nb + 1) * 128))
        want, off = reference(xc[rows], xs[:, rows], wc[n], ws[nb:nb + 1], None, dtype)
        assert (np.abs(got[rows, n] - want) <= off).all()
    # every element, to the size of the result
    x, w = torch.from_numpy(narrow.E4M3[xc]).cuda(), torch.from_numpy(narrow.E4M3[wc]).cuda()
    x = x * cuda(torch.from_numpy(xs)).double().t().repeat_interleave(128, 1)[:, :K]
    w = w * cuda(torch.from_numpy(ws)).double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
    want = x @ w.t().contiguous()
    rms = float(((y.double() - want) ** 2).sum(1).sqrt().div((want ** 2).sum(1).sqrt()).max())
    # a row's roundings are independent: bf16 2^-9 rms at most; fp32 sqrt(K) roundings of partial sums of the
    # result's size
    assert rms <= (2.0 ** -9 * 1.1 if dtype == "bf16" else 2 * U * np.sqrt(K)), rms


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_special_values(ops, dtype):
    """A NaN element or scale, an infinite scale: in their row or columns of a block, nowhere else."""
    import torch
    say(f"linear_fp8 {dtype}: NaN and infinity")
    for M, N in ((3, 264), (40, 2056), (150, 712)):
        K = 304
        xc, xs, wc, ws = operands(M, N, K, 13)
        want, off = reference(xc, xs, wc, ws, None, dtype)
        xc[1, 290], wc[200, 5] = 0x7f, 0xff
        xs[0, 2] = np.nan
        e4 = lambda a: torch.from_numpy(a).cuda().view(torch.float8_e4m3fn)  # noqa: E731
        y = f64(ops.opscale_linear_fp8(e4(xc), cuda(torch.from_numpy(xs)), e4(wc), cuda(torch.from_numpy(ws)),
                                       dtype=torch_dtype(dtype)).cpu())
        bad = np.zeros((M, N), bool)
        bad[1], bad[2], bad[:, 200] = True, True, True
        assert np.array_equal(np.isnan(y), bad)
        assert (np.abs(y - want)[~bad] <= off[~bad]).all()
        ws[1, 1] = np.inf
        xc[1, 290] = 0
        y = f64(ops.opscale_linear_fp8(e4(xc), cuda(torch.from_numpy(xs)), e4(wc), cuda(torch.from_numpy(ws)),
                                       dtype=torch_dtype(dtype)).cpu())
        assert not np.isfinite(y[:, 128:256]).any() and np.isfinite(np.delete(y, 2, 0)[:, :128]).all()
        assert np.isfinite(np.delete(y, 2, 0)[:, 256:]).all()


def test_unit_weights(ops):
    """W a scaled identity: each result is one product, exact."""
    import torch
    say("linear_fp8: identity")
    K = 384
    w = torch.eye(K, device="cuda").to(torch.float8_e4m3fn)
    ws = torch.full((3, 3), 2.0, device="cuda")
    x = cuda(gen(1, "x", (270, K), "f32"))
    for m in (3, 270):
        q, s = ops.opscale_quantize_fp8(x[:m])
        y = ops.opscale_linear_fp8(q, s, w, ws, dtype=torch.float32)
        torch.cuda.synchronize()
        assert bool((y == 2 * q.float() * s.t().repeat_interleave(128, 1)).all())


def test_empty_and_graph(ops):
    """No rows; a captured chain, replayed between eager calls."""
    import torch
    say("linear_fp8: no rows, graph")
    w = torch.zeros(256, 512, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    ws = torch.ones(2, 4, device="cuda")
    q, s = ops.opscale_quantize_fp8(torch.zeros(0, 512, device="cuda"))
    assert q.shape == (0, 512) and ops.opscale_linear_fp8(q, s, w, ws).shape == (0, 256)
    for M, N in ((5, 256), (48, 2048), (200, 512)):
        xc, xs, wc, wsc = operands(M, N, 2048, 17)
        x = cuda(gen(17, "x", (M, 2048), "bf16"))
        w = torch.from_numpy(wc).cuda().view(torch.float8_e4m3fn)
        ws = cuda(torch.from_numpy(wsc))
        ws_mem = torch.empty(ops.opscale_linear_fp8_workspace_size(M, N, 2048), dtype=torch.uint8, device="cuda")
        q, s = ops.opscale_quantize_fp8(x)
        y = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")

        def chain():
            ops.opscale_quantize_fp8(x, q, s)
            ops.opscale_linear_fp8(q, s, w, ws, y=y, workspace=ws_mem if ws_mem.numel() else None)
        chain()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            chain()
            torch.cuda.synchronize()
            with torch.cuda.graph(g, stream=side):
                chain()
        for i in range(3):
            x.copy_(cuda(gen(18 + i, "x", (M, 2048), "bf16")))
            chain()
            torch.cuda.synchronize()
            want = y.clone()
            y.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert bool((y == want).all()), i


def test_refusals(ops):
    import torch
    say("fp8: refusals")
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    for bad in (x.half(), x.cpu(), x[:, :60].contiguous(), x.t(), x[:, 4:36]):
        with pytest.raises(ops.OpscaleError):
            ops.opscale_quantize_fp8(bad)
    q, s = ops.opscale_quantize_fp8(x)
    for kw in (dict(q=q.view(torch.uint8)), dict(q=q[:3]), dict(scales=s.double()), dict(scales=s.cpu()),
               dict(scales=x.view(torch.float32)[:1, :4])):
        with pytest.raises(ops.OpscaleError):
            ops.opscale_quantize_fp8(x, **kw)
    good = dict(x=q, x_scales=s, W=torch.zeros(32, 64, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn),
                w_scales=torch.ones(1, 1, device="cuda"))
    ops.opscale_linear_fp8(**good)
    y = torch.empty(4, 32, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(x=q.view(torch.uint8)), dict(x=x), dict(W=good["W"][:, :32]), dict(W=good["W"].t()),
                dict(x_scales=s.t()), dict(x_scales=s[:, :3]), dict(w_scales=torch.ones(2, 1, device="cuda")),
                dict(w_scales=torch.ones(1, 1)), dict(bias=torch.ones(32, device="cuda")), dict(dtype=torch.float16),
                dict(y=y[:3]), dict(y=y, dtype=torch.float32), dict(y=q.view(torch.bfloat16)),
                dict(W=good["W"][:30], dtype=torch.bfloat16), dict(W=good["W"][:4])):
        with pytest.raises(ops.OpscaleError):
            ops.opscale_linear_fp8(**dict(good, **bad))


def test_timing_and_profile(ops):
    import torch
    say("fp8: timing and profile")
    M, N, K = 40, 256, 1024
    x = cuda(gen(2, "x", (M, K), "bf16"))
    (q, s), t = ops.opscale_quantize_fp8(x, timed=True)
    assert t.elapsed_us > 0 and t.alg_bytes == 3 * M * K + 4 * M * 8
    w = torch.zeros(N, K, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    ws = torch.ones(2, 8, device="cuda")
    y, t = ops.opscale_linear_fp8(q, s, w, ws, timed=True)
    assert t.elapsed_us > 0 and t.alg_flops == 2 * M * N * K
    assert t.alg_bytes == M * K + N * K + 2 * M * N + 4 * 8 * (M + 2)
    p = ops.opscale_op_profile(ops.desc_quantize_fp8(x, q, s), 1, 3)
    assert p.iters == 3 and p.us_median > 0
    mem = torch.empty(max(1, ops.opscale_linear_fp8_workspace_size(M, N, K)), dtype=torch.uint8, device="cuda")
    p = ops.opscale_op_profile(ops.desc_linear_fp8(q, s, w, ws, y, workspace=mem), 1, 3)
    assert p.us_median > 0 and p.weight_bytes == N * K + 4 * 16
