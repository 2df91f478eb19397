"""GPU linear of e4m3 operands: every tile shape with a bias, with one slice of K to many, K in ranges,
and launches whose workgroups go from tile to tile, which the host's plan says each case is.

Samples are held to the bounds that test_gpu_fp8 derives, every element to the bound with each group's
largest product taken as the sum of the group's: 2^-10 P in the place of 2^-10 sum G.
"""
import numpy as np
import pytest

import fp8_plan
from oracle import narrow
from parity_util import cuda, f64, gen, say, torch_dtype
from test_gpu_fp8 import U, ops, reference  # noqa: F401

pytestmark = pytest.mark.gpu


def codes_on_gpu(rows, K, seed, spread):
    """e4m3 bytes: spread 0, normal elements; 1, every code alike but NaN."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if spread:
        c = torch.randint(0, 254, (rows, K), generator=g, device="cuda", dtype=torch.int16)
        return torch.where(c >= 127, c + 1, c).to(torch.uint8).view(torch.float8_e4m3fn)
    x = torch.empty(rows, K, device="cuda").normal_(0, 60, generator=g)
    return x.clamp(-448, 448).to(torch.float8_e4m3fn)


def scales_of(M, N, K, seed):
    rng = np.random.default_rng([seed, M, N, K])
    nkb, nnb = -(-K // 128), -(-N // 128)
    xs = (2.0 ** rng.integers(-6, 2, size=(nkb, M)) * (1 + rng.random((nkb, M)))).astype(np.float32)
    return xs, (np.exp(0.5 * rng.normal(size=(nnb, nkb))) * 0.01).astype(np.float32)


def check(ops, M, N, K, path, chain, dtype="bf16", spread=0, bias=True, split=True):
    import torch
    p = fp8_plan.plan(M, N, K, dtype, split)
    assert p.path == path and (p.longest if p.splits == 1 and K > 256 else 1) >= chain, p
    say(f"linear_fp8 {dtype} {M} x {N} x {K} {p} spread={spread} bias={bias}")
    x, w = codes_on_gpu(M, K, 31, spread), codes_on_gpu(N, K, 32, spread)
    xs, ws = scales_of(M, N, K, 33)
    b = cuda(gen(34, "bias", (N,), dtype, 3.0)) if bias else None
    out = torch.full((M + 2, N), float("nan"), dtype=torch_dtype(dtype), device="cuda")
    call = lambda y: ops.opscale_linear_fp8(x, cuda(torch.from_numpy(xs)), w, cuda(torch.from_numpy(ws)), b, y=y,  # noqa: E731
                                            workspace=None if split else False)
    y = call(out[1:M + 1])
    again = call(torch.empty_like(y))
    torch.cuda.synchronize()
    assert torch.isnan(out[0]).all() and torch.isnan(out[M + 1]).all(), "rows around y were written"
    assert torch.equal(y, again), "two runs differ"
    # samples, with the corners
    rng = np.random.default_rng(0)
    rows = np.unique(np.r_[0, M - 1, rng.integers(0, M, 10)])
    blocks = np.unique(np.r_[0, ws.shape[0] - 1, rng.integers(0, ws.shape[0], 2)])
    xc = x.view(torch.uint8)[torch.from_numpy(rows).cuda()].cpu().numpy()
    for nb in blocks:
        n = slice(int(nb) * 128, min(N, (int(nb) + 1) * 128))
        want, off = reference(xc, xs[:, rows], w.view(torch.uint8)[n].cpu().numpy(), ws[nb:nb + 1],
                              None if b is None else f64(b[n].cpu()), dtype)
        r = np.abs(f64(y[torch.from_numpy(rows).cuda(), n].cpu()) - want) / off
        assert r.max() <= 1.0, f"{r.max():.3f} of the bound in columns {n}"
    # every element, some rows at a time
    nkb = xs.shape[0]
    value = lambda t, s, axis: t.double() * s  # noqa: E731
    wd = value(w, cuda(torch.from_numpy(ws)).double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K], 0)
    wt, wa = wd.t().contiguous(), wd.abs().t().contiguous()
    for m0 in range(0, M, 2048):
        m = slice(m0, min(M, m0 + 2048))
        xd = value(x[m], cuda(torch.from_numpy(xs)).double().t()[m].repeat_interleave(128, 1)[:, :K], 1)
        want, mass = xd @ wt, xd.abs() @ wa
        if b is not None:
            want, mass = want + b.double(), mass + b.double().abs()
        off = ((2.0 ** -10 if dtype == "bf16" else 0.0) + (80 + 4 + nkb + 65) * U) * mass
        off += (2.0 ** -8 if dtype == "bf16" else U) * (want.abs() + off) + 1e-30
        r = float(((y[m].double() - want).abs() / off).max())
        assert r <= 1.0, f"{r:.3f} of the bound in rows {m}"  # (a NaN fails)
    return y


@pytest.mark.parametrize("K", [16, 128, 144, 256, 272, 384, 4112])
@pytest.mark.parametrize("M,N,path", [(385, 8200, "128x256"), (770, 9352, "256x256"), (300, 392, "128x128")])
def test_tiles(ops, M, N, K, path):
    for spread in (0, 1):
        check(ops, M, N, K, path, 1, spread=spread, split=False)


@pytest.mark.parametrize("M,N,K,path,chain", [
    (300, 152064, 272, "128x256", 2), (300, 152064, 656, "128x256", 2),
    (8200, 12296, 400, "256x256", 2), (8200, 24584, 272, "256x256", 3)])
def test_chained_tiles(ops, M, N, K, path, chain):
    """A workgroup's stores, with the loads of a bias between them, lie behind the next tile's first loads."""
    check(ops, M, N, K, path, chain)
    check(ops, M, N, K, path, chain, bias=False, spread=1)


@pytest.mark.parametrize("M,N,K,path,dtype", [
    (1000, 3080, 12304, "256x256", "bf16"), (200, 10248, 8208, "128x256", "bf16"), (300, 392, 4112, "128x128", "bf16"),
    (300, 392, 4112, "128x128", "f32")])
def test_ranges_of_k(ops, M, N, K, path, dtype):
    assert fp8_plan.plan(M, N, K, dtype).splits > 1
    check(ops, M, N, K, path, 1, dtype)
    check(ops, M, N, K, path, 1, dtype, spread=1)


@pytest.mark.parametrize("M,N,path", [(385, 8200, "128x256"), (770, 9352, "256x256")])
def test_special_values(ops, M, N, path):
    """A NaN element or scale, an infinite scale: in their row or columns of a block, nowhere else."""
    import torch
    K = 304
    assert fp8_plan.plan(M, N, K).path == path
    say(f"linear_fp8 {M} x {N} x {K}: NaN and infinity")
    x, w = codes_on_gpu(M, K, 41, 0), codes_on_gpu(N, K, 42, 0)
    xs, ws = (cuda(torch.from_numpy(a)) for a in scales_of(M, N, K, 43))
    clean = ops.opscale_linear_fp8(x, xs, w, ws)
    x.view(torch.uint8)[M - 1, 290], w.view(torch.uint8)[N - 3, 5] = 0x7f, 0xff
    xs[0, 200] = float("nan")
    y = ops.opscale_linear_fp8(x, xs, w, ws)
    bad = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    bad[M - 1], bad[200], bad[:, N - 3] = True, True, True
    assert torch.equal(torch.isnan(y), bad) and torch.equal(y[~bad], clean[~bad])
    ws[1, 1] = float("inf")
    y = ops.opscale_linear_fp8(x, xs, w, ws)
    bad[:, 128:256] = True
    assert not torch.isfinite(y[:, 128:256]).any() and torch.equal(y[~bad], clean[~bad])


@pytest.mark.parametrize("M,N,K", [(385, 8200, 400), (8200, 12296, 400), (1000, 3080, 12304)])
def test_replayed(ops, M, N, K):
    """Captured once and replayed on other operands, between eager calls."""
    import torch
    say(f"linear_fp8 {M} x {N} x {K}: graph")
    x, w = codes_on_gpu(M, K, 51, 0), codes_on_gpu(N, K, 52, 0)
    xs, ws = (cuda(torch.from_numpy(a)) for a in scales_of(M, N, K, 53))
    b = cuda(gen(54, "bias", (N,), "bf16", 3.0))
    mem = torch.empty(max(16, ops.opscale_linear_fp8_workspace_size(M, N, K)), dtype=torch.uint8, device="cuda")
    y = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    call = lambda: ops.opscale_linear_fp8(x, xs, w, ws, b, y=y, workspace=mem)  # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i in range(3):
        x.view(torch.uint8).copy_(codes_on_gpu(M, K, 60 + i, i & 1).view(torch.uint8))
        xs.mul_(1.5)
        call()
        torch.cuda.synchronize()
        want = y.clone()
        y.zero_()
        mem.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want), i
