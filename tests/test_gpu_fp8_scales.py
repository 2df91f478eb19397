"""GPU linear of e4m3 operands at the ends of its scales' range, on every path.

The two scales of a block are multiplied first, in fp32.  Powers of two change nothing but the
exponent as long as that product, and the result, are normal numbers: results are compared bit by
bit.  Below 2^-126 the product is a multiple of 2^-149; past fp32's range it is an infinity.
"""
import numpy as np
import pytest

import fp8_plan
from parity_util import cuda, say, torch_dtype
from test_gpu_fp8 import ops  # noqa: F401
from test_gpu_fp8_paths import codes_on_gpu

pytestmark = pytest.mark.gpu

K = 304
PATHS = [(3, 264, "few"), (40, 2056, "rows"), (150, 712, "128x128"), (385, 8200, "128x256"), (770, 9352, "256x256")]


def power(e, rows, cols, mantissas=None):
    import torch
    s = torch.full((rows, cols), 2.0 ** e, dtype=torch.float64)
    return cuda((s if mantissas is None else s * mantissas).float())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,path", PATHS)
def test_powers_of_two(ops, dtype, M, N, path):
    import torch
    if dtype == "bf16":
        assert fp8_plan.plan(M, N, K).path == path
    say(f"linear_fp8 {dtype} {M} x {N} x {K}: scales at the ends")
    x, w = codes_on_gpu(M, K, 71, 0), codes_on_gpu(N, K, 72, 0)
    nnb, rng = -(-N // 128), np.random.default_rng(73)
    mx, mw = torch.from_numpy(1 + rng.random((3, M))), torch.from_numpy(1 + rng.random((nnb, 3)))
    run = lambda a, b: ops.opscale_linear_fp8(x, power(a, 3, M, mx), w, power(b, nnb, 3, mw),  # noqa: E731
                                              dtype=torch_dtype(dtype))
    unit = run(0, 0).double()
    assert bool((unit != 0).all())
    for a, b in ((126, -26), (-30, 126), (-126, 26), (40, -126), (-100, 0), (120, -40)):
        assert torch.equal(run(a, b).double(), unit * 2.0 ** (a + b)), (a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,path", PATHS)
def test_ends_of_the_product(ops, dtype, M, N, path):
    """The largest scale that opscale_quantize_fp8 gives, and W's that bring the product to the ends of fp32's
    range and past them."""
    import torch
    nnb, dt = -(-N // 128), torch_dtype(dtype)
    say(f"linear_fp8 {dtype} {M} x {N} x {K}: products of scales at the ends")
    # one element a row: 2^-9, and (every fifth row) none, in the first block; W's elements +-64 to 448
    x = torch.zeros(M, K, dtype=torch.uint8, device="cuda")
    m = torch.arange(M, device="cuda")
    at = m * 7 % 128
    x[m, at] = torch.where(m % 5 == 4, 0, 1).to(torch.uint8)
    w = torch.randint(0x68, 0x7f, (N, K), dtype=torch.uint8, device="cuda") | (torch.arange(N, device="cuda") % 2 * 128)[:, None].to(torch.uint8)
    x, w = x.view(torch.float8_e4m3fn), w.view(torch.float8_e4m3fn)
    p = (x.double() @ w.double().t().contiguous())  # each one product, at most 0.875
    run = lambda a, b, c=None: ops.opscale_linear_fp8(  # noqa: E731
        x, torch.cat([power(a, 1, M), power(a if c is None else c, 2, M)]), w, power(b, nnb, 3), dtype=dt)
    assert torch.equal(run(120, 7).double(), p * 2.0 ** 127)
    assert torch.equal(run(-100, -20).double(), p * 2.0 ** -120)
    # past the range: as an infinite scale, in each block (the second and third of every row sum to 0)
    assert bool(torch.isnan(run(120, 8)).all())
    y = run(120, 8, 0)
    assert torch.equal(torch.isnan(y), p == 0) and torch.equal(torch.isinf(y), p != 0)
    assert torch.equal(torch.sign(y.double().nan_to_num(0.0)), torch.sign(p))
    # below 2^-126: whole multiples of 2^-149, which stay (W's elements and x's are whole numbers here)
    ones = torch.where(x.view(torch.uint8) != 0, 0x38, 0).to(torch.uint8).view(torch.float8_e4m3fn)
    q = ones.double() @ w.double().t().contiguous()
    y = ops.opscale_linear_fp8(ones, power(-100, 3, M), w, power(-45, nnb, 3), dtype=torch.float32)
    assert torch.equal(y.double(), q * 2.0 ** -145)
