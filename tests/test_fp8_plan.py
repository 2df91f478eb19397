"""What the linear of e4m3 operands plans, over the whole range of sizes."""
import itertools

import pytest

import fp8_plan

pytestmark = pytest.mark.skipif(fp8_plan.CXX is None, reason="no host C++ compiler")

SIZES = list(itertools.product([1, 5, 16, 48, 128, 129, 200, 256, 300, 512, 770, 1023, 2048, 8871, 70000],
                               [8, 136, 256, 688, 2816, 4096, 6144, 12296, 28672, 57344, 152064],
                               [16, 128, 272, 400, 688, 2064, 4096, 14336, 28672, 1 << 20]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("split", [True, False])
def test_ranges_of_k(dtype, split):
    """The ranges hold each block of K once and none is empty; the workspace holds their sums."""
    for M, N, K in SIZES:
        p, nkb = fp8_plan.plan(M, N, K, dtype, split), -(-K // 128)
        assert p.splits >= 1 and (p.splits - 1) * p.chunk < nkb <= p.splits * p.chunk, (M, N, K, p)
        assert p.ws_bytes == (4 * p.splits * M * N if p.splits > 1 else 0), (M, N, K, p)
        assert split or p.splits == 1
        assert dtype == "bf16" or p.path not in ("256x256", "128x256"), (M, N, K, p)
        assert (p.path == "rows") == (5 <= p.waves <= 8), (M, N, K, p)


def test_the_library_plans_the_same():
    import paper_2608_13499_amd as ops
    size = ops.load().opscale_linear_fp8_workspace_size
    for M, N, K in SIZES:
        for dt, dtype in ((1, "bf16"), (0, "f32")):
            assert size(M, N, K, dt) == fp8_plan.plan(M, N, K, dtype).ws_bytes, (M, N, K, dtype)


def test_ranges_of_k_are_not_chained():
    """Tiles whose K is in ranges are two rounds of the CUs at most, which a chained launch would not
    join either: the stores of partial sums lie before no other item's loads."""
    some = 0
    for M, N, K in SIZES:
        p = fp8_plan.plan(M, N, K)
        if p.path in fp8_plan.TILES and p.splits > 1:
            some += 1
            assert p.items <= 512 and p.longest == 1, (M, N, K, p)
    assert some > 20
