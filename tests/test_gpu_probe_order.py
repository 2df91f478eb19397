"""The placement probe on a masked stream writes its output after the current stream's work on it."""
import pytest

pytestmark = pytest.mark.gpu


def test_probe_runs_behind_the_fill():
    import torch
    import paper_2608_13499_amd as ops
    ops.load()
    n, x, il = ops.opscale_cu_layout()
    a = torch.ones(4096, 4096, device="cuda")
    out = torch.empty(1024, 2, dtype=torch.int32, device="cuda")
    s = ops.opscale_cu_stream_create(ops.opscale_cu_mask_build(n, x, il, 0, 64))
    try:
        for _ in range(3):
            for _ in range(20):  # some milliseconds before the fill
                a @ a
            out.fill_(-1)
            ops.opscale_cu_probe(out, 2, stream=s)
            torch.cuda.synchronize()
            assert int((out[:, 0] == -1).sum()) == 0
    finally:
        ops.opscale_cu_stream_destroy(s)
