"""The rotation of the heads in fp32, element by element: sine and cosine, with the
magnitude, are rounded once each from 64 bits."""
import numpy as np
import pytest

from oracle import step
from parity_util import cuda, f64, gen, say
from test_gpu_step import i32, ops  # noqa: F401

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("scaling", ["none", "bands", "ramp"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D,rot,maxpos", [(128, 128, 131072), (64, 32, 40), (256, 256, 1 << 30)])
def test_rotation(ops, scaling, inter, D, rot, maxpos):
    """(a c - b s): half a step of each of c and s, of the two products and of the sum."""
    import torch
    T, H = 700, 4
    say(f"qk_norm_rope f32 D={D} rot={rot} {scaling} inter={inter} positions below {maxpos}")
    freq, mag = ops.opscale_rope_frequencies(rot, 10000.0, scaling, 16.0, 1.0, 32.0, 4096)
    x, y = gen(98, "q", (T, H, D), "f32"), gen(98, "k", (T, H, D), "f32")
    pos = np.random.default_rng(98).integers(0, maxpos, T).astype(np.int32)
    got, _ = ops.opscale_qk_norm_rope(cuda(x), cuda(y), i32(pos), freq, interleaved=inter, magnitude=mag)
    torch.cuda.synchronize()
    f = freq.cpu().numpy()
    want = step.qk_norm_rope(f64(x), None, 0.0, pos, f, inter, float(np.float32(mag)))
    a, b = (f64(x)[..., :rot:2], f64(x)[..., 1:rot:2]) if inter else (f64(x)[..., :rot // 2], f64(x)[..., rot // 2:rot])
    c, s = (float(np.float32(mag)) * np.abs(g(pos[:, None] * f))[:, None] for g in (np.cos, np.sin))
    bound = np.zeros_like(want)
    at = (slice(0, rot, 2), slice(1, rot, 2)) if inter else (slice(0, rot // 2), slice(rot // 2, rot))
    # (an angle in 64 bits is off by half a step of its own, 2^-53 of it)
    angle = 2.0 ** -52 * np.abs(pos[:, None] * f)[:, None] * mag * (np.abs(a) + np.abs(b))
    bound[..., at[0]] = 2 * U * (np.abs(a) * c + np.abs(b) * s) + angle
    bound[..., at[1]] = 2 * U * (np.abs(b) * c + np.abs(a) * s) + angle
    bound += U * np.abs(want)
    r = np.abs(f64(got.cpu()) - want)[..., :rot] / bound[..., :rot]
    say(f"  {r.max():.3f} of the bound")
    assert r.max() <= 1.0
    np.testing.assert_array_equal(f64(got.cpu())[..., rot:], f64(x)[..., rot:])
