"""Pins of oracle/narrow.py: values worked by hand, torch's own float8 type, and
invariants; each with a planted mistake that it catches."""
import math

import numpy as np
import pytest

from oracle import narrow


def test_values_by_hand():
    assert narrow.E2M1.tolist() == [0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6]
    e = narrow.E4M3
    # smallest, largest below normal, smallest normal, 1, 1.125, largest
    assert [e[1], e[7], e[8], e[0x38], e[0x39], e[0x7e]] == [2.0 ** -9, 7 * 2.0 ** -9, 2.0 ** -6, 1, 1.125, 448]
    assert math.isnan(e[0x7f]) and math.isnan(e[0xff]) and e[0xfe] == -448


def test_e4m3_is_torchs():
    torch = pytest.importorskip("torch")
    bits = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(bits.view(torch.float8_e4m3fn).double().numpy(), narrow.E4M3, equal_nan=True)
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.normal(size=4000) * 2.0 ** rng.integers(-12, 8, 4000), narrow.E4M3[:127],
                        0.5 * (narrow.E4M3[:126] + narrow.E4M3[1:127])])
    x = np.clip(x.astype(np.float32), -448, 448)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(narrow.encode(x, "e4m3"), want)
    assert not np.array_equal(narrow.encode(np.nextafter(x, 0) * (1 - 2.0 ** -5), "e4m3"), want)


def test_ties_go_to_the_even_code():
    ties = [.25, .75, 1.25, 1.75, 2.5, 3.5, 5.0]
    assert narrow.E2M1[narrow.encode(ties, "e2m1")].tolist() == [0, 1, 1, 2, 2, 4, 4]
    up = np.nextafter(ties, 9)
    assert narrow.E2M1[narrow.encode(up, "e2m1")].tolist() == [.5, 1, 1.5, 2, 3, 4, 6]
    assert narrow.E2M1[narrow.encode([7.9, -7.9, -0.2], "e2m1")].tolist() == [6, -6, 0]


@pytest.mark.parametrize("kind", ["e4m3", "e2m1"])
def test_exponents(kind):
    most = narrow.MOST[kind]
    for e in (-99, -3, 0, 1, 77):
        assert narrow.exponent(most * 2.0 ** e, kind) == e
        assert narrow.exponent(np.nextafter(most * 2.0 ** e, np.inf), kind) == e + 1
    assert narrow.exponent(0.0, kind) == -100 and narrow.exponent(1e-45, kind) == -100
    assert narrow.exponent(3.4028234663852886e38, kind) <= narrow.HIGHEST[kind]


def test_blocks_are_their_own():
    rng = np.random.default_rng(1)
    x = rng.normal(size=(2, 128 + 48))
    x[1, 130] = np.inf
    v, s = narrow.quantize_fp8(x)
    assert s.shape == (2, 2) and np.isnan(s).tolist() == [[False, False], [False, True]]
    back = v * np.repeat(s.T, 128, 1)[:, :176]
    assert np.abs(back - x)[0].max() <= 2.0 ** -4 * np.abs(x[0]).max()
    assert (np.abs(back - x)[0] <= 2.0 ** -4 * np.abs(x[0]) + 2.0 ** -10 * s[:, 0].max()).all()
    x[0, :128] *= 2.0 ** 20  # one block's size leaves the other's codes alone
    v2, s2 = narrow.quantize_fp8(x)
    assert np.array_equal(v2[0, 128:], v[0, 128:]) and s2[0, 0] == 2.0 ** 20 * s[0, 0] and np.array_equal(v2[0], v[0])


def test_linear_by_hand():
    """Two tokens, one output in each of two blocks of W's rows, K of 130."""
    x, w = np.zeros((2, 130)), np.zeros((129, 130))
    x[0, [0, 129]], x[1, [127, 128]] = [2, 3], [5, 7]
    w[0, [0, 129]], w[128, [127, 128]] = [1, 4], [10, 100]
    xs, ws = np.array([[1.0, 0.5], [2.0, 4.0]]), np.array([[1.0, 10.0], [0.1, 0.01]])
    y = narrow.linear_fp8(x, xs, w, ws)
    assert y[0, 0] == 2 * 1 + 3 * 4 * 2 * 10 and np.isclose(y[1, 128], 50 * 0.5 * 0.1 + 700 * 4 * 0.01)
    assert np.count_nonzero(y) == 2
    assert np.array_equal(narrow.linear_fp8(x, xs, w, ws, np.ones(129)), y + 1)


def test_pages():
    rng = np.random.default_rng(2)
    x = rng.normal(size=(2, 16, 3, 64)) * 2.0 ** rng.integers(-6, 6, size=(2, 16, 3, 1))
    x[1, 3, 2, 40] = np.nan
    pages = narrow.pack(x)
    assert pages.shape == (2, 3, 16, 34) and pages.dtype == np.uint8
    assert np.array_equal(narrow.unpack(pages), narrow.cached(x), equal_nan=True)
    # element 1 of row 2 of page 0, head 1: the high half of byte 0 of the row; its group's scale byte
    flat = pages.reshape(2, 3, -1)[0, 1]
    e = int(flat[16 * 32 + 0 * 16 + 2]) - 127
    assert narrow.E2M1[flat[2 * 32] >> 4] * 2.0 ** e == narrow.cached(x)[0, 2, 1, 1]
    assert np.isnan(narrow.cached(x)[1, 3, 2, 32:]).all() and np.isfinite(narrow.cached(x)[1, 3, 2, :32]).all()
    # half a step of each element's size, a step of the smallest ones
    ok = np.isfinite(x) & np.isfinite(narrow.cached(x))
    scale = np.repeat(np.abs(x.reshape(2, 16, 3, 2, 32)).max(-1), 32, -1)
    assert (np.abs(narrow.cached(x) - x)[ok] <= (0.25 * np.abs(x) + scale / 12)[ok]).all()
