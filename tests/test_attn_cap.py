"""The cap of attention scores as the kernels evaluate it (csrc/attn_cap.h), compiled for
the host and stepped through in fp32 as attn_mods.h does."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_13499_amd", "csrc")
CXX = shutil.which("g++") or shutil.which("c++")
U = 2.0 ** -24
LOG2E = 1.4426950408889634
f32 = np.float32

pytestmark = pytest.mark.skipif(CXX is None, reason="no host C++ compiler")


class Terms(ctypes.Structure):
    _fields_ = [("softcap", ctypes.c_float), ("cap_log2", ctypes.c_float), ("cap_rate", ctypes.c_float),
                ("cap_bound", ctypes.c_float), ("poly", ctypes.c_float * 4), ("near", ctypes.c_float * 3),
                ("floor", ctypes.c_float)]


@pytest.fixture(scope="module")
def terms(tmp_path_factory):
    d = tmp_path_factory.mktemp("cap")
    src, so = str(d / "cap.cpp"), str(d / "cap.so")
    with open(src, "w") as f:
        f.write('#include "attn_cap.h"\nextern "C" {\nvoid cap(double c, double s, opscale::CapTerms* t) '
                '{ *t = opscale::cap_terms(c, s); }\n'
                'const double* half() { return opscale::kTanhHalf; }\n'
                'const double* quarter() { return opscale::kTanhQuarter; }\n}\n')
    subprocess.run([CXX, "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{CSRC}", src, "-o", so], check=True)
    lib = ctypes.CDLL(so)
    lib.cap.argtypes = [ctypes.c_double, ctypes.c_double, ctypes.POINTER(Terms)]
    lib.cap.restype = None
    lib.half.restype = lib.quarter.restype = ctypes.POINTER(ctypes.c_double)

    def call(cap, scale):
        t = Terms()
        lib.cap(float(f32(cap)), float(f32(scale)), ctypes.byref(t))
        return t

    call.lib = lib
    return call


def _horner(x, c):
    u = x * x
    p = f32(c[-1])
    for k in reversed(c[:-1]):
        p = f32(np.float64(u) * p + f32(k))  # (a fused step: rounded once)
    return x * p


def forms(t, x):
    """The three forms of the capped score, in log2 units."""
    with np.errstate(over="ignore", invalid="ignore"):
        e = np.exp2(x * f32(t.cap_rate))
        far = f32(-2) * f32(t.cap_log2) * (f32(1) / (f32(1) + e)) + f32(t.cap_log2)
        return _horner(x, list(t.near)), _horner(x, list(t.poly)), far


def chosen(t, x):
    near, half, far = forms(t, x)
    a = np.abs(x)
    return np.where(a <= f32(0.5) * f32(t.cap_bound), near, np.where(a <= f32(t.cap_bound), half, far))


SCALES = [2.0 ** -100, 2.0 ** -40, 2.0 ** -10, 0.08838834764, 0.125, 1.0, 2.0 ** 20, 2.0 ** 60]
CAPS = [1e-44, 1e-30, 1e-12, 1e-9, 1e-8, 1.4e-8, 1e-6, 1e-3, 0.5, 5.0, 15.0, 30.0, 50.0, 52.0, 1e3, 1e5, 1e6, 1e8, 1e10,
        1e12, 1e15, 1e20, 1e30, 3e38]


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("cap", CAPS)
def test_any_cap_of_any_score(terms, scale, cap):
    """The form that a lane takes, and each form that it may be computed beside, is a number;
    the score is right to some steps of itself within the polynomials' reach and of the
    cap past it.  Where there is no cap left, that of a score of 2^28 raw units is not felt."""
    t = terms(cap, scale)
    if not t.softcap > 0:
        x = 2.0 ** 28 * scale
        assert abs(cap * np.tanh(x / cap) - x) <= 4 * U * x
        return
    x = np.unique(np.concatenate([[0.0], 2.0 ** np.arange(-60, 60, 0.37), np.arange(0.0, 2.1, 0.01) / (scale / cap)]))
    x = f32(x[x < 2.0 ** 60])
    x = np.concatenate([-x[::-1], x])
    got, (_, _, far) = np.float64(chosen(t, x)), forms(t, x)
    assert np.isfinite(got).all() and np.isfinite(far).all()
    z = np.float64(x) * (float(f32(scale)) / float(f32(cap)))
    want = float(f32(cap)) * LOG2E * np.tanh(z)
    inside = np.abs(np.float64(x)) <= t.cap_bound
    # polynomials: 5.45e-7 (9.2 steps) and their terms' roundings; past them the roundings of
    # e, 1 + e, its reciprocal and the last sum, each a step of the cap or two
    tol = np.where(inside, 14 * U * np.abs(want), 8 * U * float(t.cap_log2)) + 2.0 ** -140
    worst = np.abs(got - want) / tol
    assert worst.max() <= 1.0, (float(worst.max()), float(x[worst.argmax()]), float(z[worst.argmax()]))


@pytest.mark.parametrize("name,n,reach,error", [("half", 4, 0.5, 5.45e-7), ("quarter", 3, 0.25, 3.96e-7)])
def test_polynomials(terms, name, n, reach, error):
    """Their stated errors; and as these are the least possible, they are reached n + 1 times,
    with alternating signs."""
    c = getattr(terms.lib, name)()[:n]
    y = np.linspace(1e-6, reach, 400001)
    e = sum(k * y ** (2 * i) for i, k in enumerate(c)) / (np.tanh(y) / y) - 1
    assert 0.99 * error < np.abs(e).max() <= 1.001 * error
    signs = np.sign(e[np.abs(e) > 0.99 * np.abs(e).max()])
    assert 1 + int((np.diff(signs) != 0).sum()) == n + 1
