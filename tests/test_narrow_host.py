"""Host-side checks, without a GPU, of the entry points of 8 and 4 bits: every refusal before
anything is enqueued, workspaces, and the descriptors' layout."""
import ctypes
import os
import shutil
import subprocess

import pytest

from test_step_host import BAD_MODS, _mods

G = 1 << 38  # fake addresses spaced far apart (never dereferenced)
NAN = float("nan")


@pytest.fixture(scope="module")
def lib():
    import paper_2608_13499_amd as ops
    return ops.load()


def _err(lib):
    return lib.opscale_last_error().decode()


def caller(lib, name, good):
    def call(**kw):
        a = dict(good, **kw)
        return getattr(lib, "opscale_" + name)(*(a[n] for n in good), None, None)

    return call


def refused(lib, name, call, status, cases):
    for bad in cases:
        assert call(**bad) == status, (bad, _err(lib))
        assert name in _err(lib) or name == "attn_decode_fp4", _err(lib)


def test_quantize_fp8(lib):
    call = caller(lib, "quantize_fp8", dict(x=G, xs=4096, q=2 * G, s=3 * G, M=256, K=4096, dt=1))
    refused(lib, "quantize_fp8", call, 1, (
        dict(dt=2), dict(M=-1), dict(M=1 << 31), dict(K=0), dict(K=4088), dict(K=(1 << 20) + 16), dict(xs=4080),
        dict(xs=4100), dict(x=None), dict(q=None), dict(s=None), dict(x=G + 8), dict(q=2 * G + 4), dict(s=3 * G + 2),
        dict(q=G), dict(s=G + 256), dict(s=2 * G + 16), dict(M=(1 << 31) - 1, K=1 << 20, xs=1 << 20),
        dict(M=1 << 28, K=16, xs=16)))
    assert call(M=0) == 0 and call(M=0, x=None, q=None, s=None) == 0


def test_linear_fp8(lib):
    good = dict(x=G, xs=2 * G, W=3 * G, ws=4 * G, bias=5 * G, y=6 * G, M=256, N=512, K=4096, dt=1, work=7 * G, wb=1 << 30)
    call = caller(lib, "linear_fp8", good)
    refused(lib, "linear_fp8", call, 1, (
        dict(dt=-1), dict(M=-1), dict(M=1 << 30), dict(N=0), dict(N=(1 << 24) + 8), dict(K=0), dict(K=4104),
        dict(K=(1 << 20) + 16), dict(N=508), dict(dt=0, N=510), dict(M=1 << 25, N=1 << 16), dict(x=None), dict(xs=None),
        dict(W=None), dict(ws=None), dict(y=None), dict(x=G + 8), dict(W=3 * G + 1), dict(y=6 * G + 8),
        dict(bias=5 * G + 2), dict(xs=2 * G + 1), dict(ws=4 * G + 2), dict(y=G), dict(y=2 * G + 64), dict(y=3 * G),
        dict(y=4 * G), dict(y=5 * G)))
    # the workspace, where K is split
    need = lib.opscale_linear_fp8_workspace_size(256, 512, 4096, 1)
    assert need >= 2 * 256 * 512 * 4 and need % (256 * 512 * 4) == 0
    assert call(wb=need - 1) == 3 and "linear_fp8" in _err(lib)
    refused(lib, "linear_fp8", call, 1, (dict(work=7 * G + 4), dict(work=6 * G + 16), dict(work=G), dict(work=2 * G),
                                         dict(work=3 * G), dict(work=4 * G), dict(work=5 * G)))
    assert call(M=0) == 0
    size = lib.opscale_linear_fp8_workspace_size
    assert size(0, 512, 4096, 1) == size(5, 512, 128, 1) == size(9000, 8192, 8192, 1) == size(5, 5, 4096, 7) == 0
    assert size(256, 512, 4096, 0) == need
    # every size has splits that its partials fit, few enough for their sums' order to be short
    for M in (1, 16, 48, 128, 129, 300, 1023):
        for N in (8, 256, 6144, 57344):
            for K in (16, 688, 4096, 28672, 1 << 20):
                ws = size(M, N, K, 1)
                assert ws % (M * N * 4) == 0 and ws // (M * N * 4) <= 512 and ws // (M * N * 4) != 1


CACHE = dict(kc=3 * G, vc=4 * G)


def test_kv_write_fp4(lib):
    good = dict(k=G, v=G + 2048, kvs=6144, **CACHE, slots=5 * G, T=64, Hkv=8, D=128, bs=16, nb=512, dt=1)
    call = caller(lib, "kv_write_fp4", good)
    refused(lib, "kv_write_fp4", call, 1, (
        dict(dt=5), dict(T=-1), dict(T=1 << 28), dict(Hkv=0), dict(Hkv=1 << 14), dict(D=0), dict(bs=8), dict(bs=48),
        dict(bs=2048), dict(nb=0), dict(nb=1 << 27), dict(kvs=1016), dict(kvs=6148), dict(k=None), dict(v=None),
        dict(kc=None), dict(vc=None), dict(slots=None), dict(k=G + 2), dict(v=G + 4), dict(kc=3 * G + 8),
        dict(vc=4 * G + 1), dict(slots=5 * G + 2), dict(kc=G), dict(vc=G + 2048), dict(kc=4 * G), dict(vc=5 * G)))
    refused(lib, "kv_write_fp4", call, 2, (dict(D=96), dict(D=32), dict(D=256)))
    assert call(T=0) == 0


def test_kv_read_fp4(lib):
    good = dict(**CACHE, tab=5 * G, cu=6 * G, first=7 * G, k=G, v=G + 2048, kvs=2048, B=4, T=64, Hkv=8, D=128, bs=16, mb=64,
                nb=512, dt=1)
    call = caller(lib, "kv_read_fp4", good)
    refused(lib, "kv_read_fp4", call, 1, (
        dict(dt=5), dict(B=-1), dict(T=-1), dict(T=1 << 28), dict(Hkv=-2), dict(bs=4), dict(bs=24), dict(mb=0), dict(nb=0),
        dict(nb=(1 << 32) + 1), dict(kvs=1000), dict(kvs=2052), dict(kc=None), dict(vc=None), dict(tab=None),
        dict(cu=None), dict(k=None), dict(v=None), dict(k=G + 8), dict(v=G + 4), dict(tab=5 * G + 1), dict(cu=6 * G + 2),
        dict(first=7 * G + 3), dict(v=G), dict(v=G + 2032), dict(k=3 * G), dict(v=4 * G), dict(k=5 * G), dict(v=6 * G),
        dict(k=7 * G), dict(v=G + 4096 - 16)))
    refused(lib, "kv_read_fp4", call, 2, (dict(D=96),))
    assert call(T=0) == 0 and call(B=0) == 0


def test_attn_decode_fp4(lib):
    good = dict(q=G, qs=32 * 128, kc=2 * G, vc=3 * G, tab=4 * G, ctx=5 * G, o=6 * G, B=256, Hq=32, Hkv=8, D=128, bs=16,
                mb=512, nb=69424, mc=8192, scale=0.08, mods=None, dt=1, ws=7 * G, wsb=1 << 30)
    call = caller(lib, "attn_decode_fp4", good)
    refused(lib, "attn_decode_fp4", call, 1, (
        dict(bs=8), dict(bs=1), dict(bs=12), dict(bs=2048), dict(tab=None), dict(mb=0), dict(qs=32 * 128 - 8),
        dict(Hkv=5), dict(Hkv=0), dict(B=-1), dict(mc=0), dict(dt=9), dict(scale=NAN), dict(scale=-1.0), dict(nb=1 << 40),
        dict(q=G + 4), dict(o=G), dict(o=2 * G), dict(o=3 * G + 256), dict(o=4 * G), dict(o=5 * G), dict(ws=6 * G + 16),
        dict(ws=G), dict(ws=2 * G), dict(mods=_mods(slopes=6 * G)), dict(mods=_mods(prefix=7 * G)),
        dict(mods=_mods(starts=6 * G + 4)), dict(bs=1024, nb=(1 << 26) + 1, ws=1 << 62, o=1 << 61)))
    for bad in BAD_MODS:
        assert call(mods=_mods(**bad)) == 1, bad
        assert "attn_decode_fp4" in _err(lib)
    # a cache's bytes: o right behind it is free, its last row is not
    end = 2 * G + 69424 * 8 * 16 * 68
    assert call(o=end - 16) == 1 and "attn_decode_fp4" in _err(lib)
    need = lib.opscale_attn_decode_fp4_workspace_size(256, 32, 128, 8192)
    assert need == lib.opscale_attn_decode_mod_workspace_size(256, 32, 128, 8192)
    assert call(wsb=need - 1) == 3 and call(ws=None) == 3 and call(ws=7 * G + 8) == 3
    assert call(D=96) == 2 and call(D=256) == 2
    assert call(B=0) == 0


def test_descriptor_layouts(tmp_path):
    """The descriptors' fields lie where the header puts them."""
    if shutil.which("gcc") is None:
        pytest.skip("gcc not available")
    import paper_2608_13499_amd as ops
    L = ops._lib
    members = {"quantize_fp8": L._QuantizeFp8Args, "linear_fp8": L._LinearFp8Args, "kv_write_fp4": L._CacheWriteArgs,
               "kv_read_fp4": L._KvReadFp4Args, "attn_decode_fp4": L._DecodeModArgs}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "opscale.h"', "int main(void) {",
             'printf("desc %zu\\n", sizeof(opscale_op_desc));', 'printf("last %d\\n", (int)OPSCALE_OP_ATTN_DECODE_FP4);']
    for m, cls in members.items():
        lines += [f'printf("{m}.{f} %zu\\n", offsetof(opscale_op_desc, u.{m}.{f}) - offsetof(opscale_op_desc, u));'
                  for f, _ in cls._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["return 0; }"]))
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    r = subprocess.run(["gcc", "-I", include, "-I", "/opt/rocm/include", "-D__HIP_PLATFORM_AMD__", str(src), "-o", str(exe)],
                       capture_output=True, text=True)
    if r.returncode != 0:
        pytest.skip("cannot compile against the HIP headers here: " + r.stderr[-200:])
    out = dict(line.split() for line in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    assert int(out.pop("desc")) == ctypes.sizeof(L.OpDesc) and int(out.pop("last")) == L.OP_ATTN_DECODE_FP4
    assert {n: int(at) for n, at in out.items()} == {f"{m}.{f}": getattr(cls, f).offset for m, cls in members.items()
                                                     for f, _ in cls._fields_}


def test_profile_refusals(lib):
    import paper_2608_13499_amd as ops
    L, out = ops._lib, ops.Profile()
    for op in range(L.OP_QUANTIZE_FP8, L.OP_ATTN_DECODE_FP4 + 2):
        for dt in (0, 1):
            desc = ops.OpDesc(op=op, dt=dt)
            assert lib.opscale_op_profile(ctypes.byref(desc), 1, 1, None, 0, None, ctypes.byref(out)) == 1, op
