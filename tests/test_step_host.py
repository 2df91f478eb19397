"""Host-side checks, without a GPU, of the attention path's further entry points:
the rotation's frequencies, and every refusal before anything is enqueued."""
import ctypes
import math
import os

import numpy as np
import pytest

from oracle import step

G = 1 << 36  # fake addresses spaced far apart (never dereferenced)
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    import paper_2608_13499_amd as ops
    return ops.load()


def _err(lib):
    return lib.opscale_last_error().decode()


# ------------------------------------------------------------ frequencies ---
@pytest.mark.parametrize("scaling", ["none", "linear", "bands", "ramp"])
@pytest.mark.parametrize("rot,theta,factor,low,high,orig", [
    (128, 500000.0, 8.0, 1.0, 4.0, 8192), (64, 10000.0, 16.0, 1.0, 32.0, 4096), (2, 10000.0, 2.0, 0.5, 1.0, 1),
    (32, 1e6, 1.0, 1.0, 32.0, 32768), (256, 10000.0, 40.0, 1.0, 32.0, 4096)])
def test_frequencies(scaling, rot, theta, factor, low, high, orig):
    import paper_2608_13499_amd as ops
    f, m = ops.opscale_rope_frequencies(rot, theta, scaling, factor, low, high, orig, device="cpu")
    rf, rm = step.rope_frequencies(rot, theta, scaling, factor, low, high, orig)
    # a power, a few products and sums in 64 bits; the turns' difference loses at most
    # high / (high - low) <= 2 of it
    np.testing.assert_allclose(f.numpy(), rf, rtol=1e-13)
    assert math.isclose(m, rm, rel_tol=2 ** -24)


def test_frequencies_refusals(lib):
    import paper_2608_13499_amd as ops
    f, m = (ctypes.c_double * 128)(), ctypes.c_float()

    def call(rot=128, theta=1e4, scaling=2, factor=8.0, low=1.0, high=4.0, orig=8192, out=f):
        return lib.opscale_rope_frequencies(out, ctypes.byref(m), rot, theta, scaling, factor, low, high, orig)

    assert call() == 0
    for bad in (dict(rot=0), dict(rot=7), dict(rot=258), dict(theta=1.0), dict(theta=NAN), dict(theta=INF),
                dict(scaling=4), dict(scaling=-1), dict(factor=0.5), dict(factor=NAN), dict(low=0.0), dict(high=1.0),
                dict(high=INF), dict(high=NAN), dict(orig=0), dict(out=None)):
        assert call(**bad) == 1, bad
        assert "rope_frequencies" in _err(lib)
    assert call(scaling=0, factor=0.0, low=9.0, high=0.0, orig=0) == 0  # (not used)
    with pytest.raises(ops.OpscaleError):
        ops.opscale_rope_frequencies(64, 1e4, "other", device="cpu")


# ----------------------------------------------------------- qk_norm_rope ---
QK = dict(q=G, k=G + 32 * 256, qs=48 * 128, ks=48 * 128, qo=G, ko=G + 32 * 256, qos=48 * 128, kos=48 * 128, wq=2 * G,
          wk=3 * G, eps=1e-6, pos=4 * G, freq=5 * G, rot=128, inter=0, mag=1.0, v=G + 40 * 256, vs=48 * 128, kc=6 * G,
          vc=7 * G, slots=8 * G, bs=16, nb=100, T=1000, Hq=32, Hkv=8, D=128, dt=1)


def _qk(lib, **kw):
    a = dict(QK, **kw)
    return lib.opscale_qk_norm_rope(*(a[n] for n in QK), None, None)


def test_qk_norm_rope_refusals(lib):
    for bad in (dict(dt=2), dict(T=-1), dict(T=1 << 31), dict(Hq=0), dict(Hkv=0), dict(Hq=70000), dict(D=0),
                dict(rot=-16), dict(rot=144), dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(mag=NAN),
                dict(wq=None), dict(kc=None), dict(bs=0), dict(nb=0), dict(nb=1 << 40), dict(bs=1 << 20, nb=1 << 20),
                dict(qs=100), dict(qs=48 * 128 + 4), dict(ks=512), dict(vs=512), dict(qs=1 << 25), dict(qos=64),
                dict(q=None), dict(ko=None), dict(pos=None), dict(freq=None), dict(v=None), dict(slots=None),
                dict(q=G + 8), dict(wk=3 * G + 4), dict(kc=6 * G + 2), dict(pos=4 * G + 2), dict(freq=5 * G + 4),
                dict(slots=8 * G + 1)):
        assert _qk(lib, **bad) == 1, bad
        assert "qk_norm_rope" in _err(lib)
    for bad in (dict(D=40), dict(D=16), dict(D=272), dict(rot=24)):
        assert _qk(lib, **bad) == 2, bad
    assert _qk(lib, T=0) == 0
    assert _qk(lib, T=0, q=None, k=None, wq=None, wk=None, kc=None, vc=None, rot=0) == 0


def test_qk_norm_rope_overlaps(lib):
    """Views of one packed tensor lie side by side; anything else that an output
    could share a byte with is refused."""
    overlap = (
        dict(qo=G + 16), dict(qo=G + 256, qos=48 * 128),                # shifted against its own input
        dict(qo=G, qos=32 * 128),                                       # the same start, another stride
        dict(qo=G + 32 * 256),                                          # on k
        dict(ko=G + 31 * 256), dict(ko=G + 39 * 256),                   # on q's last head; one head on v
        dict(qo=9 * G, ko=9 * G + 24 * 256, qos=48 * 128, kos=48 * 128),  # each other
        dict(kc=G + 1600), dict(vc=G), dict(vc=6 * G), dict(vc=6 * G + 100 * 16 * 8 * 256 - 16),
        dict(kc=2 * G), dict(vc=8 * G), dict(kc=4 * G), dict(vc=5 * G),
        dict(wq=G), dict(pos=G + 64), dict(slots=G + 64), dict(freq=G + 64))
    for bad in overlap:
        assert _qk(lib, **bad) == 1, bad
        assert "overlap" in _err(lib), bad


# ----------------------------------------------------------- block_tables ---
BT = dict(ctx=G, new=2 * G, B=100, table=3 * G, mb=64, bs=16, free=4 * G, nf=1000, begin=5 * G, mt=4096, cu=6 * G,
          pos=7 * G, slots=8 * G, kv=9 * G, next=10 * G)


def _bt(lib, **kw):
    a = dict(BT, **kw)
    return lib.opscale_block_tables(*(a[n] for n in BT), None, None)


def test_block_tables_refusals(lib):
    for bad in (dict(B=-1), dict(bs=0), dict(bs=24), dict(bs=2048), dict(mb=0), dict(mb=1 << 30), dict(nf=-1),
                dict(nf=1 << 31), dict(mt=-1), dict(mt=1 << 31), dict(ctx=None), dict(new=None), dict(table=None),
                dict(free=None), dict(begin=None), dict(cu=None), dict(pos=None), dict(slots=None), dict(kv=None),
                dict(next=None), dict(ctx=G + 2), dict(slots=8 * G + 1),
                dict(next=5 * G), dict(kv=G + 396), dict(cu=2 * G + 396), dict(table=4 * G), dict(pos=8 * G + 4),
                dict(kv=6 * G + 400), dict(slots=3 * G + 100)):
        assert _bt(lib, **bad) == 1, bad
        assert "block_tables" in _err(lib)


# ----------------------------------------------- attention with modifiers ---
PF = dict(q=G, k=2 * G, v=3 * G, qs=32 * 128, kvs=8 * 128, o=4 * G, cu=5 * G, B=2, T=100, ms=64, Hq=32, Hkv=8, D=128,
          scale=0.08, causal=1, mods=None, dt=1)


def _mods(softcap=0.0, window=0, slopes=None, prefix=None, starts=None):
    import paper_2608_13499_amd as ops
    return ctypes.byref(ops.AttnMods(softcap, window, slopes, prefix, starts))


BAD_MODS = (dict(softcap=-1.0), dict(softcap=NAN), dict(softcap=INF), dict(window=-1), dict(slopes=6 * G + 2),
            dict(prefix=6 * G + 1), dict(starts=6 * G + 3))


def test_attn_prefill_mod_refusals(lib):
    def call(**kw):
        a = dict(PF, **kw)
        return lib.opscale_attn_prefill_mod(*(a[n] for n in PF), None, None)

    for bad in (dict(Hkv=5), dict(qs=100), dict(ms=0), dict(cu=None), dict(scale=NAN), dict(scale=0.0), dict(q=G + 8),
                dict(dt=3), dict(B=-1), dict(T=-1), dict(o=G), dict(o=2 * G + 16), dict(o=3 * G), dict(o=5 * G),
                dict(mods=_mods(slopes=4 * G)), dict(mods=_mods(prefix=4 * G + 64)), dict(mods=_mods(starts=4 * G))):
        assert call(**bad) == 1, bad
    for bad in BAD_MODS:
        assert call(mods=_mods(**bad)) == 1, bad
        assert "attn_prefill_mod" in _err(lib)
    assert call(scale=2.0 ** -65, mods=_mods(slopes=6 * G)) == 1 and "2^-64" in _err(lib)
    assert call(D=96) == 2
    assert call(T=0) == 0 and call(B=0) == 0


DC = dict(q=G, qs=32 * 128, kc=2 * G, vc=3 * G, tab=4 * G, ctx=5 * G, o=6 * G, B=256, Hq=32, Hkv=8, D=128, bs=16, mb=512,
          nb=69424, mc=8192, scale=0.08, mods=None, dt=1, ws=7 * G, wsb=1 << 30)


def test_attn_decode_mod_refusals(lib):
    def call(**kw):
        a = dict(DC, **kw)
        return lib.opscale_attn_decode_mod(*(a[n] for n in DC), None, None)

    need = lib.opscale_attn_decode_mod_workspace_size(256, 32, 128, 8192)
    for bad in (dict(bs=12), dict(tab=None), dict(mb=0), dict(qs=32 * 128 - 8), dict(qs=48 * 128 + 4), dict(Hkv=5),
                dict(B=-1), dict(mc=0), dict(dt=9), dict(scale=NAN), dict(scale=-1.0), dict(nb=1 << 40), dict(q=G + 4),
                dict(o=G), dict(o=2 * G), dict(o=3 * G + 256), dict(o=4 * G), dict(o=5 * G), dict(ws=6 * G + 16),
                dict(ws=G), dict(ws=2 * G), dict(mods=_mods(slopes=6 * G)), dict(mods=_mods(prefix=7 * G)),
                dict(mods=_mods(starts=6 * G + 4))):
        assert call(**bad) == 1, bad
    for bad in BAD_MODS:
        assert call(mods=_mods(**bad)) == 1, bad
        assert "attn_decode_mod" in _err(lib)
    # keys of one sequence and slots of the cache
    free = dict(tab=1 << 60, o=1 << 61, ws=3 << 60)
    assert call(bs=1024, mb=(1 << 21) - 1, B=0) == 0 and call(bs=1, mb=(1 << 31) - 1023, **free) == 1
    assert "2^31 - 1024" in _err(lib)
    assert call(bs=1024, nb=(1 << 26) + 1, **free) == 1 and "2^36" in _err(lib)
    assert call(wsb=need - 1) == 3 and call(ws=None) == 3 and call(ws=7 * G + 8) == 3
    assert call(D=256) == 2
    assert call(B=0) == 0


# ------------------------------------------------------------- profiling ---
def test_descriptor_layouts(tmp_path):
    """The descriptors' fields lie where the header puts them."""
    import shutil
    import subprocess
    if shutil.which("gcc") is None:
        pytest.skip("gcc not available")
    import paper_2608_13499_amd as ops
    L = ops._lib
    members = {"qk_norm_rope": L._QkNormRopeArgs, "block_tables": L._BlockTablesArgs,
               "attn_prefill_mod": L._PrefillModArgs, "attn_decode_mod": L._DecodeModArgs}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "opscale.h"', "int main(void) {",
             'printf("desc %zu\\n", sizeof(opscale_op_desc));', 'printf("mods %zu\\n", sizeof(opscale_attn_mods));',
             'printf("last %d\\n", (int)OPSCALE_OP_ATTN_DECODE_MOD);']
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
    assert int(out.pop("desc")) == ctypes.sizeof(L.OpDesc) and int(out.pop("mods")) == ctypes.sizeof(L.AttnMods)
    assert int(out.pop("last")) == L.OP_ATTN_DECODE_MOD
    assert {n: int(at) for n, at in out.items()} == {f"{m}.{f}": getattr(cls, f).offset for m, cls in members.items()
                                                     for f, _ in cls._fields_}


def test_profile_refusals(lib):
    import paper_2608_13499_amd as ops
    L, out = ops._lib, ops.Profile()
    for op in (L.OP_QK_NORM_ROPE, L.OP_BLOCK_TABLES, L.OP_ATTN_PREFILL_MOD, L.OP_ATTN_DECODE_MOD, 13):
        assert lib.opscale_op_profile(ctypes.byref(ops.OpDesc(op=op, dt=1)), 1, 1, None, 0, None, ctypes.byref(out)) == 1, op
