"""The plan of the linear of e4m3 operands (csrc/gemm_fp8_plan.h), compiled for the host."""
import collections
import ctypes
import functools
import os
import shutil
import subprocess
import tempfile

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_13499_amd", "csrc")
CXX = shutil.which("g++") or shutil.which("c++")

Plan = collections.namedtuple("Plan", "path waves splits chunk ws_bytes items longest")
PATHS = ("rows", "256x256", "128x256", "128x128", "few")
TILES = {"256x256": (256, 256), "128x256": (128, 256), "128x128": (128, 128)}


@functools.lru_cache(None)
def _lib():
    with tempfile.TemporaryDirectory() as d:
        src, so = os.path.join(d, "plan.cpp"), os.path.join(d, "plan.so")
        with open(src, "w") as f:
            f.write('''
#include "gemm_fp8_plan.h"
using namespace opscale;
extern "C" {
void plan(int64_t M, int64_t N, int64_t K, int bf16, int split_ok, int64_t* out) {
  const LinearFp8Plan p = plan_linear_fp8(M, N, K, bf16 != 0, split_ok != 0);
  out[0] = p.path, out[1] = p.waves, out[2] = p.splits, out[3] = p.chunk, out[4] = (int64_t)p.ws_bytes;
}
// the most items that a workgroup of a chained launch takes
int longest(int64_t items) {
  const int rounds = (int)((items + kNumCUs - 1) / kNumCUs);
  int most = 0;
  for (int g = 0; g < rounds; ++g) {
    const Chain c = chain_of(g, rounds, true);
    if (c.len > most) most = c.len;
  }
  return most;
}
}
''')
        subprocess.run([CXX, "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{CSRC}", src, "-o", so], check=True)
        lib = ctypes.CDLL(so)
    lib.plan.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int] * 2 + [ctypes.c_void_p]
    lib.plan.restype = None
    lib.longest.argtypes = [ctypes.c_int64]
    return lib


def plan(M, N, K, dtype="bf16", split=True):
    """items: of a tile kernel (tiles and ranges of K); longest: the most of them that a chain would join."""
    out = (ctypes.c_int64 * 5)()
    _lib().plan(M, N, K, dtype == "bf16", split, out)
    path, items = PATHS[out[0]], 0
    if path in TILES:
        bm, bn = TILES[path]
        items = -(-M // bm) * -(-N // bn) * out[2]
    return Plan(path, out[1], out[2], out[3], out[4], items, _lib().longest(items) if items else 0)
