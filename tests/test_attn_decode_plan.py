"""Workgroups of decode attention with modifiers, compiled for the host."""
import ctypes
import itertools
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_13499_amd", "csrc")
CXX = shutil.which("g++") or shutil.which("c++")

pytestmark = pytest.mark.skipif(CXX is None, reason="no host C++ compiler")


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("decode_plan")
    src, so = str(d / "plan.cpp"), str(d / "plan.so")
    with open(src, "w") as f:
        f.write('''
#include "attn_decode_plan.h"
extern "C" {
int workgroups(int B, int len, int window, int prefix, int groups, int waves) {
  return opscale::mod_workgroups(B, len, window, prefix != 0, groups, waves);
}
int most(int B, int len) { return opscale::mod_workgroups_most(B, len); }
}
''')
    subprocess.run([CXX, "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{CSRC}", src, "-o", so], check=True)
    return ctypes.CDLL(so)


CASES = list(itertools.product([1, 2, 4, 16, 64, 65, 512, 700], [1, 31, 64, 700, 8192, 32768, 1 << 20, (1 << 31) - 1],
                               [0, 1, 16, 128, 4096, (1 << 31) - 1], [1, 2, 5, 71, 600], [1, 2, 4, 8]))


def test_a_window_takes_no_workgroups_from_a_prefix(plan):
    """A prefix may be as long as the context, whatever the window: its call has the
    workgroups of one without a window, or more."""
    for B, n, window, groups, waves in CASES:
        assert plan.workgroups(B, n, window, 1, groups, waves) >= plan.workgroups(B, n, 0, 0, groups, waves), \
            (B, n, window, groups, waves)


def test_a_window_alone_bounds_them(plan):
    """Without a prefix there are no more workgroups than tiles the window can reach, and one a sequence."""
    for B, n, window, groups, waves in CASES:
        if window:
            tiles = B * min(-(-n // 32), window // 32 + 2)
            assert 1 <= plan.workgroups(B, n, window, 0, groups, waves) <= tiles + B


def test_workspaces_hold_any_of_them(plan):
    for B, n, window, groups, waves in CASES:
        for prefix in (0, 1):
            assert 1 <= plan.workgroups(B, n, window, prefix, groups, waves) <= plan.most(B, n) <= 512
