"""The workspace of the rotation's gradients holds what the workgroups write into it: the functions that size, kernel and launch share, compiled for the
CPU, and the size that the library states."""
import ctypes
import itertools
import os
import subprocess

import pytest

from helpers import built_package

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_16579_amd", "csrc")
SOURCE = r'''
#include "arl2_rope_plan.h"
extern "C" {
int groups(int B, int L, int D, int H, int Hk, int f32) { return arl2::rope_bwd_workgroups(B, L, arl2::rope_shape((H + Hk) * (D / 16), f32, true), f32); }
int part(int by_heads, int D, int H, int Hk) { return arl2::rope_part(by_heads, D, H, Hk); }
}
'''


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("rope_plan")
    (d / "shim.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Werror", "-I", CSRC, "-o", str(d / "shim.so"), str(d / "shim.cpp")], check=True)
    return ctypes.CDLL(str(d / "shim.so"))


@pytest.fixture(scope="module")
def A():
    A = built_package()
    A.load_library()
    return A


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,Hk", [(1, 0), (2, 0), (1, 1), (3, 0), (8, 0), (12, 12), (32, 8), (40, 8), (96, 0), (96, 96)])
def test_the_workspace_holds_all_parts(A, plan, D, H, Hk):
    for (B, L), by_heads, f32 in itertools.product([(1, 1), (1, 9), (3, 5), (1, 4680), (2, 8400011)], (0, 1), (0, 1)):
        part = plan.part(by_heads, D, H, Hk)
        # a part holds each weight's gradient once, and there are no keys' where there are no keys
        assert part == (D + (D if Hk else 0) if by_heads else (H + Hk) * D)
        groups, have = plan.groups(B, L, D, H, Hk, f32), A.arl2_rope_workspace_bytes(B, H, Hk, L, D)
        assert 1 <= groups <= B * L
        assert groups * part * 4 <= have, (B, L, by_heads, f32)
