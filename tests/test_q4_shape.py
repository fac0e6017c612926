"""Sizes of 4-bit matrices, compiled for the host from the kernels' own header, and the group sizes that the binding hands on."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import workloads as W
from paper_2501_05370_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include "q4_shape.h"
extern "C" int groups_of(int K, int group) { return q4::groups_of(K, group); }
extern "C" int many_columns(int ntiles) { return q4::many_columns(ntiles); }
extern "C" int many_groups(int ntiles) { return q4::many_groups(ntiles); }
extern "C" long pack_grid(long blocks) { return q4::pack_grid(blocks); }
"""


@pytest.fixture(scope="module")
def shape(tmp_path_factory):
    d = tmp_path_factory.mktemp("shape")
    (d / "s.cpp").write_text(SOURCE)
    lib = str(d / "s.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2501_05370_amd", "csrc"),
                    str(d / "s.cpp"), "-o", lib], check=True)
    return ctypes.CDLL(lib)


@pytest.mark.parametrize("group", [32, 64, 128, 256, 1 << 20, (1 << 31) - 128])
@pytest.mark.parametrize("K", [1, 31, 32, 33, 1000, 1 << 20])
def test_groups_of_a_row(shape, K, group):
    """The largest group of 32 bits plus K does not fit them: a row still has its one scale."""
    assert shape.groups_of(K, group) == -(-K // group)


@pytest.mark.parametrize("group", [(1 << 32) + 32, (1 << 31), 0, -128])
def test_groups_beyond_32_bits_are_refused(group):
    q, s = np.zeros((4, 32), np.uint8), np.zeros((4, 1), np.uint16)
    with pytest.raises(B.SDError, match="group"):
        B.Q4Matrix.sdden_q4_create(q, s, 64, group)
    with pytest.raises(B.SDError, match="group=-?[0-9]* must be positive"):
        B.Denoiser.sdden_mlp4_create(W.random_mlp(np.random.default_rng(0), 8, 8, 2), group, 4, 4)


@pytest.mark.parametrize("N", [1, 16, 128, 129, 1024, 1025, 12288, 1 << 20])
def test_launches_stay_below_the_limit_of_threads(shape, N):
    """A grid has to stay below 2^32 threads: the rows of a call are spread over as many launches as that takes."""
    ntiles = -(-N // 16)
    columns, groups = shape.many_columns(ntiles), shape.many_groups(ntiles)
    assert columns % 8 == 0 and columns * 128 >= N and groups >= 2047
    assert columns * groups * 256 < 1 << 32 <= columns * (groups + 1) * 256


def test_the_layout_kernel_s_grid(shape):
    fn = shape.pack_grid
    fn.argtypes, fn.restype = [ctypes.c_long], ctypes.c_long
    for blocks in (1, 3, 4, 5, (1 << 22) - 1, 1 << 22, 1 << 26, 1 << 29):
        assert fn(blocks) == min(-(-blocks // 4), 1 << 20)
