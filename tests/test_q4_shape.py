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
