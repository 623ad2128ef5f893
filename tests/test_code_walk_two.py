"""What an 8-bit operand of a product with an epilogue asks for (CodeWalkTwo in csrc/code_walk.h), on the host: each step of its waves' share of the sum once, two steps ahead, and nothing outside
that share -- also where the share is a single step, and in what is asked for behind the last one."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from tests.test_code_walk import ROOT, SHARES, STAGES, STEP


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("code_walk_two") / "code_walk_two.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", os.path.join(ROOT, "tests", "c", "code_walk_two_host.cpp"), "-o", so], check=True)
    fn = ctypes.CDLL(so).code_walk_two

    def call(k0, k_end, writes):
        out = np.zeros(writes + 2, np.int32)
        fn(k0, k_end, writes, out.ctypes.data_as(ctypes.c_void_p))
        return out.tolist()
    return call


@pytest.mark.parametrize("k0,k_end", SHARES)
def test_requests(walk, k0, k_end):
    steps = (k_end - k0) // STEP
    asked = walk(k0, k_end, STAGES + steps)
    assert asked[:steps] == list(range(k0, k_end, STEP))             # in order, before each is written
    assert all(k0 <= k and k + STEP <= k_end for k in asked), asked
