"""What an 8-bit operand of the grouped products asks for (csrc/code_walk.h), on the host: each step of its waves' share of the sum once, a step ahead, and nothing
outside that share -- also where the share is a single step, and in what is asked for behind the last one."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STEP = 64
STAGES = 2       # steps that are written to LDS before the first one is multiplied; one more is written for each that is


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("code_walk") / "code_walk.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", os.path.join(ROOT, "tests", "c", "code_walk_host.cpp"), "-o", so], check=True)
    fn = ctypes.CDLL(so).code_walk

    def call(k0, k_end, writes):
        out = np.zeros(writes + 1, np.int32)
        fn(k0, k_end, writes, out.ctypes.data_as(ctypes.c_void_p))
        return out.tolist()
    return call


# rows of 128 codes up to 1152, whole or in two halves: (first, end) of a set of waves
SHARES = [s for wide in range(128, 1153, 128) for s in ((0, wide), (0, wide // 2), (wide // 2, wide))]


@pytest.mark.parametrize("k0,k_end", SHARES)
def test_requests(walk, k0, k_end):
    steps = (k_end - k0) // STEP
    asked = walk(k0, k_end, STAGES + steps)
    assert asked[:steps] == list(range(k0, k_end, STEP))             # in order, before each is written
    assert all(k0 <= k and k + STEP <= k_end for k in asked), asked
