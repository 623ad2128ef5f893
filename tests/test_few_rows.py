"""The rules for products of few rows (csrc/few_rows.h), on the host.  Rows of a block of the fp32 gradient: no length of the sum is a case of its own, and calls of few blocks keep 16 rows.  Two sets of
waves for an 8-bit tile: only where every tile, whatever the heights, has a CU of its own."""
import ctypes
import os
import subprocess

import pytest

from tests.test_code_walk import ROOT


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("few_rows") / "few_rows.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", os.path.join(ROOT, "tests", "c", "few_rows_host.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)
    lib.dgrad_sixteens.argtypes = [ctypes.c_longlong, ctypes.c_longlong, ctypes.c_int]
    lib.two_sets8.argtypes = [ctypes.c_longlong, ctypes.c_longlong, ctypes.c_longlong, ctypes.c_int]
    return lib


@pytest.fixture(scope="module")
def sixteens(rules):
    return rules.dgrad_sixteens


@pytest.mark.parametrize("k", [512, 513, 520, 640, 1024, 4096])
def test_few_blocks_take_16_rows(sixteens, k):
    """Two experts of 100 rows, 512 <- 512, are 72 blocks of 32 rows and 64 columns on 256 CUs; 16 rows an expert never fill 32."""
    assert [sixteens(each, blocks, k) for each, blocks in ((300, 1), (100, 72), (300, 44), (16, 10000), (1, 10000))] == [1] * 5


def test_more_blocks_and_shorter_sums_never_turn_back(sixteens):
    for blocks in (1, 44, 72, 159, 160, 232, 511, 512, 5000):
        of_k = [sixteens(100, blocks, k) for k in range(512, 4097)]
        assert of_k == sorted(of_k, reverse=True) and of_k[0] == of_k[1]       # (a sum of 512 is none of its own)
    for k in (512, 576, 577, 2048):
        of_blocks = [sixteens(100, b, k) for b in range(1, 2000)]
        assert of_blocks == sorted(of_blocks) and of_blocks[-1] == 2


def test_two_sets_of_waves_have_a_cu_for_every_tile(rules):
    """Tiles of the two heights are dealt to eight XCDs of 32 CUs apart: at most 32 on each, however the experts fall to the heights."""
    taken = 0
    for groups in range(1, 300):
        for cols in range(1, 300):
            if not rules.two_sets8(40, groups, cols, 4096):
                assert groups * cols > 240
                continue
            taken += 1
            assert all(-(-high * cols // 8) + -(-(groups - high) * cols // 8) <= 32 for high in range(groups + 1)), (groups, cols)
    assert taken > 500
    assert not rules.two_sets8(65, 2, 2, 4096) and not rules.two_sets8(32, 8, 32, 1024)          # (more than one height of tile; a short sum)
    assert rules.two_sets8(32, 8, 32, 4096) and not rules.two_sets8(32, 16, 20, 2048) and not rules.two_sets8(40, 64, 6, 1024)
