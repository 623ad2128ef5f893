"""The router's weights behind a row's last choice (GPU): 0, also in a row whose probabilities are NaN, for every number of lanes that a row takes."""
import numpy as np
import pytest

from tests import experts_ref as E
from tests import gpu_util as U
from tests import operators_ref as R
from tests.test_gpu_route import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("e", [4, 8, 20, 32, 33, 100, 200, 400, 700, 1500])
def test_rows_with_nan_and_fewer_experts_than_choices(e, bf16):
    """NaN or +infinity among fewer than k experts that are there: NaN for those, and 0 beside every choice of no expert."""
    k = 4
    l = np.full((9, e), -np.inf, np.float32)
    l[0, :2] = np.nan, 1
    l[1, [0, e - 1]] = np.inf, 2
    l[2, :3] = np.nan, 1, 0
    l[3, 1] = np.inf
    l[4, 3] = np.nan
    l[5, :2] = 1, 0
    l[6] = U.round_to(np.random.default_rng(e).normal(size=e), bf16)
    l[7, [1, 2, 3]] = np.inf, np.inf, np.nan
    for normalize in (False, True):
        want = E.route(l, k, normalize)
        for stats in (False, True):
            got = run(l, k, normalize, bf16, stats=stats)
            assert np.array_equal(got["expert"], want["expert"])
            assert np.array_equal(np.isnan(got["weight"]), np.isnan(want["weight"])) and not got["weight"][want["expert"] < 0].any()
            fine = ~np.isnan(want["weight"])
            # exp, its sum over up to 1500 experts and the weights': 100 roundings, 2 |l - max| < 20 of them for exp's argument; twice with the division of sums
            assert np.all(np.abs(got["weight"][fine] - want["weight"][fine]) <= 240 * R.U32 * want["weight"][fine])
