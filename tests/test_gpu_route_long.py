"""The router and its gradient (GPU) where blocks take several turns over the rows: the next turn's logits are asked for ahead, and what a row's choices left in LDS must not reach the next row.

Bounds as in test_gpu_route.py: (100 + 2 |l - max|) roundings of 2^-24 for a probability, three times that of the gradient's terms without their signs, one rounding of the storage type.  The
terms: with D = sum p share + sum p g the gradient is p (share - D) + p g, so that the balance's share and the weight's g, which may all but cancel (share = 0.598, g = -0.598 in one of 3 million),
are terms of their own: p (share + sum p share) + p (|g| + sum p |g|).  The means: a lane group adds a probability a turn, then come at most 6 joins of a wave's groups and 3 of its waves, and the
blocks in 64 bits."""
import numpy as np
import pytest

from tests import experts_ref as E
from tests import operators_ref as R
from tests.test_gpu_route import problem, run, spread

pytestmark = pytest.mark.gpu
# rows, experts, k, turns: rows of a turn are 256 lanes by the lanes of a row, times 1024 blocks (experts of 257 to 512: 512, more than 1024: 256)
SHAPES = [(530000, 6, 2, 3), (140000, 20, 4, 3), (33000, 100, 4, 3), (20000, 256, 8, 2), (17000, 400, 5, 3), (9000, 700, 3, 3), (2500, 1100, 6, 3)]


@pytest.mark.parametrize("bf16,normalize,in_place", [(False, False, True), (False, True, False), (True, True, True), (True, False, False)])
@pytest.mark.parametrize("rows,e,k,turns", SHAPES)
def test_several_turns(rows, e, k, turns, bf16, normalize, in_place):
    l = problem(rows, e, bf16, 3)
    dw = np.random.default_rng(rows).normal(size=(rows, k)).astype(np.float32)
    dw[l.max(1) == -np.inf] = np.nan                                  # (what stands beside no choice is not used)
    got = run(l, k, normalize, bf16, dweight=dw, balance_grad=0.3 * rows, in_place=in_place)
    want = E.route(l, k, normalize)
    assert np.array_equal(got["expert"], want["expert"]) and np.array_equal(got["counts"], want["counts"])
    rel = spread(l)
    at = np.take_along_axis(rel, np.maximum(want["expert"], 0), 1).max(1, keepdims=True)
    assert np.all(np.abs(got["weight"] - want["weight"]) <= (2 if normalize else 1) * at * want["weight"])
    size = (want["p"] * (rel + (turns + 9) * R.U32)).sum(0) / want["counts"][-1]
    assert np.all(np.abs(got["mean"] - want["mean"]) <= size + R.U32 * want["mean"])
    share = want["counts"][:e] / want["counts"][:e].sum()
    assert abs(got["balance"] - want["balance"]) <= e * (share * size).sum() + 2 * R.U32 * want["balance"]
    with np.errstate(invalid="ignore"):
        d = E.route_backward(l, k, normalize, dw, 0.3 * rows)[0]
        terms = E.route_backward(l, k, normalize, dw, 0.0)[1] + E.route_backward(l, k, normalize, np.zeros_like(dw), 0.3 * rows)[1]
    assert np.all(np.abs(got["dlogits"] - d) <= 3 * rel.max(1, keepdims=True) * terms + (R.UBF * np.abs(d) + 2.0 ** -134 if bf16 else 2.0 ** -149))
    assert not got["dlogits"][l == -np.inf].any()
