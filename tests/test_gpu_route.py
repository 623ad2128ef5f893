"""The router and its gradient (GPU) against 64 bits: every number of lanes a row takes, ties, experts that are not there, rows without any, what is not finite, odd strides,
and many rows.  Choices and counts are whole numbers and equal.

Bounds, relative: exp is off by a few roundings of 2^-24 and |l - max| of them for the rounding of its argument, its sum over 4096 experts in 64 lanes by 64 + 6, the weights' sum by
16: (100 + 2 |l - max|) roundings; sums over the rows of a block, its waves and the blocks: up to 8 rows a lane group in these cases, 3 waves, and the blocks in 64 bits: 32 more.  The gradient's
terms have two such factors, sums over 70 more, and a few products: 3 (100 + 2 |l - max|) of the terms without their signs; and one rounding of the storage type."""
import numpy as np
import pytest

from paper_2102_10485_amd import binding as B
from tests import experts_ref as E
from tests import gpu_util as U
from tests import operators_ref as R
from tests.test_gpu_rms_norm import host, matrix

pytestmark = pytest.mark.gpu
# rows, experts, k
SHAPES = [(1, 1, 1), (4, 64, 2), (300, 3, 3), (1000, 8, 2), (70, 9, 4), (65, 32, 1), (33, 33, 5), (129, 100, 8), (17, 128, 16), (40, 130, 3), (9, 256, 8), (6, 512, 16),
          (5, 513, 4), (3, 1000, 2), (4, 1030, 7), (2, 4096, 16)]


def run(l, k, normalize, bf16, pad=0, offset=0, stats=True, dweight=None, balance_grad=0.0, use_counts=True, in_place=False):
    torch = U.torch_mod()
    rows, e = l.shape
    prec, st = B.BF16 if bf16 else B.FP32, e + pad
    ml = matrix(l, bf16, st, offset)
    expert = torch.full((rows * k + 8,), 77, dtype=torch.int32, device="cuda")
    weight = torch.full((rows * k + 8,), float("nan"), device="cuda")
    counts, mean, balance = torch.full((e + 1,), -5, dtype=torch.int32, device="cuda"), torch.full((e,), float("nan"), device="cuda"), torch.full((1,), float("nan"), device="cuda")
    n = B.route_bytes(rows, e)
    work = torch.full((max(n, 16),), 255, dtype=torch.uint8, device="cuda")
    if stats:
        B.route(prec, ml[2], st, rows, e, k, normalize, expert.data_ptr(), weight.data_ptr(), counts.data_ptr(), mean.data_ptr(), balance.data_ptr(), work.data_ptr(), n)
    else:
        B.route(prec, ml[2], st, rows, e, k, normalize, expert.data_ptr(), weight.data_ptr(), 0, 0, 0, 0, 0)
    torch.cuda.synchronize()
    assert bool((expert[rows * k:] == 77).all()) and bool(weight[rows * k:].isnan().all())
    out = dict(expert=expert[:rows * k].view(rows, k).cpu().numpy(), weight=weight[:rows * k].view(rows, k).cpu().numpy(), counts=counts.cpu().numpy(), mean=mean.cpu().numpy(),
               balance=float(balance))
    if dweight is not None:
        dw = torch.from_numpy(dweight).cuda()
        md = ml if in_place else matrix(np.zeros_like(l), bf16, st, offset)
        B.route_backward(prec, ml[2], st, rows, e, k, normalize, expert.data_ptr(), dw.data_ptr(), counts.data_ptr() if use_counts else 0, balance_grad, md[2], st)
        torch.cuda.synchronize()
        rest = md[0].clone()
        rest[offset:offset + rows * st].view(rows, st)[:, :e] = float("nan")
        assert bool(rest.isnan().all())
        out["dlogits"] = host(md[1])
    return out


def problem(rows, e, bf16, seed=0, masked=True):
    rng = np.random.default_rng([rows, e, seed])
    l = U.round_to(rng.normal(size=(rows, e)) * 2 + rng.normal(size=e), bf16)
    if masked:
        l[rng.random((rows, e)) < 0.2] = -np.inf
        l[rng.random(rows) < 0.1] = -np.inf
    return l


def spread(l):
    there = np.isfinite(l)
    top = np.where(there, l, -np.inf).max(1, keepdims=True, initial=-np.inf)
    return np.where(there, 100 + 2 * np.abs(np.where(there, l - np.where(np.isfinite(top), top, 0), 0)), 0) * R.U32


def check(got, l, k, normalize, stats=True):
    want = E.route(l, k, normalize)
    rel = spread(l)
    assert np.array_equal(got["expert"], want["expert"])
    at = np.take_along_axis(rel, np.maximum(want["expert"], 0), 1).max(1, keepdims=True)
    assert np.all(np.abs(got["weight"] - want["weight"]) <= (2 if normalize else 1) * at * want["weight"])
    if stats:
        assert np.array_equal(got["counts"], want["counts"])
        counted = max(1, want["counts"][-1])
        size = (want["p"] * (rel + 32 * R.U32)).sum(0) / counted
        assert np.all(np.abs(got["mean"] - want["mean"]) <= size + R.U32 * want["mean"])
        e = l.shape[1]
        share = want["counts"][:e] / max(1, want["counts"][:e].sum())
        assert abs(got["balance"] - want["balance"]) <= e * (share * size).sum() + 2 * R.U32 * want["balance"]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,e,k", SHAPES)
def test_forward_and_gradient(rows, e, k, bf16):
    for pad, offset, normalize, masked in ((0, 0, True, False), (8, 8, False, True), (3, 1, True, True), (1, 0, False, False)):
        l = problem(rows, e, bf16, pad, masked)
        dw = np.random.default_rng(pad).normal(size=(rows, k)).astype(np.float32)
        dw[l.max(1) == -np.inf] = np.nan                              # (what stands beside no choice is not used)
        got = run(l, k, normalize, bf16, pad, offset, True, dw, 0.3, in_place=pad == 8)
        check(got, l, k, normalize)
        with np.errstate(invalid="ignore"):
            want, size = E.route_backward(l, k, normalize, dw, 0.3)
        rel = 3 * np.maximum(spread(l).max(1, keepdims=True), 0)
        assert np.all(np.abs(got["dlogits"] - want) <= rel * size + (R.UBF * np.abs(want) + 2.0 ** -134 if bf16 else 2.0 ** -149)), np.abs(got["dlogits"] - want).max()
        assert not got["dlogits"][l == -np.inf].any()
        plain = run(l, k, normalize, bf16, pad, offset, stats=False)
        assert np.array_equal(plain["expert"], got["expert"]) and np.array_equal(plain["weight"], got["weight"]) and plain["counts"][0] == -5


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("e,k", [(5, 3), (20, 4), (64, 8), (100, 4), (300, 6), (600, 4), (2000, 5)])
def test_ties(e, k, bf16):
    """Equal logits: the lowest index first; -0 and 0 are equal, numbers below the smallest normal one are told apart."""
    rng = np.random.default_rng(e)
    l = rng.integers(-1, 2, (50, e)).astype(np.float32)
    l[l == 0] = np.where(rng.random((l == 0).sum()) < 0.5, -0.0, 0.0)
    l[10] = 3.5
    l[11] = 0.0
    l[12, e // 2], l[13, e - 1] = 9, 9
    l[14] = -1
    l[14, [1, e - 1]] = 2.0 ** -130, 2.0 ** -131
    check(run(l, k, True, bf16), l, k, True)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("e", [6, 30, 100, 200, 700, 1500])
def test_values_that_are_not_finite(e, bf16):
    """NaN is never chosen; a row with one, or with +infinity, has NaN for the experts that are there, and no other row has.  The type's lowest value is a number."""
    rng = np.random.default_rng(e)
    l = U.round_to(rng.normal(size=(12, e)), bf16)
    lowest = float(U.from_bf16_bits(np.uint16(0xFF7F)).item()) if bf16 else np.finfo(np.float32).min
    l[1, 2], l[3, 0], l[4] = np.nan, np.inf, np.nan
    l[5] = -np.inf
    l[5, 3] = np.nan
    l[6] = lowest
    l[7] = lowest
    l[7, 4] = 0
    l[8] = -np.inf
    l[8, 5] = lowest
    k = 3
    dw = rng.normal(size=(12, k)).astype(np.float32)
    for normalize in (False, True):
        got = run(l, k, normalize, bf16, stats=True, dweight=dw, balance_grad=0.0, use_counts=False)
        want = E.route(l, k, normalize)
        assert np.array_equal(got["expert"], want["expert"]) and np.array_equal(got["counts"], want["counts"])
        assert np.array_equal(np.isnan(got["weight"]), np.isnan(want["weight"])) and np.isnan(got["balance"])
        fine = ~np.isnan(want["weight"])
        assert np.all(np.abs(got["weight"][fine] - want["weight"][fine]) <= 300 * R.U32)
        assert np.array_equal(got["expert"][[4, 5]], np.full((2, k), -1)) and np.array_equal(got["expert"][8], [5, -1, -1])
        d = got["dlogits"]
        there = (l > -np.inf) & ~np.isnan(l)
        assert np.isfinite(d[[0, 2, 4, 5, 6, 7, 8, 9, 10, 11]]).all() and not d[~there].any()
        assert np.isnan(d[1][there[1]]).all() and np.isnan(d[3][there[3]]).all() and not d[[4, 5]].any()


@pytest.mark.parametrize("e,k", [(8, 2), (64, 6), (256, 8), (1000, 1)])
def test_many_rows(e, k):
    """More rows than all blocks take at a time: 70000 of them.  A lane group adds up to 70000 / (512 blocks, 4 rows at a time) = 35 rows."""
    l = problem(70000, e, True, 3)
    want = E.route(l, k, True)
    got = run(l, k, True, True)
    assert np.array_equal(got["expert"], want["expert"]) and np.array_equal(got["counts"], want["counts"])
    assert np.all(np.abs(got["weight"] - want["weight"]) <= 2 * spread(l).max() * want["weight"])
    size = (want["p"] * (spread(l) + 64 * R.U32)).sum(0) / want["counts"][-1]
    assert np.all(np.abs(got["mean"] - want["mean"]) <= size)
    share = want["counts"][:e] / want["counts"][:e].sum()
    assert abs(got["balance"] - want["balance"]) <= e * (share * size).sum() + 2 * R.U32 * want["balance"]
    again = run(l, k, True, True)
    assert all(np.array_equal(got[n], again[n]) for n in ("expert", "weight", "counts", "mean")) and got["balance"] == again["balance"]


def test_all_the_same_and_all_one():
    """Balance is 1 where all experts get the same, and the number of experts where one gets everything; without any expert it is 0."""
    l = np.eye(16, dtype=np.float32).repeat(8, 0)
    assert abs(run(l, 1, True, False)["balance"] - 1) < 1e-5
    l = np.full((40, 16), -np.inf, np.float32)
    l[:, 3] = 1
    got = run(l, 1, True, False)
    assert got["balance"] == 16 and got["mean"][3] == 1 and got["mean"].sum() == 1
    got = run(np.full((40, 16), -np.inf, np.float32), 2, True, False, dweight=np.ones((40, 2), np.float32), balance_grad=1.0)
    assert got["balance"] == 0 and not got["mean"].any() and not got["counts"].any() and not got["dlogits"].any() and not got["weight"].any()


def test_no_rows():
    torch = U.torch_mod()
    counts, mean, balance = torch.full((6,), 7, dtype=torch.int32, device="cuda"), torch.ones(5, device="cuda"), torch.ones(1, device="cuda")
    B.route(B.BF16, 0, 5, 0, 5, 2, True, 0, 0, counts.data_ptr(), mean.data_ptr(), balance.data_ptr(), 0, 0)
    B.route_backward(B.BF16, 0, 5, 0, 5, 2, True, 0, 0, counts.data_ptr(), 1.0, 0, 5)
    torch.cuda.synchronize()
    assert not counts.any() and not mean.any() and not balance.any()
