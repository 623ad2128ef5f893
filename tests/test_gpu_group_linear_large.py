"""The grouped products at sizes that reach the tile kernels (GPU): whole tiles and experts' last ones of every height, many experts, rows of any alignment, weight gradients in
parts, and memory beyond 4 GiB.  Sums of whole numbers are exact in fp32 and pin every element; bounds as in test_gpu_group_linear.py."""
import numpy as np
import pytest

from paper_2102_10485_amd import binding as B
from tests import gpu_util as U
from tests import operators_ref as R
from tests.test_gpu_group_linear import problem8, run, run8

pytestmark = pytest.mark.gpu


def offsets(counts):
    return [0] + [int(v) for v in np.cumsum(counts)]


RNG = np.random.default_rng(7)
CASES = {
    # experts with none, one, and up to 600 rows, more than 64 of them: whole tiles, and last ones of every height
    "many": (offsets(RNG.permutation([0, 0, 1, 2, 64, 65, 128, 129, 192, 193, 256, 257, 600] + list(RNG.integers(1, 30, 60)))), 72, 1032),
    "eight": (offsets([80, 1, 0, 150, 128, 40, 129, 112]), 1000, 1000),
    "odd": (offsets([80, 1, 0, 150, 128, 40, 129, 112]), 1001, 999),
    "odd inputs": (offsets([700, 33]), 333, 2048),
    "wide outputs": (offsets([15] * 5 + [0] + [16] * 4 + [3]), 36, 3300),
    "wide inputs": (offsets([15] * 5 + [0] + [16] * 4 + [3]), 3300, 36),
    "long": (offsets([1, 1999]), 264, 2056),
    "parts": (offsets([3, 1900]), 96, 200),
    "odd parts": (offsets([5, 0, 2500]), 101, 77),
    # many whole tiles of 256, and last ones of a half and of a quarter
    "few ends, outputs": (offsets([1300, 1124]), 72, 6008),
    "few ends, inputs": (offsets([1300, 1124]), 6008, 72),
    "few ends, one step": (offsets([1300, 1124]), 40, 6008),
}


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("name", list(CASES))
def test_whole_numbers_are_exact(name, bf16):
    offs, n_in, n_out = CASES[name]
    groups, rows = len(offs) - 1, offs[-1] + 5                       # (five rows of no expert)
    rng = np.random.default_rng([n_in, n_out])
    x, w, dy = (rng.integers(-2, 3, s).astype(np.float32) for s in ((rows, n_in), (groups, n_out, n_in), (rows, n_out)))
    rnd = lambda v: U.round_to(v.astype(np.float32), bf16)  # noqa: E731
    y, dx, dw = rnd(R.linear(x, w, offs)[0]), rnd(R.linear(dy, w.transpose(0, 2, 1), offs)[0]), R.linear_wgrad(x, dy, offs, groups)[0]
    for pad, offset in ((0, 0), (3, 1)) if name in ("many", "odd") else ((0, 0),):
        assert np.array_equal(run("y", bf16, x, w, offs, groups, n_in, n_out, pad, offset), y)
        assert np.array_equal(run("dx", bf16, dy, w, offs, groups, n_in, n_out, pad, offset), dx)
        assert np.array_equal(run("dw", bf16, x, dy, offs, groups, n_in, n_out, pad, offset), dw)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("name", ["many", "odd", "wide outputs", "wide inputs", "long", "parts"])
def test_errors(name, bf16):
    offs, n_in, n_out = CASES[name]
    groups, rows = len(offs) - 1, offs[-1]
    rng = np.random.default_rng([n_in, n_out, 1])
    x, w, dy = (U.round_to(rng.normal(size=s), bf16) for s in ((rows, n_in), (groups, n_out, n_in), (rows, n_out)))
    out = R.UBF if bf16 else 0
    for got, (want, size), k in ((run("y", bf16, x, w, offs, groups, n_in, n_out), R.linear(x, w, offs), n_in),
                                 (run("dx", bf16, dy, w, offs, groups, n_in, n_out), R.linear(dy, w.transpose(0, 2, 1), offs), n_out)):
        assert np.all(np.abs(got - want) <= (k + 1) * R.U32 * size + out * np.abs(want))
    dw, size = R.linear_wgrad(x, dy, offs, groups)
    assert np.all(np.abs(run("dw", bf16, x, dy, offs, groups, n_in, n_out) - dw) <= (rows + 1) * R.U32 * size)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("name", ["many", "odd", "long"])
def test_values_that_are_not_finite_stay_with_their_expert(name, bf16):
    offs, n_in, n_out = CASES[name]
    groups, rows = len(offs) - 1, offs[-1]
    rng = np.random.default_rng(3)
    x, w, dy = (rng.integers(-2, 3, s).astype(np.float32) for s in ((rows, n_in), (groups, n_out, n_in), (rows, n_out)))
    row = rows // 2
    expert = int(np.searchsorted(offs, row, side="right")) - 1
    x[row, n_in - 1], dy[row, n_out - 1] = np.nan, np.inf
    y, dx, dw = run("y", bf16, x, w, offs, groups, n_in, n_out), run("dx", bf16, dy, w, offs, groups, n_in, n_out), run("dw", bf16, x, dy, offs, groups, n_in, n_out)
    assert np.isnan(y[row]).all() and np.isfinite(np.delete(y, row, 0)).all()
    assert not np.isfinite(dx[row]).any() and np.isfinite(np.delete(dx, row, 0)).all()
    with np.errstate(invalid="ignore"):
        want = R.linear_wgrad(x, dy, offs, groups)[0]
    assert np.array_equal(np.isfinite(dw), np.isfinite(want)) and np.array_equal(np.isnan(dw[expert]), np.isnan(want[expert]))
    assert np.array_equal(dw[np.isfinite(want)], want[np.isfinite(want)])


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("name", ["many", "odd", "long", "wide outputs", "odd inputs", "few ends, outputs"])
def test_eight_bits(name, bf16):
    offs, n_in, n_out = CASES[name]
    x8, xs, w8, ws = problem8(offs, n_in, n_out, 5)
    y, size = R.linear(R.decode(x8, xs), R.decode(w8, ws), offs)
    got = run8(x8, xs, w8, ws, offs, n_in, n_out, bf16, 3 if name == "odd" else 0)
    assert np.all(np.abs(got - y) <= (R.padded(n_in) + 1) * R.U32 * size + (R.UBF * np.abs(y) if bf16 else 0))


def test_the_same_bits_again():
    offs, n_in, n_out = CASES["many"]
    groups = len(offs) - 1
    rng = np.random.default_rng(1)
    x, w, dy = (rng.normal(size=s).astype(np.float32) for s in ((offs[-1], n_in), (groups, n_out, n_in), (offs[-1], n_out)))
    for bf16 in (False, True):
        for kind, a, b in (("y", x, w), ("dx", dy, w), ("dw", x, dy)):
            assert np.array_equal(run(kind, bf16, a, b, offs, groups, n_in, n_out), run(kind, bf16, a, b, offs, groups, n_in, n_out))


@pytest.mark.parametrize("rows", [5, 300])
def test_weights_and_rows_beyond_4_gib(rows):
    """The last of seventy experts' weights start at 4.6 GB; rows 2^27 elements apart reach 5 GB and more (64 rows: 17 GB)."""
    torch = U.torch_mod()
    groups, n_in, n_out = 70, 8192, 4096
    rng = np.random.default_rng(rows)
    last = rng.integers(-2, 3, (n_out, n_in)).astype(np.float32)
    w = torch.zeros((groups, n_out, n_in), dtype=torch.bfloat16, device="cuda")
    w[-1] = torch.from_numpy(last).cuda()
    offs = torch.tensor([0] * groups + [rows], dtype=torch.int32, device="cuda")
    x, dy = rng.integers(-1, 2, (rows, n_in)).astype(np.float32), rng.integers(-1, 2, (rows, n_out)).astype(np.float32)
    tx, tdy = torch.from_numpy(x).cuda().bfloat16(), torch.from_numpy(dy).cuda().bfloat16()
    y, dx = torch.zeros((rows, n_out), dtype=torch.bfloat16, device="cuda"), torch.zeros((rows, n_in), dtype=torch.bfloat16, device="cuda")
    B.group_linear(B.BF16, tx.data_ptr(), n_in, w.data_ptr(), offs.data_ptr(), groups, rows, n_in, n_out, y.data_ptr(), n_out)
    B.group_linear_dgrad(B.BF16, tdy.data_ptr(), n_out, w.data_ptr(), offs.data_ptr(), groups, rows, n_in, n_out, dx.data_ptr(), n_in)
    assert np.array_equal(y.float().cpu().numpy(), U.round_to(x @ last.T, True))
    assert np.array_equal(dx.float().cpu().numpy(), U.round_to(dy @ last, True))
    if rows > 64:
        return
    stride = 1 << 27
    far = torch.zeros(64 * stride, dtype=torch.bfloat16, device="cuda").view(64, stride)
    at = [0, 20, 40, 61, 63]
    far[at, :n_in] = tx
    out = torch.zeros((64, n_out), dtype=torch.bfloat16, device="cuda")
    offs = torch.tensor([0] * groups + [64], dtype=torch.int32, device="cuda")
    B.group_linear(B.BF16, far.data_ptr(), stride, w.data_ptr(), offs.data_ptr(), groups, 64, n_in, n_out, out.data_ptr(), n_out)
    assert torch.equal(out[at], y)
    far.zero_()
    B.group_linear(B.BF16, tx.data_ptr(), n_in, w.data_ptr(), torch.tensor([0] * groups + [rows], dtype=torch.int32, device="cuda").data_ptr(), groups, rows, n_in, n_out,
                   far.data_ptr(), stride)
    assert torch.equal(far[:rows, :n_out], y) and not bool(far[:rows, n_out:n_out + 64].any())
    gain = torch.ones(n_in, device="cuda")
    z, inv = torch.zeros((64, n_in), dtype=torch.bfloat16, device="cuda"), torch.zeros(64, device="cuda")
    far[:, :n_in] = 3
    B.rms_norm(B.BF16, far.data_ptr(), stride, 0, 0, gain.data_ptr(), 0.0, 64, n_in, 0, 0, z.data_ptr(), n_in, 0, 0, inv.data_ptr())
    assert bool((z == 1).all()) and np.allclose(inv.cpu().numpy(), 1 / 3, rtol=1e-6)


# Next to many whole tiles of 256, experts' last rows are taken in half the columns by two sets of waves, which share the sum: sums of one step (the second set has none), of two,
# three and five, outputs that end eight or sixteen columns behind a tile, and rows that end anywhere in a half or a quarter of the height.
ENDS = [([2580, 2404], 40, 3208), ([2580, 2404], 72, 3208), ([2580, 2404], 136, 3216), ([2561, 2432], 264, 3208), ([2624, 0, 2369], 128, 3208)]
NO_EXPERT = 5


def assert_ends_are_narrow(counts, rows, width):
    """The rules of the launch, on the same counts: 256 x 256 tiles, and ends of at most a quarter of the whole tiles' number."""
    assert (rows // 256 + len(counts)) * -(-width // 256) >= 256 and rows // len(counts) > 32
    rest = [n % 256 for n in counts + [NO_EXPERT]]
    whole = sum(n // 256 for n in counts + [NO_EXPERT]) + sum(r > 128 for r in rest)
    half, low = sum(64 < r <= 128 for r in rest), sum(0 < r <= 64 for r in rest)
    assert half > 0 and low > 0 and 4 * (half + low) <= whole


@pytest.mark.parametrize("counts,short,wide", ENDS)
def test_ends_in_half_the_columns(counts, short, wide):
    offs, groups = offsets(counts), len(counts)
    rows = offs[-1] + NO_EXPERT
    assert_ends_are_narrow(counts, rows, wide)
    rng = np.random.default_rng([short, wide])
    a, w = (rng.integers(-2, 3, s).astype(np.float32) for s in ((rows, short), (groups, wide, short)))
    want = U.round_to(R.linear(a, w, offs)[0].astype(np.float32), True)
    assert np.array_equal(run("y", True, a, w, offs, groups, short, wide), want)
    assert np.array_equal(run("dx", True, a, w.transpose(0, 2, 1).copy(), offs, groups, wide, short), want)
    # what is not finite in the last expert's last row reaches that row alone
    a[offs[-1] - 1, short - 1] = np.nan
    for got in (run("y", True, a, w, offs, groups, short, wide), run("dx", True, a, w.transpose(0, 2, 1).copy(), offs, groups, wide, short)):
        assert np.isnan(got[offs[-1] - 1]).all() and np.array_equal(np.delete(got, offs[-1] - 1, 0), np.delete(want, offs[-1] - 1, 0))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("counts,short,wide", ENDS)
def test_ends_in_half_the_columns_in_eight_bits(counts, short, wide, bf16):
    offs = offsets(counts)
    assert_ends_are_narrow(counts, offs[-1] + NO_EXPERT, wide)
    x8, xs, w8, ws = problem8(offs, short, wide, NO_EXPERT)
    y, size = R.linear(R.decode(x8, xs), R.decode(w8, ws), offs)
    got = run8(x8, xs, w8, ws, offs, short, wide, bf16)
    assert np.all(np.abs(got - y) <= (R.padded(short) + 1) * R.U32 * size + (R.UBF * np.abs(y) if bf16 else 0))


@pytest.mark.parametrize("bf16", [False, True])
def test_more_tiles_than_a_launch_has_threads_for(bf16):
    """2050 experts of 2^20 outputs and one input: 2^24 tiles and more of 256 threads each.  Whole numbers; experts without rows get zeros."""
    torch = U.torch_mod()
    groups, n_out, kind = 2050, 1 << 20, torch.bfloat16 if bf16 else torch.float32
    starts = np.zeros(groups + 1, np.int32)
    starts[1:], starts[1025:], starts[2050:] = 2, 3, 5                # two rows of the first expert, one of the 1025th, two of the last
    x = torch.tensor([[1.0], [2.0], [3.0], [1.0], [-1.0]], device="cuda").to(kind)
    dy = torch.randint(-2, 3, (5, n_out), device="cuda", generator=torch.Generator("cuda").manual_seed(1)).to(kind)
    dw = torch.full((groups, n_out), float("nan"), device="cuda")
    nbytes = B.group_linear_wgrad_bytes(groups, 5, 1, n_out)
    offs = torch.from_numpy(starts).cuda()
    B.group_linear_wgrad(B.BF16 if bf16 else B.FP32, x.data_ptr(), 1, dy.data_ptr(), n_out, offs.data_ptr(), groups, 5, 1, n_out, dw.data_ptr(), 0, nbytes)
    f = dy.float()
    assert nbytes == 0 and torch.equal(dw[0], f[0] + 2 * f[1]) and torch.equal(dw[1024], 3 * f[2]) and torch.equal(dw[2049], f[3] - f[4])
    for lo, hi in ((1, 1024), (1025, 2049)):
        assert int(dw[lo:hi].count_nonzero()) == 0 and not bool(dw[lo:hi].isnan().any())


# (rows fall unevenly, so that experts end inside tiles; the sizes take tiles of 64 and of 128)
FP32_TILES = [([40, 0, 130, 90], 200, 136), ([1500, 1201], 333, 2056)]


@pytest.mark.parametrize("counts,n_in,n_out", FP32_TILES)
def test_fp32_values_that_are_not_finite_leave_other_outputs_alone(counts, n_in, n_out):
    """The outputs that a NaN or an infinity is not summed into have the bits that they have without it; the others are what fp32 arithmetic gives."""
    offs, groups = offsets(counts), len(counts)
    rows = offs[-1]
    rng = np.random.default_rng([n_in, n_out, 4])
    x, w, dy = (rng.normal(size=s).astype(np.float32) for s in ((rows, n_in), (groups, n_out, n_in), (rows, n_out)))
    clean = [run(k, False, a, b, offs, groups, n_in, n_out) for k, a, b in (("y", x, w), ("dx", dy, w), ("dw", x, dy))]
    x[5, 3], x[rows - 1, n_in - 1], dy[7, 2], dy[rows - 2, 0] = np.nan, np.inf, -np.inf, np.nan
    x[20, 1], x[21, 1], dy[20, 4], dy[21, 4] = np.inf, -np.inf, 1.0, 1.0               # (NaN where both are summed)
    with np.errstate(invalid="ignore"):
        want = R.linear(x, w, offs)[0], R.linear(dy, w.transpose(0, 2, 1), offs)[0], R.linear_wgrad(x, dy, offs, groups)[0]
    touched = np.zeros((rows, 1), bool), np.zeros((rows, 1), bool), np.zeros((groups, n_out, n_in), bool)
    touched[0][[5, rows - 1, 20, 21]] = touched[1][[7, rows - 2, 20, 21]] = True
    touched[2][0, :, [1, 3]] = touched[2][-1, :, n_in - 1] = touched[2][0, [2, 4]] = touched[2][-1, 0] = True
    for kind, a, b, old, ref, at in zip(("y", "dx", "dw"), (x, dy, x), (w, w, dy), clean, want, touched):
        got = run(kind, False, a, b, offs, groups, n_in, n_out)
        assert np.array_equal(np.where(at, 0, got), np.where(at, 0, old)), kind
        assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(np.isinf(got), np.isinf(ref)), kind
        assert np.array_equal(np.signbit(got[np.isinf(ref)]), np.signbit(ref[np.isinf(ref)])), kind


@pytest.mark.parametrize("counts,n_in,n_out", FP32_TILES)
def test_fp32_values_out_of_the_parts_range(counts, n_in, n_out):
    """Rows of 1e33 and weights of 1e-30 and less, sums of 1e25 and more: what three bf16 parts cannot hold is summed in fp32."""
    offs, groups = offsets(counts), len(counts)
    rows = offs[-1]
    rng = np.random.default_rng([n_in, n_out, 5])
    x, w, dy = (rng.normal(size=s).astype(np.float32) for s in ((rows, n_in), (groups, n_out, n_in), (rows, n_out)))
    x[::3] *= np.float32(1e33)
    dy[1::5] *= np.float32(3e34)
    w[0] *= np.float32(1e-30)
    w[-1] *= np.float32(1e-8)
    y, size = R.linear(x, w, offs)
    assert np.all(np.abs(run("y", False, x, w, offs, groups, n_in, n_out) - y) <= (n_in + 1) * R.U32 * size)
    dx, size = R.linear(dy, w.transpose(0, 2, 1), offs)
    assert np.all(np.abs(run("dx", False, dy, w, offs, groups, n_in, n_out) - dx) <= (n_out + 1) * R.U32 * size)
    dy = (rng.normal(size=dy.shape) * 1e-30).astype(np.float32)
    dw, size = R.linear_wgrad(x, dy, offs, groups)
    assert np.all(np.abs(run("dw", False, x, dy, offs, groups, n_in, n_out) - dw) <= (rows + 1) * R.U32 * size)
