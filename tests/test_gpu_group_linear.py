"""Products grouped by label (GPU) against 64-bit sums: every direction and type, empty experts, rows of no expert, odd sizes, strides and alignments,
what lies beside the operands, and values that are not finite.

Bounds: a sum of k products in fp32, in whatever order, is off by at most k roundings of 2^-24 of the sum of their magnitudes (bf16 and 8-bit products are
exact; the three parts of an fp32 value leave out less than 2^-24 of a product: one rounding more); the storage type's rounding comes on top."""
import numpy as np
import pytest

from paper_2102_10485_amd import binding as B
from tests import gpu_util as U
from tests import operators_ref as R
from tests.test_gpu_rms_norm import host, matrix

pytestmark = pytest.mark.gpu

# offsets, inputs, outputs
SHAPES = [
    ([0, 1], 8, 8), ([0, 1], 1, 1), ([0, 3], 7, 5), ([0, 0, 1, 1], 64, 64), ([0, 5, 5, 130, 131], 96, 40),
    ([0, 17, 33, 200], 130, 257), ([0, 64, 128, 300], 264, 136), ([0, 1, 2, 3, 4, 5, 6, 7, 8], 512, 72), ([0, 300], 1000, 33),
    ([0, 2, 140, 140, 273], 72, 520), ([0] + [i // 2 for i in range(1, 150)] + [90], 40, 48),
]


def run(kind, bf16, a, other, offs, groups, n_in, n_out, pad=0, offset=0):
    """kind: "y", "dx" (a: the rows; other: w) or "dw" (a: x, other: dy)."""
    torch = U.torch_mod()
    prec = B.BF16 if bf16 else B.FP32
    rows = len(a)
    o = torch.from_numpy(np.asarray(offs, np.int32)).cuda()
    ma = matrix(a, bf16, a.shape[1] + pad, offset)
    if kind == "dw":
        mo = matrix(other, bf16, n_out + pad, offset)
        n = B.group_linear_wgrad_bytes(groups, rows, n_in, n_out)
        work = torch.full((max(n, 16),), 255, dtype=torch.uint8, device="cuda")
        out = torch.full((groups * n_in * n_out + 9,), float("nan"), device="cuda")
        B.group_linear_wgrad(prec, ma[2], n_in + pad, mo[2], n_out + pad, o.data_ptr(), groups, rows, n_in, n_out, out.data_ptr() + 4 * (offset % 8),
                             work.data_ptr() if n else 0, n)
        torch.cuda.synchronize()
        at = offset % 8
        assert bool(out[:at].isnan().all()) and bool(out[at + groups * n_in * n_out:].isnan().all())
        return out[at:at + groups * n_in * n_out].view(groups, n_out, n_in).cpu().numpy()
    w = torch.full((other.size + 8,), float("nan"), dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
    w[offset:offset + other.size] = torch.from_numpy(other.ravel())
    pw = w.data_ptr() + offset * w.element_size()
    cols = n_out if kind == "y" else n_in
    mo = matrix(np.full((rows, cols), 7.0), bf16, cols + pad, offset)
    call = B.group_linear if kind == "y" else B.group_linear_dgrad
    call(prec, ma[2], a.shape[1] + pad, pw, o.data_ptr(), groups, rows, n_in, n_out, mo[2], cols + pad)
    torch.cuda.synchronize()
    rest = mo[0].clone()
    rest[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] = float("nan")
    assert bool(rest.isnan().all())
    return host(mo[1])


def problem(offs, n_in, n_out, bf16, extra=0, whole=False, seed=0):
    rng = np.random.default_rng([len(offs), n_in, n_out, seed])
    rows, groups = offs[-1] + extra, len(offs) - 1

    def values(*shape):
        return rng.integers(-2, 3, shape).astype(np.float32) if whole else U.round_to(rng.normal(size=shape), bf16)

    return values(rows, n_in), values(groups, n_out, n_in), values(rows, n_out)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_all_directions(case, bf16):
    offs, n_in, n_out = SHAPES[case]
    groups = len(offs) - 1
    for pad, offset, extra in ((0, 0, 0), (8, 8, 3), (1, 1, 0)):
        x, w, dy = problem(offs, n_in, n_out, bf16, extra, seed=pad)
        out = R.UBF if bf16 else 0
        y, size = R.linear(x, w, offs)
        assert np.all(np.abs(run("y", bf16, x, w, offs, groups, n_in, n_out, pad, offset) - y) <= (n_in + 1) * R.U32 * size + out * np.abs(y))
        dx, size = R.linear(dy, w.transpose(0, 2, 1), offs)
        assert np.all(np.abs(run("dx", bf16, dy, w, offs, groups, n_in, n_out, pad, offset) - dx) <= (n_out + 1) * R.U32 * size + out * np.abs(dx))
        dw, size = R.linear_wgrad(x, dy, offs, groups)
        assert np.all(np.abs(run("dw", bf16, x, dy, offs, groups, n_in, n_out, pad, offset) - dw) <= (len(x) + 1) * R.U32 * size)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("offs,n_in,n_out", [([0, 40, 41, 300], 128, 192), ([0, 260, 600], 320, 264), ([0, 9], 1024, 512), ([0, 1030], 256, 256)])
def test_whole_numbers_are_exact(offs, n_in, n_out, bf16):
    """Sums of whole numbers have no rounding in fp32: every element is pinned (bf16 outputs: to its rounding)."""
    groups = len(offs) - 1
    x, w, dy = problem(offs, n_in, n_out, bf16, whole=True)
    rnd = lambda v: U.round_to(v.astype(np.float32), bf16)  # noqa: E731
    assert np.array_equal(run("y", bf16, x, w, offs, groups, n_in, n_out), rnd(R.linear(x, w, offs)[0]))
    assert np.array_equal(run("dx", bf16, dy, w, offs, groups, n_in, n_out), rnd(R.linear(dy, w.transpose(0, 2, 1), offs)[0]))
    assert np.array_equal(run("dw", bf16, x, dy, offs, groups, n_in, n_out), R.linear_wgrad(x, dy, offs, groups)[0])


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n_in,n_out", [(64, 128), (33, 50)])
def test_offsets_that_are_none(n_in, n_out, bf16):
    """Decreasing offsets and offsets outside the rows count as the nearest that are valid; nothing is read or written elsewhere."""
    offs = [5, 20, 12, 40, 1 << 30, -7, 60]
    rng = np.random.default_rng(5)
    x, w, dy = (rng.integers(-2, 3, s).astype(np.float32) for s in ((70, n_in), (6, n_out, n_in), (70, n_out)))
    assert np.array_equal(run("y", bf16, x, w, offs, 6, n_in, n_out), U.round_to(R.linear(x, w, offs)[0], bf16))
    assert np.array_equal(run("dx", bf16, dy, w, offs, 6, n_in, n_out), U.round_to(R.linear(dy, w.transpose(0, 2, 1), offs)[0], bf16))
    assert np.array_equal(run("dw", bf16, x, dy, offs, 6, n_in, n_out), R.linear_wgrad(x, dy, offs, 6)[0])


def test_no_experts():
    x, dy = np.ones((5, 16), np.float32), np.ones((5, 8), np.float32)
    for bf16 in (False, True):
        assert not run("y", bf16, x, np.zeros((0, 8, 16), np.float32), [0], 0, 16, 8).any()
        assert not run("dx", bf16, dy, np.zeros((0, 8, 16), np.float32), [0], 0, 16, 8).any()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n_in,n_out", [(128, 64), (37, 29)])
def test_values_that_are_not_finite(n_in, n_out, bf16):
    """They reach the outputs that they are summed into, as in fp32 arithmetic, and no other expert's or row's."""
    offs, groups = [0, 20, 50, 50, 90], 4
    x, w, dy = problem(offs, n_in, n_out, bf16, extra=4)
    x[30, 3], x[31, 0], dy[25, 2] = np.inf, np.nan, -np.inf
    x[92, 1] = dy[93, 1] = np.nan                                    # rows of no expert
    with np.errstate(invalid="ignore"):
        y, dx, dw = R.linear(x, w, offs)[0], R.linear(dy, w.transpose(0, 2, 1), offs)[0], R.linear_wgrad(x, dy, offs, groups)[0]
    for got, want in ((run("y", bf16, x, w, offs, groups, n_in, n_out), y), (run("dx", bf16, dy, w, offs, groups, n_in, n_out), dx),
                      (run("dw", bf16, x, dy, offs, groups, n_in, n_out), dw)):
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isinf(got), np.isinf(want))
        inf = np.isinf(want)
        assert np.array_equal(np.sign(got[inf]), np.sign(want[inf]))
        fine = np.isfinite(want)
        assert np.all(np.abs(got[fine] - want[fine]) <= 1e-5 * np.sqrt(200) * 10 + R.UBF * np.abs(want[fine]))


def test_fp32_values_of_any_size():
    """The largest and the smallest fp32 values: products that overflow do, small ones keep 24 bits."""
    offs = [0, 4]
    x, w, dy = (v.copy() for v in problem(offs, 32, 16, False))
    x[0] *= 1e38
    x[1] *= 1e-38
    x[2] *= 3e30
    with np.errstate(over="ignore"):
        y, size = R.linear(x, w, offs)
        want = np.where(np.abs(y) > np.finfo(np.float32).max, np.inf * np.sign(y), y)
    got = run("y", False, x, w, offs, 1, 32, 16)
    near = np.abs(np.abs(y) - np.finfo(np.float32).max) < 1e37       # (sums whose last terms decide)
    partial = size > np.finfo(np.float32).max                        # (chains that may overflow on the way)
    ok = ~near & ~partial
    assert np.all(np.abs(got[ok] - want[ok]) <= 33 * R.U32 * size[ok] + 2e-45)
    assert np.all(np.isfinite(got[1:]))


# ---- 8 bits ----

def run8(x8, xs, w8, ws, offs, n_in, n_out, bf16, pad=0):
    torch = U.torch_mod()
    groups, rows = len(offs) - 1, len(x8)
    t = [torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in (x8, xs, w8, ws, np.asarray(offs, np.int32))]
    whole, view, p = matrix(np.zeros((rows, n_out)), bf16, n_out + pad)
    B.group_linear8(*(a.data_ptr() for a in t), groups, rows, n_in, n_out, B.BF16 if bf16 else B.FP32, p, n_out + pad)
    torch.cuda.synchronize()
    return host(view)


def problem8(offs, n_in, n_out, extra=0, seed=0):
    rng = np.random.default_rng([len(offs), n_in, n_out, seed, 8])
    rows, groups, k = offs[-1] + extra, len(offs) - 1, R.padded(n_in)

    def codes(*shape):
        q = rng.integers(0, 127, shape).astype(np.uint8) | (rng.integers(0, 2, shape) << 7).astype(np.uint8)
        q[..., n_in:] = 0
        return q

    def scales(*shape):
        return rng.integers(110, 130, shape).astype(np.uint8)

    return codes(rows, k), scales(rows, k // 128), codes(groups, n_out, k), scales(groups, n_out, k // 128)


SHAPES8 = [([0, 1], 128, 16), ([0, 1], 1, 1), ([0, 3, 3, 7], 200, 37), ([0, 0, 130, 131], 384, 130), ([0, 20, 300], 1152, 264), ([0, 8], 2048, 96),
           ([0] + [i for i in range(1, 70)], 256, 48), ([0, 600], 256, 520)]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("case", range(len(SHAPES8)))
def test_eight_bits(case, bf16):
    offs, n_in, n_out = SHAPES8[case]
    for pad, extra in ((0, 0), (3, 5)):
        x8, xs, w8, ws = problem8(offs, n_in, n_out, extra)
        y, size = R.linear(R.decode(x8, xs), R.decode(w8, ws), offs)
        got = run8(x8, xs, w8, ws, offs, n_in, n_out, bf16, pad)
        assert np.all(np.abs(got - y) <= (R.padded(n_in) + 1) * R.U32 * size + (R.UBF * np.abs(y) if bf16 else 0))


def test_eight_bits_every_code_and_scale():
    """Each code and each scale byte of either side against itself alone: a product of one value with one, exact."""
    x8 = np.zeros((256, 128), np.uint8)
    x8[:, 5] = np.arange(256)
    w8 = np.zeros((1, 256, 128), np.uint8)
    w8[0, :, 5] = np.arange(256)
    xs, ws = np.full((256, 1), 120, np.uint8), np.full((1, 256, 1), 131, np.uint8)
    got = run8(x8, xs, w8, ws, [0, 256], 128, 256, False)
    want = R.TABLE[:, None] * R.TABLE[None] * 2.0 ** -3
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.nan_to_num(got), np.nan_to_num(want.astype(np.float32)))
    x8[:, 5], w8[0, :, 5] = 0x38, 0x38                               # ones
    xs[:, 0], ws[0, :, 0] = np.clip(np.arange(256), 1, 254), np.clip(np.arange(256), 1, 254)
    got = run8(x8, xs, w8, ws, [0, 256], 128, 256, False)
    e = xs.astype(int) + ws[0].astype(int).T - 254
    normal = (e >= -126) & (e <= 127)
    assert np.array_equal(got[normal], (2.0 ** e[normal]).astype(np.float32))


def test_eight_bits_after_the_norm():
    """The norm's 8-bit output and quantized weights through the product, against the product of the unrounded values: 2^-4 a value."""
    torch = U.torch_mod()
    rng = np.random.default_rng(11)
    rows, n_in, n_out, offs = 50, 300, 70, [0, 20, 20, 50]
    x, w = rng.normal(size=(rows, n_in)).astype(np.float32), (rng.normal(size=(3, n_out, n_in)) / 17).astype(np.float32)
    tx, tw, gain = torch.from_numpy(x).cuda(), torch.from_numpy(w).cuda(), torch.ones(n_in, device="cuda")
    k = R.padded(n_in)
    x8, xs = torch.empty((rows, k), dtype=torch.uint8, device="cuda"), torch.empty((rows, k // 128), dtype=torch.uint8, device="cuda")
    w8, ws = torch.empty((3, n_out, k), dtype=torch.uint8, device="cuda"), torch.empty((3, n_out, k // 128), dtype=torch.uint8, device="cuda")
    o, y = torch.tensor(offs, dtype=torch.int32, device="cuda"), torch.empty((rows, n_out), device="cuda")
    B.rms_norm(B.FP32, tx.data_ptr(), n_in, 0, 0, gain.data_ptr(), 1e-5, rows, n_in, 0, 0, 0, 0, x8.data_ptr(), xs.data_ptr(), 0)
    B.quantize8(B.FP32, tw.data_ptr(), n_in, 3 * n_out, n_in, w8.data_ptr(), ws.data_ptr())
    B.group_linear8(x8.data_ptr(), xs.data_ptr(), w8.data_ptr(), ws.data_ptr(), o.data_ptr(), 3, rows, n_in, n_out, B.FP32, y.data_ptr(), n_out)
    ref = R.norm(x, None, np.ones(n_in, np.float32), 1e-5, None)[2]
    want, size = R.linear(ref, w, offs)
    # independent roundings of at most 2^-4 each (and 2^-10 of the block's scale near zero) on both sides
    err = np.linalg.norm(y.cpu().numpy() - want) / np.linalg.norm(want)
    assert err <= np.sqrt(2) * 2.0 ** -4


@pytest.mark.parametrize("rows_of_codes", [True, False])
def test_eight_bits_of_the_smallest_and_the_largest_blocks(rows_of_codes):
    """Every finite code in blocks of the lowest and the highest exponents against single weights.  An element counts as the bf16 number nearest to it: a multiple of 2^-133 (off by half
    of that at most, and not at all from E = -124 on), and infinite from 2^128 on; products with one weight are exact, up to what fp32 holds."""
    codes = np.array([c for c in range(256) if c & 127 != 127], np.uint8)
    n, exponents = len(codes), np.array([-126, -125, -124, -123, 117, 118, 119, 120, 121, 127])
    x8 = np.zeros((n * len(exponents), 128), np.uint8)
    x8[:, 5] = np.tile(codes, len(exponents))
    xs = np.repeat(exponents + 127, n).astype(np.uint8)[:, None]
    value = R.TABLE[x8[:, 5]] * 2.0 ** (xs[:, 0].astype(np.float64) - 127)
    for e in (110, -20):                                             # of the weights 1, 1.125 ... 3.75 times 2^e
        w8, ws = np.zeros((1, 16, 128), np.uint8), np.full((1, 16, 1), 127 + e, np.uint8)
        w8[0, :, 5] = 0x38 + np.arange(16)
        w = R.decode(w8[0], ws[0])[:, 5]
        got = run8(x8, xs, w8, ws, [0, len(x8)], 128, 16, False) if rows_of_codes else run8(w8[0], ws[0], x8[None], xs[None], [0, 16], 128, len(x8), False).T
        with np.errstate(over="ignore", invalid="ignore"):
            want = np.where(np.abs(value) < 2.0 ** 128, value, np.inf * np.sign(value))[:, None] * w
            want = np.where(np.abs(want) < 2.0 ** 128, want, np.inf * np.sign(want))
        off = np.where(np.abs(value) < 2.0 ** -122, 2.0 ** -134, 0.0) * (value % 2.0 ** -133 != 0)
        near = np.isfinite(want)
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~near], want[~near])
        error = np.abs(got[near].astype(np.float64) - want[near])
        assert np.all(error <= (off[:, None] * np.abs(w))[near] + (2.0 ** -149 if e < 0 else 0.0)), (e, error.max())
