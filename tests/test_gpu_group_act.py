"""Products grouped by label with bias, activation and residual, and the gradients through the activation (GPU): against 64-bit sums at the sizes that reach every kernel, odd ones, strides and
alignments, empty experts and rows of none, in place, and what is not finite.

Bounds.  Sums as in test_gpu_group_linear.py: k + 1 roundings of 2^-24 of the terms' magnitudes, two more for the bias or the other gradient.  An activation's slope is below 1.13.  GELU in
fp32: erfc and exp to 8 roundings, and z^2 of them from the rounding of their arguments; for bf16 a polynomial within 4.7e-6 and the hardware's exp2, whose argument z^2 / (2 ln 2) is rounded
three times: 2^-17 + 2 z^2 roundings.  SiLU: exp(-z) with |z| roundings of its argument, the reciprocal, the product: 8 + 4 |z|.  Results below 2^-126 may become zero.  The residual's addition is
one rounding of the terms, and the storage type's comes on top."""
import numpy as np
import pytest

from paper_2102_10485_amd import binding as B
from tests import experts_ref as E
from tests import gpu_util as U
from tests import operators_ref as R
from tests.test_gpu_group_linear import SHAPES, SHAPES8, problem8
from tests.test_gpu_group_linear_large import CASES, offsets
from tests.test_gpu_rms_norm import host, matrix

pytestmark = pytest.mark.gpu
TINY = 2.0 ** -120


def act_error(z, kind, bf16):
    """Of the factor that the activation multiplies z with, or of its slope, relative."""
    z = np.clip(np.abs(z), 0, 1e4)
    return np.zeros_like(z) if kind <= E.RELU else (8 + (2 if bf16 else 1) * 2 * z * z) * R.U32 + (2.0 ** -17 if bf16 else 0) if kind == E.GELU else (8 + 4 * z) * R.U32


def weights(w, bf16, offset=0):
    torch = U.torch_mod()
    t = torch.full((w.size + 16,), float("nan"), dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
    t[offset:offset + w.size] = torch.from_numpy(np.ascontiguousarray(w, np.float32).ravel())
    return t, t.data_ptr() + offset * t.element_size()


def floats(a, offset):
    """fp32, `offset` elements behind the allocation's start."""
    torch = U.torch_mod()
    t = torch.full((a.size + 16,), float("nan"), device="cuda")
    t[offset:offset + a.size] = torch.from_numpy(np.ascontiguousarray(a, np.float32).ravel())
    return t, t.data_ptr() + 4 * offset


def unwritten(m, offset, rows, stride, cols):
    rest = m[0].clone()
    rest[offset:offset + rows * stride].view(rows, stride)[:, :cols] = float("nan")
    assert bool(rest.isnan().all())
    return host(m[1])


def forward(bf16, x, w, offs, bias, act, residual, pad=0, offset=0, store_z=True, in_place=False):
    torch = U.torch_mod()
    groups, n_out, n_in = w.shape
    rows = len(x)
    o = torch.from_numpy(np.asarray(offs, np.int32)).cuda()
    mx, mw = matrix(x, bf16, n_in + pad, offset), weights(w, bf16, offset)
    mb = floats(bias, offset % 4) if bias is not None else (None, 0)
    mr = matrix(residual, bf16, n_out + pad, offset) if residual is not None else None
    mz = matrix(np.full((rows, n_out), 7.0), bf16, n_out + pad, offset)
    my = mr if in_place else matrix(np.full((rows, n_out), 7.0), bf16, n_out + pad, offset)
    B.group_linear_act(B.BF16 if bf16 else B.FP32, mx[2], n_in + pad, mw[1], o.data_ptr(), groups, rows, n_in, n_out, mb[1], act, mr[2] if mr else 0, n_out + pad,
                       mz[2] if store_z else 0, n_out + pad, my[2], n_out + pad)
    torch.cuda.synchronize()
    z = unwritten(mz, offset, rows, n_out + pad, n_out)
    assert store_z or np.array_equal(z, np.full_like(z, 7.0))
    return z, unwritten(my, offset, rows, n_out + pad, n_out)


def dgrad(bf16, dy, w, offs, act, z, other, pad=0, offset=0, into=None):
    torch = U.torch_mod()
    groups, n_out, n_in = w.shape
    rows = len(dy)
    o = torch.from_numpy(np.asarray(offs, np.int32)).cuda()
    md, mw = matrix(dy, bf16, n_out + pad, offset), weights(w, bf16, offset)
    mo = matrix(other, bf16, n_in + pad, offset) if other is not None else None
    mz = matrix(z, bf16, n_in + pad, offset) if z is not None else None
    mx = {None: matrix(np.full((rows, n_in), 7.0), bf16, n_in + pad, offset), "other": mo, "z": mz}[into]
    B.group_linear_dgrad_act(B.BF16 if bf16 else B.FP32, md[2], n_out + pad, mw[1], o.data_ptr(), groups, rows, n_in, n_out, mo[2] if mo else 0, n_in + pad, act,
                             mz[2] if mz else 0, n_in + pad, mx[2], n_in + pad)
    torch.cuda.synchronize()
    return unwritten(mx, offset, rows, n_in + pad, n_in)


def expert_rows(offs, rows, groups):
    """Each row's expert, and -1."""
    o = R.clean_offsets(offs, rows)
    g = np.searchsorted(o, np.arange(rows), side="right") - 1
    return np.where(np.arange(rows) < o[groups], np.minimum(g, groups - 1), -1)


def reference(x, w, offs, bias, residual):
    """Sums with the bias, their size; the residual: zeros for rows of no expert."""
    g = expert_rows(offs, len(x), len(w))
    z, size = R.linear(x, w, offs)
    if bias is not None:
        b = np.where((g >= 0)[:, None], bias.astype(np.float64)[g], 0.0)
        z, size = z + b, size + np.abs(b)
    r = np.zeros_like(z) if residual is None else np.where((g >= 0)[:, None], residual.astype(np.float64), 0.0)
    return z, size, r


def check_forward(got, bf16, x, w, offs, bias, act, residual, k, store_z=True):
    z, size, r = reference(x, w, offs, bias, residual)
    out, e = R.UBF if bf16 else 0, (k + 3) * R.U32 * size
    if store_z:
        assert np.all(np.abs(got[0] - z) <= e + out * np.abs(z))
    a = E.act(z, act)
    y = a + r
    assert np.all(np.abs(got[1] - y) <= 1.13 * e + act_error(z, act, bf16) * np.abs(z) * (np.abs(a) / np.maximum(np.abs(z), TINY)) + R.U32 * (np.abs(a) + np.abs(r)) + out * np.abs(y) + TINY)


def problem(offs, n_in, n_out, bf16, extra=0, whole=False, seed=0):
    rng = np.random.default_rng([len(offs), n_in, n_out, seed])
    rows, groups = offs[-1] + extra, len(offs) - 1

    def values(*shape, by=1.0):
        return rng.integers(-2, 3, shape).astype(np.float32) if whole else U.round_to(rng.normal(size=shape) * by, bf16)

    return dict(x=values(rows, n_in), w=values(groups, n_out, n_in, by=n_in ** -0.5), bias=values(groups, n_out).astype(np.float32), residual=values(rows, n_out), dy=values(rows, n_out),
                z=values(rows, n_in), other=values(rows, n_in))


def check_dgrad(got, bf16, p, offs, act, other):
    g = expert_rows(offs, len(p["dy"]), len(p["w"]))
    d, size = R.linear(p["dy"], p["w"].transpose(0, 2, 1), offs)
    o = np.where((g >= 0)[:, None], p["other"].astype(np.float64), 0.0) if other else 0.0
    d, size = d + o, size + np.abs(o)
    s = E.slope(p["z"], act)
    parts = np.abs(E.phi(p["z"])) + np.abs(p["z"]) if act == E.GELU else 1 + np.abs(p["z"]) if act == E.SILU else 0.0     # (the slope's terms)
    want = d * s
    bound = (p["dy"].shape[1] + 3) * R.U32 * size * np.maximum(np.abs(s), 1e-3) + np.abs(d) * act_error(p["z"], act, bf16) * parts + 2 * R.U32 * np.abs(want) + (R.UBF * np.abs(want) if bf16 else 0)
    assert np.all(np.abs(got - want) <= bound + TINY)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_all_sizes(case, bf16):
    offs, n_in, n_out = SHAPES[case]
    for pad, offset, extra, act in ((0, 0, 0, E.GELU), (8, 8, 3, E.RELU), (1, 1, 2, E.SILU), (3, 2, 0, E.NONE), (1, 3, 1, E.GELU)):
        p = problem(offs, n_in, n_out, bf16, extra, seed=pad)
        bias, res = p["bias"] if pad != 3 else None, p["residual"] if pad != 8 else None
        got = forward(bf16, p["x"], p["w"], offs, bias, act, res, pad, offset, store_z=pad != 1, in_place=pad == 1)
        check_forward(got, bf16, p["x"], p["w"], offs, bias, act, res, n_in, store_z=pad != 1)
        got = dgrad(bf16, p["dy"], p["w"], offs, act, p["z"] if act else None, p["other"] if pad != 8 else None, pad, offset, {0: None, 1: "other", 8: "z", 3: None}[pad])
        check_dgrad(got, bf16, p, offs, act, pad != 8)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("name", list(CASES))
def test_tiles(name, bf16):
    """At the sizes of the tile kernels: whole numbers through max(z, 0), exact; and the other activations within their bounds."""
    offs, n_in, n_out = CASES[name]
    p = problem(offs, n_in, n_out, bf16, 5, whole=True)
    z, _, r = reference(p["x"], p["w"], offs, p["bias"], p["residual"])
    rnd = lambda v: U.round_to(v.astype(np.float32), bf16)  # noqa: E731
    for pad, offset in ((0, 0), (3, 1)) if name in ("many", "odd") else ((0, 0),):
        got = forward(bf16, p["x"], p["w"], offs, p["bias"], E.RELU, p["residual"], pad, offset)
        assert np.array_equal(got[0], rnd(z)) and np.array_equal(got[1], rnd(E.act(z, E.RELU) + r))
        got = dgrad(bf16, p["dy"], p["w"], offs, E.RELU, p["z"], p["other"], pad, offset)
        g = expert_rows(offs, len(p["dy"]), len(p["w"]))
        d = R.linear(p["dy"], p["w"].transpose(0, 2, 1), offs)[0] + np.where((g >= 0)[:, None], p["other"], 0)
        assert np.array_equal(got, rnd(d * (p["z"] > 0)))
    if name in ("many", "odd", "long", "few ends, outputs", "wide inputs"):
        for act in (E.GELU, E.SILU):
            p = problem(offs, n_in, n_out, bf16, 5)
            check_forward(forward(bf16, p["x"], p["w"], offs, p["bias"], act, p["residual"]), bf16, p["x"], p["w"], offs, p["bias"], act, p["residual"], n_in)
            check_dgrad(dgrad(bf16, p["dy"], p["w"], offs, act, p["z"], p["other"]), bf16, p, offs, act, True)


def test_tiles_of_128_in_fp32():
    """1128 tiles forward and in dgrad, whole numbers: exact."""
    for offs, n_in, n_out in (([0, 2900, 3000], 40, 6000), ([0, 2900, 3000], 6000, 40)):
        p = problem(offs, n_in, n_out, False, 5, whole=True)
        z, _, r = reference(p["x"], p["w"], offs, p["bias"], p["residual"])
        if n_in == 40:
            got = forward(False, p["x"], p["w"], offs, p["bias"], E.RELU, p["residual"])
            assert np.array_equal(got[0], z) and np.array_equal(got[1], E.act(z, E.RELU) + r)
        else:
            d = R.linear(p["dy"], p["w"].transpose(0, 2, 1), offs)[0]
            d[:3000] += p["other"][:3000]
            assert np.array_equal(dgrad(False, p["dy"], p["w"], offs, E.RELU, p["z"], p["other"]), d * (p["z"] > 0))


@pytest.mark.parametrize("bf16", [False, True])
def test_the_same_bits_again_and_in_two_calls_at_once(bf16):
    """Two calls with workspaces of their own on two streams, and one after the other."""
    torch = U.torch_mod()
    offs, n_in, n_out = CASES["eight"]
    groups, rows, kind, prec = len(offs) - 1, offs[-1], torch.bfloat16 if bf16 else torch.float32, B.BF16 if bf16 else B.FP32
    p = problem(offs, n_in, n_out, bf16)
    x, w, r, dy, bias, o = (torch.from_numpy(np.asarray(v)).cuda() for v in (p["x"], p["w"], p["residual"], p["dy"], p["bias"], np.asarray(offs, np.int32)))
    x, w, r, dy = (v.to(kind) for v in (x, w, r, dy))
    size = B.group_act_backward_bytes(groups, rows, n_out)

    def passes(stream):
        z, y, dz, dx, dbias, work = torch.empty_like(r), torch.empty_like(r), torch.empty_like(r), torch.empty_like(x), torch.empty_like(bias), torch.empty(size, dtype=torch.uint8, device="cuda")
        s = stream.cuda_stream
        B.group_linear_act(prec, x.data_ptr(), n_in, w.data_ptr(), o.data_ptr(), groups, rows, n_in, n_out, bias.data_ptr(), E.GELU, r.data_ptr(), n_out, z.data_ptr(), n_out, y.data_ptr(), n_out, s)
        B.group_act_backward(prec, dy.data_ptr(), n_out, E.GELU, z.data_ptr(), n_out, o.data_ptr(), groups, rows, n_out, dz.data_ptr(), n_out, dbias.data_ptr(), work.data_ptr(), size, s)
        B.group_linear_dgrad_act(prec, dz.data_ptr(), n_out, w.data_ptr(), o.data_ptr(), groups, rows, n_in, n_out, 0, 0, E.SILU, x.data_ptr(), n_in, dx.data_ptr(), n_in, s)
        return z, y, dz, dbias, dx, work

    first = passes(torch.cuda.current_stream())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    both = [passes(s) for s in streams]
    torch.cuda.synchronize()
    for again in both:
        assert all(torch.equal(a, b) for a, b in zip(first[:5], again[:5]))


@pytest.mark.parametrize("bf16", [False, True])
def test_without_an_epilogue_it_is_the_plain_product(bf16):
    """No bias, activation or residual: the bits of gan_group_linear and its gradient."""
    from tests.test_gpu_group_linear import run
    for offs, n_in, n_out in (CASES["many"], CASES["odd"], SHAPES[5], SHAPES[8]):
        p = problem(offs, n_in, n_out, bf16, 2)
        groups = len(offs) - 1
        z, y = forward(bf16, p["x"], p["w"], offs, None, E.NONE, None)
        assert np.array_equal(y, run("y", bf16, p["x"], p["w"], offs, groups, n_in, n_out)) and np.array_equal(z, y)
        assert np.array_equal(dgrad(bf16, p["dy"], p["w"], offs, E.NONE, None, None), run("dx", bf16, p["dy"], p["w"], offs, groups, n_in, n_out))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("offs,n_in,n_out", SHAPES8 + [CASES[n] for n in ("many", "odd", "long", "wide outputs", "few ends, outputs")] +
                         [(offsets([30, 33, 0, 64, 65, 20, 1, 40]), 600, 4200), (offsets([300, 0, 129, 90]), 520, 6000),                       # (297 tiles for two sets of waves, 329 for one)
                          (offsets([40, 0, 70, 20, 32, 33, 1, 50]), 4000, 1100)])      # (few tiles of a long sum)
def test_eight_bits(offs, n_in, n_out, bf16):
    torch = U.torch_mod()
    x8, xs, w8, ws = problem8(offs, n_in, n_out, 3)
    rng = np.random.default_rng(n_in)
    rows, groups = len(x8), len(offs) - 1
    x, w = R.decode(x8, xs), R.decode(w8, ws)
    by = max(1.0, np.abs(R.linear(x, w, offs)[0]).max() / 8)
    scale = np.float32(2.0 ** np.floor(-np.log2(by)))                 # sums of a few units, by a power of two
    xs = (xs.astype(int) + int(np.log2(scale))).astype(np.uint8)
    x = R.decode(x8, xs)
    bias, res = rng.normal(size=(groups, n_out)).astype(np.float32), U.round_to(rng.normal(size=(rows, n_out)), bf16)
    t = [torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in (x8, xs, w8, ws, np.asarray(offs, np.int32), bias)]
    for act in (E.GELU, E.SILU, E.RELU):
        for pad, in_place in ((0, False), (3, True)):
            mr = matrix(res, bf16, n_out + pad)
            my = mr if in_place else matrix(np.full((rows, n_out), 7.0), bf16, n_out + pad)
            B.group_linear8_act(*(a.data_ptr() for a in t[:5]), groups, rows, n_in, n_out, t[5].data_ptr(), act, mr[2], n_out + pad, B.BF16 if bf16 else B.FP32, my[2], n_out + pad)
            torch.cuda.synchronize()
            check_forward((None, unwritten(my, 0, rows, n_out + pad, n_out)), bf16, x, w, offs, bias, act, res, R.padded(n_in), store_z=False)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n_in", [2, 40])
def test_the_activations_at_every_size_of_z(n_in, bf16):
    """Sums from -200 to 200, the smallest numbers, infinities and NaN: the activation of the bias alone (weights of zero), and its slope."""
    z = np.concatenate([np.linspace(-200, 200, 401), np.linspace(-15, 15, 601), [0.0, -0.0, 2.0 ** -120, -2.0 ** -120, 3e38, -3e38, np.inf, -np.inf, np.nan]]).astype(np.float32)
    z = U.round_to(z, bf16)
    n = len(z)
    w, x = np.zeros((1, n, n_in), np.float32), np.ones((3, n_in), np.float32)
    ones = np.ones((1, n_in, n), np.float32)                          # [experts][outputs = n_in][inputs = n]
    for act in E.ACTS:
        got = forward(bf16, x, w, [0, 3], z[None], act, None)[1]
        want = E.act(z, act)
        with np.errstate(invalid="ignore"):
            assert np.array_equal(np.isnan(got), np.broadcast_to(np.isnan(want), got.shape))
            fine = np.isfinite(want)
            assert np.array_equal(got[:, ~fine & ~np.isnan(want)], np.broadcast_to(want[~fine & ~np.isnan(want)], (3, (~fine & ~np.isnan(want)).sum())))
            assert np.all(np.abs(got - want)[:, fine] <= ((act_error(z, act, bf16) + (R.UBF if bf16 else 0) + R.U32) * np.abs(want))[fine] + 2.0 ** -119)
            s = E.slope(z, act)
            got = dgrad(bf16, np.ones((2, n_in), np.float32), ones, [0, 2], act, np.stack([z, z]) if act else None, None) / n_in
            parts = 1 + np.abs(np.clip(z, -15, 15)) * np.exp(-np.clip(z, -15, 15) ** 2 / 2) if act == E.GELU else 1.0 if act <= E.RELU else 1 + np.abs(np.clip(z, -100, 100)) * np.exp(-np.abs(np.clip(z, -100, 100)))
            fine = np.isfinite(s)
            assert np.array_equal(np.isnan(got), np.broadcast_to(np.isnan(s), got.shape))
            assert np.all(np.abs(got - s)[:, fine] <= ((act_error(np.clip(z, -15, 15), act, bf16) * parts) + (R.UBF if bf16 else R.U32) * 2 * np.abs(s) + 4 * R.U32)[fine])


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n_in,n_out", [(64, 128), (33, 50), (600, 1100)])
def test_offsets_that_are_none(n_in, n_out, bf16):
    """Decreasing offsets and offsets outside the rows count as the nearest that are valid; nothing is read or written elsewhere.  Whole numbers."""
    offs = [5, 20, 12, 40, 1 << 30, -7, 60]
    rng = np.random.default_rng(5)
    m = lambda *s: rng.integers(-2, 3, s).astype(np.float32)  # noqa: E731
    x, w, bias, res, dy, z, other = m(70, n_in), m(6, n_out, n_in), m(6, n_out), m(70, n_out), m(70, n_out), m(70, n_in), m(70, n_in)
    s, _, r = reference(x, w, offs, bias, res)
    got = forward(bf16, x, w, offs, bias, E.RELU, res)
    assert np.array_equal(got[0], U.round_to(s.astype(np.float32), bf16)) and np.array_equal(got[1], U.round_to((E.act(s, E.RELU) + r).astype(np.float32), bf16))
    g = expert_rows(offs, 70, 6)
    d = (R.linear(dy, w.transpose(0, 2, 1), offs)[0] + np.where((g >= 0)[:, None], other, 0)) * (z > 0)
    assert np.array_equal(dgrad(bf16, dy, w, offs, E.RELU, z, other), U.round_to(d.astype(np.float32), bf16))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n_in,n_out", [(128, 64), (37, 29)])
def test_values_that_are_not_finite_stay_with_their_row(n_in, n_out, bf16):
    """In a row of the operands, in one expert's bias, and in rows of no expert, whose residual, z and other hold NaN: their results are zero."""
    offs = [0, 20, 50, 50, 90]
    p = problem(offs, n_in, n_out, bf16, extra=6)
    p["x"][30, 3] = p["dy"][31, 2] = np.nan
    p["residual"][60, 1], p["other"][61, 1], p["z"][62, 2] = np.inf, np.nan, np.nan
    p["bias"][0, 4] = np.nan
    for name in ("residual", "other", "z", "x", "dy"):
        p[name][92] = np.nan
    z, y = forward(bf16, p["x"], p["w"], offs, p["bias"], E.GELU, p["residual"])
    assert np.isnan(y[30]).all() and np.isnan(y[:20, 4]).all() and np.isinf(y[60, 1]) and not y[90:].any() and not z[90:].any()
    y[30], y[:20, 4], y[60, 1], z[30], z[:20, 4] = 0, 0, 0, 0, 0
    assert np.isfinite(y).all() and np.isfinite(z).all()
    dx = dgrad(bf16, p["dy"], p["w"], offs, E.GELU, p["z"], p["other"])
    assert np.isnan(dx[31]).all() and np.isnan(dx[61, 1]) and np.isnan(dx[62, 2]) and not dx[90:].any()
    dx[31], dx[61, 1], dx[62, 2] = 0, 0, 0
    assert np.isfinite(dx).all()


# ---- the gradient through the activation, and of the bias ----

def act_backward(bf16, dy, act, z, offs, groups, pad=0, offset=0, into=None, want_dz=True, want_dbias=True):
    torch = U.torch_mod()
    rows, cols = dy.shape
    st = cols + pad
    o = torch.from_numpy(np.asarray(offs, np.int32)).cuda()
    md = matrix(dy, bf16, st, offset)
    mz = matrix(z, bf16, st, offset) if z is not None else None
    mo = {None: matrix(np.full((rows, cols), 7.0), bf16, st, offset), "dy": md, "z": mz}[into]
    n = B.group_act_backward_bytes(groups, rows, cols)
    work = torch.full((max(n, 16),), 255, dtype=torch.uint8, device="cuda")
    dbias = torch.full((groups * cols + 4,), float("nan"), device="cuda")
    B.group_act_backward(B.BF16 if bf16 else B.FP32, md[2], st, act, mz[2] if mz else 0, st, o.data_ptr(), groups, rows, cols, mo[2] if want_dz else 0, st,
                         dbias.data_ptr() if want_dbias else 0, work.data_ptr(), n)
    torch.cuda.synchronize()
    assert bool(dbias[groups * cols if want_dbias else 0:].isnan().all())
    return unwritten(mo, offset, rows, st, cols), dbias[:groups * cols].view(groups, cols).cpu().numpy()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("offs,cols,extra", [([0, 1], 1, 0), ([0, 3], 7, 2), ([0, 5, 5, 130, 131], 40, 0), ([0, 17, 64, 200], 257, 5), ([0, 0, 65], 520, 0), ([0, 300], 1000, 1), ([0, 64, 128, 256], 2056, 70),
                                             ([0] + [i // 2 for i in range(1, 300)] + [180], 48, 9), ([0, 9000], 33, 0), ([0, 512], 130, 0), ([0, 400, 512], 24, 1), ([5, 20, 12, 40, 1 << 30, -7, 60], 64, -50), ([0, 2], 40000, 0)])
def test_act_backward(offs, cols, extra, bf16):
    """dbias: up to 512 rows a chain of every sixteenth and four joins, at most 36; beyond, 8 rows, four joins, and chains of every 64th of the tiles of 32 rows, 3 + 7 joins: 40 + rows / 256 roundings of the terms at
    most, and those of the slope."""
    rng = np.random.default_rng([len(offs), cols])
    groups, rows = len(offs) - 1, offs[-1] + extra if extra >= 0 else 70
    g = expert_rows(offs, rows, groups)
    for pad, offset, act, into in ((0, 0, E.GELU, None), (8, 8, E.SILU, "dy"), (3, 1, E.RELU, "z"), (0, 0, E.NONE, None)):
        dy, z = (U.round_to(rng.normal(size=(rows, cols)), bf16) for _ in range(2))
        dz, dbias = act_backward(bf16, dy, act, z if act else None, offs, groups, pad, offset, into)
        parts = np.abs(E.phi(z)) + np.abs(z) if act == E.GELU else 1 + np.abs(z) if act == E.SILU else 1.0
        want = np.where((g >= 0)[:, None], dy * E.slope(z, act), 0.0)
        e = np.abs(dy) * (act_error(z, act, bf16) * parts) + 2 * R.U32 * np.abs(want)
        assert np.all(np.abs(dz - want) <= e + (R.UBF * np.abs(want) if bf16 else 0) + TINY)
        for k in range(groups):
            mine = g == k
            size = (np.abs(want[mine]) * (40 + rows / 256) * R.U32 + e[mine]).sum(0)
            assert np.all(np.abs(dbias[k] - want[mine].sum(0)) <= size + TINY), k
    alone = act_backward(bf16, dy, act, None, offs, groups, want_dz=False)
    assert np.array_equal(alone[1], dbias) and np.array_equal(alone[0], np.full_like(dz, 7.0))
    assert np.array_equal(act_backward(bf16, dy, act, None, offs, groups, want_dbias=False)[0], dz)


def test_act_backward_without_rows_and_experts():
    torch = U.torch_mod()
    offs, dbias = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.ones((3, 64), device="cuda")
    B.group_act_backward(B.BF16, 0, 64, E.GELU, 0, 64, offs.data_ptr(), 3, 0, 64, 0, 64, dbias.data_ptr(), 0, 0)
    torch.cuda.synchronize()
    assert not dbias.any()
    dy, dz = torch.ones((5, 64), device="cuda"), torch.ones((5, 64), device="cuda")
    B.group_act_backward(B.FP32, dy.data_ptr(), 64, E.NONE, 0, 0, offs.data_ptr(), 0, 5, 64, dz.data_ptr(), 64, dbias.data_ptr(), 0, 0)
    B.group_linear_act(B.BF16, 0, 64, dbias.data_ptr(), offs.data_ptr(), 3, 0, 64, 32, 0, E.GELU, 0, 32, 0, 32, 0, 32)
    w0 = torch.zeros(16, device="cuda")
    y = torch.ones((5, 64), device="cuda")
    B.group_linear_act(B.FP32, dy.data_ptr(), 64, 0, offs.data_ptr(), 0, 5, 64, 64, w0.data_ptr(), E.SILU, dy.data_ptr(), 64, 0, 0, y.data_ptr(), 64)
    torch.cuda.synchronize()
    assert not dz.any() and not y.any()


def test_rows_far_apart():
    """Rows 2^31 elements apart (bf16: 4 GiB), of every matrix of the epilogues."""
    torch = U.torch_mod()
    rows, n, stride = 3, 72, (1 << 31) + 8
    a, b, c = (torch.zeros((rows - 1) * stride + n, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    at = lambda t, r: t[r * stride:r * stride + n]  # noqa: E731
    for r in range(rows):
        at(a, r).fill_(r + 1)
        at(c, r).fill_(r + 1)
    offs, w, bias = torch.tensor([0, 1, 3], dtype=torch.int32, device="cuda"), torch.eye(n, device="cuda").bfloat16().repeat(2, 1, 1), torch.tensor([[-3.0], [10.0]], device="cuda").repeat(1, n)
    B.group_linear_act(B.BF16, a.data_ptr(), stride, w.data_ptr(), offs.data_ptr(), 2, rows, n, n, bias.data_ptr(), E.RELU, c.data_ptr(), stride, b.data_ptr(), stride,
                       c.data_ptr(), stride)
    torch.cuda.synchronize()
    assert [float(at(b, r)[n - 1]) for r in range(rows)] == [-2, 12, 13] and [float(at(c, r)[0]) for r in range(rows)] == [1, 14, 16]
    work = torch.zeros(B.group_act_backward_bytes(2, rows, n), dtype=torch.uint8, device="cuda")
    dbias = torch.zeros((2, n), device="cuda")
    B.group_act_backward(B.BF16, c.data_ptr(), stride, E.RELU, b.data_ptr(), stride, offs.data_ptr(), 2, rows, n, c.data_ptr(), stride, dbias.data_ptr(), work.data_ptr(), work.numel())
    B.group_linear_dgrad_act(B.BF16, c.data_ptr(), stride, w.data_ptr(), offs.data_ptr(), 2, rows, n, n, b.data_ptr(), stride, E.RELU, b.data_ptr(), stride, b.data_ptr(), stride)
    torch.cuda.synchronize()
    assert dbias[:, 5].tolist() == [0, 30] and [float(at(b, r)[3]) for r in range(rows)] == [0, 26, 29]
