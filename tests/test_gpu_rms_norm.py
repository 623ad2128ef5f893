"""The root-mean-square norm, its gradient and the 8-bit format (GPU) against 64-bit sums: lengths that end in every form of the kernels, odd
ones, strides, memory that is not 16-byte aligned, values that are not finite.

Bounds.  A lane adds at most 40 squares in a chain, and log2(64 * 16) more sums follow; with the divide, the root and the products an element of
y is off by at most half of 64 roundings (the root halves the sum's error) and a few more: 40 roundings of 2^-24, and one of the storage type."""
import numpy as np
import pytest

from paper_2102_10485_amd import binding as B
from tests import gpu_util as U
from tests import operators_ref as R

pytestmark = pytest.mark.gpu
EPS = 1e-5
SHAPES = [(1, 1), (3, 5), (2, 127), (5, 128), (7, 129), (4, 512), (3, 520), (9, 1000), (5, 2048), (3, 2056), (2, 4104), (2, 8192), (3, 8200),
          (1, 16384), (2, 16392), (2, 32776), (1, 40001)]


def matrix(a, bf16, stride, offset=0):
    """A device buffer whose row i starts at offset + i * stride; what lies between the rows is NaN."""
    torch = U.torch_mod()
    rows, cols = a.shape
    t = torch.full((offset + rows * stride + 8,), float("nan"), dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
    view = t[offset:offset + rows * stride].view(rows, stride)[:, :cols]
    view.copy_(torch.from_numpy(np.ascontiguousarray(a, np.float32)))
    return t, view, view.data_ptr()


def host(view):
    return view.float().cpu().numpy()


def forward(x, residual, gain, bf16, pad=0, offset=0, eight=False):
    torch = U.torch_mod()
    rows, cols = x.shape
    st = cols + pad
    kind = torch.bfloat16 if bf16 else torch.float32
    _, _, px = mx = matrix(x, bf16, st, offset)
    mr = matrix(residual, bf16, st, offset) if residual is not None else None
    ms, my = (matrix(np.zeros_like(x), bf16, st, offset) for _ in range(2))
    inv = torch.zeros(rows, device="cuda")
    g = torch.from_numpy(gain).cuda()
    wide = R.padded(cols)
    q, sc = (torch.full(s, 77, dtype=torch.uint8, device="cuda") for s in ((rows, wide), (rows, wide // 128)))
    B.rms_norm(B.BF16 if bf16 else B.FP32, px, st, mr[2] if mr else 0, st, g.data_ptr(), EPS, rows, cols, ms[2], st, my[2], st,
               q.data_ptr() if eight else 0, sc.data_ptr() if eight else 0, inv.data_ptr())
    torch.cuda.synchronize()
    for whole, view, _ in (ms, my):                              # nothing is written between the rows or behind them
        rest = whole.clone()
        rest[offset:offset + rows * st].view(rows, st)[:, :cols] = float("nan")
        assert bool(rest.isnan().all())
    assert kind == my[1].dtype
    return host(ms[1]), host(my[1]), inv.cpu().numpy(), q.cpu().numpy(), sc.cpu().numpy()


def inputs(rows, cols, bf16, seed):
    rng = np.random.default_rng([rows, cols, seed])
    x, r = (U.round_to(rng.normal(size=(rows, cols)) * np.exp(rng.normal(size=cols)), bf16) for _ in range(2))
    return x, r, rng.normal(1, 0.2, cols).astype(np.float32)


def bound(bf16):
    return 40 * R.U32 + (R.UBF if bf16 else 0)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_forward(rows, cols, bf16):
    for pad, offset, with_residual in ((0, 0, True), (8, 8, False), (3, 1, True)):
        x, r, gain = inputs(rows, cols, bf16, pad)
        r = r if with_residual else None
        s, y, inv, q, sc = forward(x, r, gain, bf16, pad, offset, eight=True)
        es, einv, ey = R.norm(x, r, gain, EPS, lambda v: U.round_to(v, bf16))
        assert np.array_equal(s, es.astype(np.float32))
        assert np.all(np.abs(inv - einv) <= 40 * R.U32 * einv)
        assert np.all(np.abs(y - ey) <= bound(bf16) * np.abs(ey))
        # 8 bits: the least scale that holds the block (up to y's own error), codes to the nearest, zeros behind the last column
        wide = np.zeros((rows, R.padded(cols)))
        wide[:, :cols] = ey
        top, full = np.abs(wide).reshape(rows, -1, 128).max(-1), 448 * 2.0 ** (sc.astype(np.float64) - 127)
        assert np.all(top <= full * (1 + 1e-5)) and np.all((top * (1 + 1e-5) > full / 2) | (sc == 1))
        ulp = np.maximum(np.exp2(np.floor(np.log2(np.maximum(np.abs(wide), 1e-300)))), np.repeat(full / 448, 128, -1) * 2.0 ** -6) / 8
        assert np.all(np.abs(R.decode(q, sc) - wide) <= 0.5 * ulp + 40 * R.U32 * np.abs(wide))
        assert not q[:, cols:].any()


def test_zero_rows_and_rows_of_zeros():
    torch = U.torch_mod()
    x = np.zeros((3, 300), np.float32)
    s, y, inv, q, sc = forward(x, None, np.ones(300, np.float32), True, eight=True)
    assert not y.any() and not q.any() and np.all(sc == 1) and np.allclose(inv, EPS ** -0.5, rtol=1e-6)
    t = torch.zeros(1, device="cuda")
    B.rms_norm(B.FP32, t.data_ptr(), 64, 0, 0, t.data_ptr(), EPS, 0, 64, 0, 0, t.data_ptr(), 64, 0, 0, 0)
    dg = torch.ones(64, device="cuda")
    B.rms_norm_backward(B.FP32, t.data_ptr(), 64, t.data_ptr(), 64, t.data_ptr(), t.data_ptr(), 0, 0, 0, 64, t.data_ptr(), 64, dg.data_ptr(), 0, 0)
    assert not dg.cpu().numpy().any()


@pytest.mark.parametrize("cols", [96, 1024, 4096, 40000])
def test_values_that_are_not_finite_stay_in_their_rows(cols):
    x, r, gain = inputs(4, cols, True, 9)
    clean = forward(x, r, gain, True, eight=True)
    x[1, cols // 2], x[2, 0] = np.inf, np.nan
    s, y, inv, q, sc = forward(x, r, gain, True, eight=True)
    for a, b in zip((s, y, inv, q, sc), clean):
        assert np.array_equal(a[[0, 3]], b[[0, 3]])
    # an infinity: the norm is infinite, finite values become zero, the infinity NaN; a NaN: the whole row
    assert inv[1] == 0 and np.isnan(y[1, cols // 2]) and not np.delete(y[1], cols // 2).any()
    assert q[1, cols // 2] & 0x7F == 0x7F and not (np.delete(q[1], cols // 2) & 0x7F).any()
    assert np.isnan(y[2]).all() and np.all(q[2, :cols] & 0x7F == 0x7F)


@pytest.mark.parametrize("bf16", [False, True])
def test_quantize8_is_the_format(bf16):
    torch = U.torch_mod()
    rng = np.random.default_rng(3)
    for rows, cols, pad in ((1, 1, 0), (5, 128, 0), (4, 1000, 0), (3, 129, 2), (70, 640, 0)):
        x = rng.normal(size=(rows, cols)) * np.exp(3 * rng.normal(size=(rows, cols)))
        x[rng.random(x.shape) < 0.1] = 0
        x = U.round_to(x, bf16)
        x[0, 0] = 448 if cols == 128 else x[0, 0]
        if rows > 3:
            x[1, cols // 2], x[2, 1], x[3, 0] = np.inf, -np.inf, np.nan
        whole, view, p = matrix(x, bf16, cols + pad)
        wide = R.padded(cols)
        q, sc = (torch.full(s, 77, dtype=torch.uint8, device="cuda") for s in ((rows, wide), (rows, wide // 128)))
        B.quantize8(B.BF16 if bf16 else B.FP32, p, cols + pad, rows, cols, q.data_ptr(), sc.data_ptr())
        full = np.zeros((rows, wide), np.float32)
        full[:, :cols] = x
        es = R.scale_bytes(full)
        assert np.array_equal(sc.cpu().numpy(), es)
        got, want = q.cpu().numpy(), R.nearest_codes(full, es)
        assert np.array_equal(got & 0x7F, want & 0x7F)
        assert np.array_equal(got[np.isfinite(full)], want[np.isfinite(full)])


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,cols", SHAPES + [(70, 40), (1030, 264), (300, 2500), (70, 17000)])
def test_backward(rows, cols, bf16):
    torch = U.torch_mod()
    for pad, offset, with_dsum in ((0, 0, True), (8, 8, False), (5, 1, True)):
        rng = np.random.default_rng([rows, cols, pad, 1])
        s, _, gain = inputs(rows, cols, bf16, 5)
        dy, ds = (U.round_to(rng.normal(size=(rows, cols)), bf16) for _ in range(2))
        st = cols + pad
        ms, mdy, mds, mdx = (matrix(a, bf16, st, offset) for a in (s, dy, ds, np.zeros_like(s)))
        inv = torch.from_numpy((1 / np.sqrt((s.astype(np.float64) ** 2).mean(1) + EPS)).astype(np.float32)).cuda()
        g, dg, n = torch.from_numpy(gain).cuda(), torch.zeros(cols, device="cuda"), B.rms_norm_backward_bytes(rows, cols)
        work = torch.full((n // 4,), float("nan"), device="cuda")
        B.rms_norm_backward(B.BF16 if bf16 else B.FP32, mdy[2], st, ms[2], st, g.data_ptr(), inv.data_ptr(), mds[2] if with_dsum else 0, st, rows, cols,
                            mdx[2], st, dg.data_ptr(), work.data_ptr(), n)
        edx, edg, size, gsize = R.norm_backward(dy, s, gain, EPS, ds if with_dsum else None)
        dx = host(mdx[1])
        # (inv as given carries one rounding, its square and the mean's chain the rest)
        assert np.all(np.abs(dx - edx) <= 64 * R.U32 * size + (R.UBF * np.abs(edx) if bf16 else 0))
        # a lane adds at most rows / blocks terms, then 32 chains of at most 32 partial sums are joined
        assert np.all(np.abs(dg.cpu().numpy() - edg) <= (min(rows, 8) + 4 + 64 + 4) * R.U32 * gsize)


def test_gradient_against_differences():
    """Central differences of the forward kernel's own fp32 output along random directions: h = 2^-7 leaves h^2/6 of the third derivative
    (below 1e-4 of the gradient's size) and 2^-24 / h = 8e-6 of rounding."""
    torch = U.torch_mod()
    rng = np.random.default_rng(0)
    rows, cols, h = 6, 200, 2.0 ** -7
    x, d, w = (rng.normal(size=(rows, cols)).astype(np.float32) for _ in range(3))
    gain, dgain_dir = rng.normal(1, 0.2, cols).astype(np.float32), rng.normal(size=cols).astype(np.float32)

    def value(x, gain):
        return float((forward(x.astype(np.float32), None, gain.astype(np.float32), False)[1].astype(np.float64) * w).sum())

    tx, tg, tw = (torch.from_numpy(a).cuda() for a in (x, gain, w))
    inv = torch.from_numpy(forward(x, None, gain, False)[2]).cuda()
    dx, dg, n = torch.zeros_like(tx), torch.zeros_like(tg), B.rms_norm_backward_bytes(rows, cols)
    work = torch.zeros(n, dtype=torch.uint8, device="cuda")
    B.rms_norm_backward(B.FP32, tw.data_ptr(), cols, tx.data_ptr(), cols, tg.data_ptr(), inv.data_ptr(), 0, 0, rows, cols, dx.data_ptr(), cols, dg.data_ptr(),
                        work.data_ptr(), n)
    dx, dg = dx.cpu().numpy().astype(np.float64), dg.cpu().numpy().astype(np.float64)
    along_x = (value(x + h * d, gain) - value(x - h * d, gain)) / (2 * h)
    along_g = (value(x, gain + h * dgain_dir) - value(x, gain - h * dgain_dir)) / (2 * h)
    assert abs(along_x - (dx * d).sum()) <= 1e-3 * np.linalg.norm(dx) * np.linalg.norm(d)
    assert abs(along_g - (dg * dgain_dir).sum()) <= 1e-3 * np.linalg.norm(dg) * np.linalg.norm(dgain_dir)


@pytest.mark.parametrize("cols", [512, 4096, 40000])
def test_in_place(cols):
    """sum over x, y over the residual's... and dx over dy: the same bits as with memory of their own."""
    torch = U.torch_mod()
    x, r, gain = inputs(5, cols, True, 2)
    s, y, inv, _, _ = forward(x, r, gain, True)
    tx, tr = (torch.from_numpy(a).cuda().bfloat16() for a in (x, r))
    tg, ty, tinv = torch.from_numpy(gain).cuda(), torch.empty_like(tx), torch.empty(5, device="cuda")
    B.rms_norm(B.BF16, tx.data_ptr(), cols, tr.data_ptr(), cols, tg.data_ptr(), EPS, 5, cols, tx.data_ptr(), cols, ty.data_ptr(), cols, 0, 0, tinv.data_ptr())
    assert np.array_equal(host(tx), s) and np.array_equal(host(ty), y)
    n = B.rms_norm_backward_bytes(5, cols)
    work, dx, dg, dg2 = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty_like(tx), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    B.rms_norm_backward(B.BF16, ty.data_ptr(), cols, tx.data_ptr(), cols, tg.data_ptr(), tinv.data_ptr(), tr.data_ptr(), cols, 5, cols, dx.data_ptr(), cols,
                        dg.data_ptr(), work.data_ptr(), n)
    B.rms_norm_backward(B.BF16, ty.data_ptr(), cols, tx.data_ptr(), cols, tg.data_ptr(), tinv.data_ptr(), tr.data_ptr(), cols, 5, cols, ty.data_ptr(), cols,
                        dg2.data_ptr(), work.data_ptr(), n)
    assert torch.equal(dx, ty) and torch.equal(dg, dg2)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("cols", [512, 1536, 4096, 8192, 16384, 40000])
def test_results_of_many_megabytes_are_those_of_each_row(cols, bf16):
    """Twelve rows again and again, more than 64 MiB of them: each has the bits that a call on the twelve gives, forward, into 8 bits and backward."""
    torch = U.torch_mod()
    kind, e, n = (torch.bfloat16, 2, 12) if bf16 else (torch.float32, 4, 12)
    times = 80 * 2 ** 20 // (n * cols * e) + 1
    x, r, gain = inputs(n, cols, bf16, 4)
    dy = U.round_to(np.random.default_rng(cols).normal(size=(n, cols)), bf16)
    g = torch.from_numpy(gain).cuda()

    def run(times):
        rows, wide = n * times, R.padded(cols)
        tx, tr, tdy = (torch.from_numpy(a).to(kind).cuda().repeat(times, 1) for a in (x, r, dy))
        s, y, dx = (torch.full_like(tx, float("nan")) for _ in range(3))
        q, sc = (torch.full(k, 77, dtype=torch.uint8, device="cuda") for k in ((rows, wide), (rows, wide // 128)))
        inv = torch.zeros(rows, device="cuda")
        precision = B.BF16 if bf16 else B.FP32
        B.rms_norm(precision, tx.data_ptr(), cols, tr.data_ptr(), cols, g.data_ptr(), EPS, rows, cols, s.data_ptr(), cols, y.data_ptr(), cols, q.data_ptr(),
                   sc.data_ptr(), inv.data_ptr())
        B.rms_norm_backward(precision, tdy.data_ptr(), cols, s.data_ptr(), cols, g.data_ptr(), inv.data_ptr(), tr.data_ptr(), cols, rows, cols, dx.data_ptr(),
                            cols, 0, 0, 0)
        return s, y, q, sc, inv, dx

    for one, many in zip(run(1), run(times)):
        assert bool((many.view(times, *one.shape) == one).all())


@pytest.mark.parametrize("bits,cols", [(26, 8), (24, 1032), (22, 4104)])
def test_more_rows_than_a_launch_has_threads_for(bits, cols):
    """2^26 rows of a wave, 2^24 of four and 2^22 of sixteen are 2^32 threads, more than one launch can have.  The same 1021 rows again and again, y over x (34 GB of
    the longer rows): each has the bits that a call on them alone gives; codes and scales of the shortest too."""
    torch = U.torch_mod()
    n = 1021
    times = (1 << bits) // n + 2
    x, _, gain = inputs(n, cols, True, 6)
    g = torch.from_numpy(gain).cuda()

    def run(times):
        rows, wide, eight = n * times, R.padded(cols), cols < 128
        t = torch.empty((times, n, cols), dtype=torch.bfloat16, device="cuda")
        t[:] = torch.from_numpy(x).cuda().bfloat16()
        inv = torch.zeros((times, n), device="cuda")
        q, sc = (torch.full((times, n, k), 77, dtype=torch.uint8, device="cuda") if eight else None for k in (wide, wide // 128))
        B.rms_norm(B.BF16, t.data_ptr(), cols, 0, 0, g.data_ptr(), EPS, rows, cols, 0, 0, t.data_ptr(), cols, q.data_ptr() if eight else 0,
                   sc.data_ptr() if eight else 0, inv.data_ptr())
        return [t, inv] + ([q, sc] if eight else [])

    for one, many in zip(run(1), run(times)):
        for k in range(0, times, 4096):
            assert bool((many[k:k + 4096] == one).all())


def test_gradient_of_more_rows_than_a_launch_has_threads_for():
    """The gradient of 2^26 rows, its sums by column included: the same rows again and again, whole numbers of which the sums are exact."""
    torch = U.torch_mod()
    cols, rows = 8, (1 << 26) + 5
    s = torch.full((rows, cols), 2.0, dtype=torch.bfloat16, device="cuda")
    dy = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    dy[::4099, 3] = 1.0
    inv, g, dg, n = torch.full((rows,), 0.5, device="cuda"), torch.ones(cols, device="cuda"), torch.zeros(cols, device="cuda"), B.rms_norm_backward_bytes(rows, cols)
    work = torch.empty(n, dtype=torch.uint8, device="cuda")
    B.rms_norm_backward(B.BF16, dy.data_ptr(), cols, s.data_ptr(), cols, g.data_ptr(), inv.data_ptr(), 0, 0, rows, cols, dy.data_ptr(), cols, dg.data_ptr(),
                        work.data_ptr(), n)
    want = np.zeros(cols)
    want[3] = -(-rows // 4099)
    assert np.array_equal(dg.cpu().numpy(), want)
    # inv * (h - s * inv^2 * mean(h s)) = (h - 1/8) / 2 in the rows that have a gradient
    row = torch.tensor([-0.0625] * 3 + [0.4375] + [-0.0625] * 4, device="cuda").bfloat16()
    assert bool((dy[::4099] == row).all()) and int((dy != 0).sum()) == 8 * int(want[3])


@pytest.mark.parametrize("bf16", [False, True])
def test_gain_of_more_columns_than_a_launch_has_threads_for(bf16):
    """2^27 columns and some: 32 columns a block of 1024 threads are 2^32 threads and more.  Whole numbers: sums are exact."""
    torch = U.torch_mod()
    cols, kind = (1 << 27) + 40, torch.bfloat16 if bf16 else torch.float32
    s, inv = torch.full((2, cols), 2.0, device="cuda").to(kind), torch.tensor([0.5, 0.25], device="cuda")
    dy = (torch.arange(2 * cols, device="cuda") % 8).view(2, cols).to(kind)
    gain, dx, dg = torch.zeros(cols, device="cuda"), torch.zeros((2, cols), device="cuda").to(kind), torch.full((cols,), float("nan"), device="cuda")
    n = B.rms_norm_backward_bytes(2, cols)
    work = torch.empty(n, dtype=torch.uint8, device="cuda")
    B.rms_norm_backward(B.BF16 if bf16 else B.FP32, dy.data_ptr(), cols, s.data_ptr(), cols, gain.data_ptr(), inv.data_ptr(), 0, 0, 2, cols, dx.data_ptr(), cols,
                        dg.data_ptr(), work.data_ptr(), n)
    assert torch.equal(dg, dy[0].float() + 0.5 * dy[1].float()) and not bool(dx.any())


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("cols", [1, 96, 129, 1000, 1032, 4104, 16392, 40001])
def test_padding_is_zero_whatever_the_row_holds(cols, bf16):
    """A row with a NaN, one with an infinity, and (eps 0) one of zeros, whose norm is 0/0: codes behind the last column are zero in all of them."""
    torch = U.torch_mod()
    x, _, gain = inputs(4, cols, bf16, 3)
    x[0, cols // 2], x[1, 0], x[2] = np.nan, np.inf, 0
    wide, g = R.padded(cols), torch.from_numpy(gain).cuda()
    for pad, offset in ((0, 0), (3, 1)):
        _, view, p = matrix(x, bf16, cols + pad, offset)
        q, sc = (torch.full(s, 77, dtype=torch.uint8, device="cuda") for s in ((4, wide), (4, wide // 128)))
        B.rms_norm(B.BF16 if bf16 else B.FP32, p, cols + pad, 0, 0, g.data_ptr(), 0.0, 4, cols, 0, 0, 0, 0, q.data_ptr(), sc.data_ptr(), 0)
        q, sc = q.cpu().numpy(), sc.cpu().numpy()
        assert not q[:, cols:].any()
        assert np.all(q[[0, 2], :cols] & 0x7F == 0x7F) and q[1, 0] & 0x7F == 0x7F and np.all(np.isfinite(R.decode(q, sc)[3]))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("cols", [96, 1000, 4096, 16392])
def test_backward_of_tiny_rows(cols, bf16):
    """Without eps, rows of 1e-20 have inv_rms of 1e20, whose square is no fp32 number; their gradient is.  Bounds as in test_backward."""
    torch = U.torch_mod()
    s, _, gain = inputs(3, cols, bf16, 8)
    s = U.round_to(s * np.float32(1e-20), bf16)
    dy = U.round_to(np.random.default_rng(cols).normal(size=s.shape), bf16)
    edx, edg, size, gsize = R.norm_backward(dy, s, gain, 0.0, None)
    inv = torch.from_numpy((1 / np.sqrt((s.astype(np.float64) ** 2).mean(1))).astype(np.float32)).cuda()
    ms, mdy, mdx = (matrix(a, bf16, cols) for a in (s, dy, np.zeros_like(s)))
    g, dg, n = torch.from_numpy(gain).cuda(), torch.zeros(cols, device="cuda"), B.rms_norm_backward_bytes(3, cols)
    work = torch.zeros(n, dtype=torch.uint8, device="cuda")
    B.rms_norm_backward(B.BF16 if bf16 else B.FP32, mdy[2], cols, ms[2], cols, g.data_ptr(), inv.data_ptr(), 0, 0, 3, cols, mdx[2], cols, dg.data_ptr(), work.data_ptr(), n)
    assert np.all(np.abs(host(mdx[1]) - edx) <= 64 * R.U32 * size + (R.UBF * np.abs(edx) if bf16 else 0))
    assert np.all(np.abs(dg.cpu().numpy() - edg) <= (3 + 4 + 64 + 4) * R.U32 * gsize)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,cols", [(5003, 264), (5003, 1000), (3001, 1536), (1501, 2500), (1501, 8192), (701, 16384), (201, 16400)])
def test_backward_of_several_rows_a_block(rows, cols, bf16):
    """More rows than all blocks have at a time, in every form of the kernel, and not a multiple of them.  A lane adds the terms of its rows in a chain, four waves are joined where a
    row is a wave's, and the blocks' partial sums are added in 32 chains that are joined; a term has four roundings."""
    torch = U.torch_mod()
    for pad, offset, with_dsum in ((0, 0, True), (3, 1, False)):
        rng = np.random.default_rng([rows, cols, pad, 2])
        s, _, gain = inputs(rows, cols, bf16, 11)
        dy, ds = (U.round_to(rng.normal(size=(rows, cols)), bf16) for _ in range(2))
        st, n = cols + pad, B.rms_norm_backward_bytes(rows, cols)
        blocks, at_a_time = n // (4 * cols), 4 if cols <= 1024 else 1
        chain = -(-rows // (blocks * at_a_time))
        assert chain > 1 and rows % (blocks * at_a_time)
        ms, mdy, mds, mdx = (matrix(a, bf16, st, offset) for a in (s, dy, ds, np.zeros_like(s)))
        inv = torch.from_numpy((1 / np.sqrt((s.astype(np.float64) ** 2).mean(1) + EPS)).astype(np.float32)).cuda()
        g, dg = torch.from_numpy(gain).cuda(), torch.full((cols,), float("nan"), device="cuda")
        work = torch.full((n // 4,), float("nan"), device="cuda")
        B.rms_norm_backward(B.BF16 if bf16 else B.FP32, mdy[2], st, ms[2], st, g.data_ptr(), inv.data_ptr(), mds[2] if with_dsum else 0, st, rows, cols, mdx[2], st,
                            dg.data_ptr(), work.data_ptr(), n)
        edx, edg, size, gsize = R.norm_backward(dy, s, gain, EPS, ds if with_dsum else None)
        assert np.all(np.abs(host(mdx[1]) - edx) <= 64 * R.U32 * size + (R.UBF * np.abs(edx) if bf16 else 0))
        assert np.all(np.abs(dg.cpu().numpy() - edg) <= (4 + chain + 4 + -(-blocks // 32) + 32) * R.U32 * gsize)
