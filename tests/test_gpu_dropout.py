"""Dropout (GPU) against the generator's definition: every element, odd widths, strides and alignments, what is dropped, in place, in a graph, and places beyond 2^32.

Bounds: the factor is rounded to fp32, the product and the sum once each: 3 roundings of 2^-24 of the terms; and one of the storage type."""
import numpy as np
import pytest

from paper_2102_10485_amd import binding as B
from tests import experts_ref as E
from tests import gpu_util as U
from tests import operators_ref as R
from tests.test_gpu_rms_norm import host, matrix

pytestmark = pytest.mark.gpu
SEED = 0xFEDCBA9876543210
SHAPES = [(1, 1), (3, 7), (2, 8), (5, 9), (17, 64), (33, 100), (9, 1000), (700, 8), (600, 3), (3, 4104), (2, 32776), (2, 40001), (257, 264)]


def run(x, residual, bf16, p, pad=0, offset=0, site=0, step=0, into=None):
    torch = U.torch_mod()
    rows, cols = x.shape
    st = cols + pad
    mx = matrix(x, bf16, st, offset)
    mr = matrix(residual, bf16, st, offset) if residual is not None else None
    my = {None: matrix(np.zeros_like(x), bf16, st, offset), "x": mx, "residual": mr}[into]
    B.dropout(B.BF16 if bf16 else B.FP32, mx[2], st, mr[2] if mr else 0, st, rows, cols, p, SEED, site, step, 0, my[2], st)
    torch.cuda.synchronize()
    rest = my[0].clone()
    rest[offset:offset + rows * st].view(rows, st)[:, :cols] = float("nan")
    assert bool(rest.isnan().all())                                   # nothing is written between the rows or behind them
    return host(my[1])


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_every_element(rows, cols, bf16):
    for pad, offset, p, with_residual, into in ((0, 0, 0.1, True, None), (8, 8, 0.5, False, "x"), (3, 1, 0.25, True, "residual"), (0, 0, 0.0, True, None), (1, 0, 0.999, False, None)):
        rng = np.random.default_rng([rows, cols, pad])
        x, r = (U.round_to(rng.normal(size=(rows, cols)), bf16) for _ in range(2))
        keep, scale = E.keep(rows, cols, p, SEED, 7, 123456)
        kept = np.where(keep, x * scale, 0)
        want = kept + (r if with_residual else 0)
        got = run(x, r if with_residual else None, bf16, p, pad, offset, 7, 123456, into)
        size = np.abs(kept) + (np.abs(r) if with_residual else 0)
        assert np.all(np.abs(got - want) <= 3 * R.U32 * size + (R.UBF * np.abs(want) if bf16 else 0))
        if not with_residual:
            assert np.array_equal(got != 0, keep & (x != 0))


@pytest.mark.parametrize("bf16", [False, True])
def test_what_is_dropped_is_gone(bf16):
    """Infinities and NaN among the dropped reach nothing; among the kept they stay."""
    x = np.full((20, 40), np.nan, np.float32)
    x[::2] = np.inf
    keep, _ = E.keep(20, 40, 0.5, SEED, 0, 0)
    got = run(x, None, bf16, 0.5)
    assert np.array_equal(got[~keep], np.zeros((~keep).sum())) and np.array_equal(np.isnan(got), keep & np.isnan(x)) and np.array_equal(np.isinf(got), keep & np.isinf(x))
    got = run(x, np.ones_like(x), bf16, 0.5)
    assert np.array_equal(got[~keep], np.ones((~keep).sum()))


def test_gradient_and_graph():
    """The same call on the gradient has the same mask; a captured one has the next step's mask at every replay."""
    torch = U.torch_mod()
    rows, cols = 50, 136
    x, y, dy, dx = (torch.ones((rows, cols), device="cuda") for _ in range(4))
    step = torch.zeros(1, dtype=torch.int32, device="cuda")
    stream = torch.cuda.Stream()

    def both():
        s = torch.cuda.current_stream().cuda_stream
        B.dropout(B.FP32, x.data_ptr(), cols, 0, 0, rows, cols, 0.3, SEED, 2, 10, step.data_ptr(), y.data_ptr(), cols, s)
        B.dropout(B.FP32, dy.data_ptr(), cols, 0, 0, rows, cols, 0.3, SEED, 2, 10, step.data_ptr(), dx.data_ptr(), cols, s)

    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        both()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
        step += 1
    step.fill_(-3)                                                    # (the sum is taken modulo 2^32)
    for t in range(4):
        graph.replay()
        torch.cuda.synchronize()
        keep, scale = E.keep(rows, cols, 0.3, SEED, 2, 10 - 3 + t)
        assert np.array_equal(y.cpu().numpy(), np.where(keep, np.float32(scale), 0)) and torch.equal(y, dx)


def test_places_beyond_2_32():
    """2^30 rows of 36 columns are 5 * 2^30 groups of eight: places of more than 32 bits, 77 GB, in place."""
    torch = U.torch_mod()
    rows, cols = 1 << 30, 36
    x = torch.ones(rows * cols, dtype=torch.bfloat16, device="cuda").view(rows, cols)
    B.dropout(B.BF16, x.data_ptr(), cols, 0, 0, rows, cols, 0.4, SEED, 1, 2, 0, x.data_ptr(), cols)
    torch.cuda.synchronize()
    for first in (0, (1 << 32) // 5 - 50, rows - 100):
        keep, scale = E.keep(np.arange(first, first + 100), cols, 0.4, SEED, 1, 2)
        assert np.array_equal(x[first:first + 100].float().cpu().numpy(), np.where(keep, U.round_to(np.float32(scale), True), 0)), first


def test_rows_far_apart():
    """Rows 2^31 elements apart (bf16: 4 GiB)."""
    torch = U.torch_mod()
    rows, cols, stride = 3, 72, (1 << 31) + 8
    x = torch.zeros(2 * stride + cols, dtype=torch.bfloat16, device="cuda")
    for r in range(rows):
        x[r * stride:r * stride + cols] = r + 1
    B.dropout(B.BF16, x.data_ptr(), stride, 0, 0, rows, cols, 0.5, SEED, 0, 0, 0, x.data_ptr(), stride)
    torch.cuda.synchronize()
    keep, scale = E.keep(rows, cols, 0.5, SEED, 0, 0)
    for r in range(rows):
        assert np.array_equal(x[r * stride:r * stride + cols].float().cpu().numpy(), np.where(keep[r], scale * (r + 1), 0).astype(np.float32))
