"""AdamW over many tensors (GPU).  Every operation is rounded to fp32 on its own, so the same operations in numpy give the same bits: no tolerance."""
import numpy as np
import pytest

from paper_2102_10485_amd import binding as B
from tests import gpu_util as U
from tests import operators_ref as R

pytestmark = pytest.mark.gpu
HYPER = dict(lr=2e-4, beta1=0.9, beta2=0.999, eps=1e-8)


class Both:
    """The kernel's tensors and numpy's side by side."""

    def __init__(self, sizes, bf16, bits, copies=True, decay=True, offset=0, seed=0, scale=1e-2):
        torch = self.torch = U.torch_mod()
        rng = self.rng = np.random.default_rng([seed, len(sizes), bits])
        self.sizes, self.bf16, self.eight, self.offset, self.scale = sizes, bf16, bits == 8, offset, scale
        self.blocks = [-(-n // 128) for n in sizes]
        self.first = np.concatenate([[0], np.cumsum(self.blocks)]) * 128
        assert B.adamw_blocks(sizes) == sum(self.blocks)
        total = int(self.first[-1])
        kind = torch.bfloat16 if bf16 else torch.float32

        def own(dtype):                                             # every tensor in memory of its own, `offset` elements from its start
            return [torch.full((n + offset + 3,), float("nan"), dtype=dtype, device="cuda") for n in sizes]

        self.p, self.g, self.c = own(torch.float32), own(kind), own(torch.bfloat16) if copies else None
        self.np_p = [rng.normal(size=n).astype(np.float32) for n in sizes]
        for t, a in zip(self.p, self.np_p):
            t[offset:offset + a.size] = torch.from_numpy(a)
        dt = torch.uint8 if self.eight else torch.float32
        self.m, self.v = (torch.zeros(total, dtype=dt, device="cuda") for _ in range(2))
        self.ms, self.vs = (torch.zeros(total // 128, dtype=torch.uint8, device="cuda") if self.eight else None for _ in range(2))
        self.decay = [0.1 * (i % 3) for i in range(len(sizes))] if decay else None
        at = lambda ts: [t.data_ptr() + offset * t.element_size() for t in ts]  # noqa: E731
        self.plan = B.AdamW(sizes, at(self.p), at(self.g), B.BF16 if bf16 else B.FP32, at(self.c) if copies else None, self.decay, bits, self.m.data_ptr(),
                            self.v.data_ptr(), self.ms.data_ptr() if self.eight else 0, self.vs.data_ptr() if self.eight else 0)
        self.np_m, self.np_v = (np.zeros(total, np.uint8 if self.eight else np.float32) for _ in range(2))
        self.np_ms, self.np_vs = (np.zeros(total // 128, np.uint8) for _ in range(2))

    def step(self, t, seed=3, special=None):
        o = self.offset
        for k, n in enumerate(self.sizes):
            g = U.round_to((self.rng.normal(size=n) * self.scale * np.exp(2 * self.rng.normal(size=n))).astype(np.float32), self.bf16)
            if special is not None and n > 5:
                g[:len(special)] = special
            self.g[k][o:o + n] = self.torch.from_numpy(g)
            a, b = int(self.first[k]), int(self.first[k + 1])
            r = R.adamw(self.np_p[k], g, self.np_m[a:b], self.np_v[a:b], self.np_ms[a // 128:b // 128], self.np_vs[a // 128:b // 128],
                        self.decay[k] if self.decay else 0.0, step=t, seed=seed, eight=self.eight, first=a, **HYPER)
            self.np_p[k], self.np_m[a:b], self.np_v[a:b] = r[:3]
            if self.eight:
                self.np_ms[a // 128:b // 128], self.np_vs[a // 128:b // 128] = r[3:]
        self.plan.step(HYPER["lr"], HYPER["beta1"], HYPER["beta2"], HYPER["eps"], t, seed)

    def check(self):
        o = self.offset
        same = lambda a, b: np.array_equal(a, b, equal_nan=a.dtype.kind == "f")  # noqa: E731
        for k, n in enumerate(self.sizes):
            whole = self.p[k].cpu().numpy()
            assert same(whole[o:o + n], self.np_p[k]), k
            assert np.isnan(whole[:o]).all() and np.isnan(whole[o + n:]).all()
            if self.c is not None:
                c = self.c[k].float().cpu().numpy()
                assert same(c[o:o + n], U.round_to(self.np_p[k], True)) and np.isnan(c[:o]).all() and np.isnan(c[o + n:]).all()
        assert same(self.m.cpu().numpy(), self.np_m) and same(self.v.cpu().numpy(), self.np_v)
        if self.eight:
            assert same(self.ms.cpu().numpy(), self.np_ms) and same(self.vs.cpu().numpy(), self.np_vs)


SIZES = [[1], [128], [5, 0, 129, 127, 2048], [2049, 3, 10000], [7] * 40 + [4096] * 3]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("case", range(len(SIZES)))
def test_steps(case, bf16, bits):
    for offset, copies, decay in ((0, True, True), (1, True, False), (4, False, True)):
        b = Both(SIZES[case], bf16, bits, copies, decay, offset)
        for t in (1, 2, 3):
            b.step(t)
        b.check()


@pytest.mark.parametrize("bits", [32, 8])
def test_late_steps_and_small_gradients(bits):
    b = Both([3000, 17], False, bits, scale=1e-9)
    for t in (100000, 100001):
        b.step(t, seed=0xFFFFFFFF)
    b.check()


@pytest.mark.parametrize("bits", [32, 8])
def test_gradients_that_are_not_finite(bits):
    """They reach their own values' moments and parameter alone; a block's scale follows from its finite values."""
    b = Both([300, 129], False, bits)
    b.step(1)
    b.step(2, special=[np.inf, -np.inf, np.nan, 0, 3e38])
    b.step(3)
    b.check()
    p = b.p[0].cpu().numpy()
    assert np.isnan(p[:3]).all() and np.isfinite(p[5:300]).all()


def test_zero_gradients_change_nothing():
    b = Both([200], False, 8, decay=False)
    before = b.np_p[0].copy()
    b.scale = 0.0
    b.step(1)
    b.check()
    assert np.array_equal(b.p[0].cpu().numpy()[:200], before) and not b.m.cpu().numpy().any() and not (b.v.cpu().numpy() & 0x7F).any()


def test_eight_bit_moments_follow_the_32_bit_ones():
    """A constant |gradient| after moments of four times it: sqrt(v) has to come down to it, by 0.05 % a step.  Rounding to nearest would hold it where it is.
    The mean over 4096 values: each is a random walk of steps of one code (1/8 of its binade at most) around the exact moment, pulled back as fast as
    the moment moves, whose variance stays below a code times the moment / 2: deviation of the mean below 0.35 / sqrt(4096) = 0.6 %."""
    torch = U.torch_mod()
    n, steps = 4096, 1500
    p, g = torch.zeros(n, device="cuda"), torch.full((n,), 1e-3, device="cuda")
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    ms, vs = (torch.zeros(n // 128, dtype=torch.uint8, device="cuda") for _ in range(2))
    plan = B.AdamW([n], [p.data_ptr()], [g.data_ptr()], B.FP32, None, None, 8, m.data_ptr(), v.data_ptr(), ms.data_ptr(), vs.data_ptr())
    start = np.full((n // 128, 128), 4e-3, np.float32)
    sb = R.scale_bytes(start)
    v.copy_(torch.from_numpy(R.nearest_codes(start, sb).ravel()))
    vs.copy_(torch.from_numpy(sb.ravel()))
    exact = float(R.decode(R.nearest_codes(start, sb), sb)[0, 0]) ** 2
    for t in range(1, steps + 1):
        plan.step(1e-4, 0.9, 0.999, 1e-8, t, 77)
        exact = 0.999 * exact + 0.001 * 1e-6
    root = R.decode(v.cpu().numpy().reshape(-1, 128), vs.cpu().numpy()[:, None])
    # (the mean of the squares: rounding a root by chance adds its variance, below a code (12.5 %) squared / 4)
    assert abs((root ** 2).mean() / exact - 1) <= 0.125 ** 2 / 4 + 6 * 0.006 * 2
    first = R.decode(m.cpu().numpy().reshape(-1, 128), ms.cpu().numpy()[:, None])
    assert abs(first.mean() / 1e-3 - 1) <= 0.02


def test_moments_beyond_2_to_the_32():
    """A tensor behind one of 2^32 values: its moments' indices, and the bits mixed from them, pass 32 bits."""
    torch = U.torch_mod()
    sizes = [1 << 32, 300]
    p, g = torch.zeros(sizes[0], device="cuda"), torch.zeros(sizes[0], dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(2)
    p2, g2 = rng.normal(size=300).astype(np.float32), U.round_to(rng.normal(size=300) * 1e-2, True)
    tp, tg = torch.from_numpy(p2).cuda(), torch.from_numpy(g2).cuda().bfloat16()
    blocks = B.adamw_blocks(sizes)
    m, v = (torch.zeros(blocks * 128, dtype=torch.uint8, device="cuda") for _ in range(2))
    ms, vs = (torch.zeros(blocks, dtype=torch.uint8, device="cuda") for _ in range(2))
    plan = B.AdamW(sizes, [p.data_ptr(), tp.data_ptr()], [g.data_ptr(), tg.data_ptr()], B.BF16, None, None, 8, m.data_ptr(), v.data_ptr(), ms.data_ptr(), vs.data_ptr())
    g[-1] = 1.0
    plan.step(HYPER["lr"], HYPER["beta1"], HYPER["beta2"], HYPER["eps"], 1, 5)
    z, zs = np.zeros(384, np.uint8), np.zeros(3, np.uint8)
    want = R.adamw(p2, g2, z, z, zs, zs, 0.0, step=1, seed=5, eight=True, first=1 << 32, **HYPER)
    first = 1 << 32
    assert np.array_equal(tp.cpu().numpy(), want[0])
    assert np.array_equal(m[first:].cpu().numpy(), want[1]) and np.array_equal(v[first:].cpu().numpy(), want[2])
    assert np.array_equal(ms[first // 128:].cpu().numpy(), want[3]) and np.array_equal(vs[first // 128:].cpu().numpy(), want[4])
    assert float(p[-1]) < 0 and not bool(p[-2])                      # only the value that has a gradient moved


def test_more_tensors_than_a_launch_has_threads_for():
    """2^24 + 5 tensors of one value: a block of 256 threads each, 2^32 threads and more.  Bit for bit, as everywhere here."""
    import ctypes
    torch = U.torch_mod()
    n = (1 << 24) + 5
    rng = np.random.default_rng(4)
    p, g = rng.normal(size=n).astype(np.float32), rng.normal(size=n).astype(np.float32)
    tp, tg = torch.from_numpy(p).cuda(), torch.from_numpy(g).cuda()
    m, v = (torch.zeros((n, 128), device="cuda") for _ in range(2))
    at = np.arange(n, dtype=np.int64) * 4
    sizes, pp, pg = np.ones(n, np.int64), at + tp.data_ptr(), at + tg.data_ptr()
    as_pointers = lambda a: a.ctypes.data_as(ctypes.POINTER(ctypes.c_void_p))  # noqa: E731
    lib, h = B.load_library(), ctypes.c_void_p()
    B._operator(lib.gan_adamw_create(n, sizes.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)), as_pointers(pp), as_pointers(pg), B.FP32, None, None, 32, m.data_ptr(),
                                     v.data_ptr(), None, None, ctypes.byref(h)))
    B._operator(lib.gan_adamw_step(h, HYPER["lr"], HYPER["beta1"], HYPER["beta2"], HYPER["eps"], 1, 5, None))
    B._operator(lib.gan_adamw_destroy(h))
    want = R.adamw(p, g, np.zeros(n, np.float32), np.zeros(n, np.float32), None, None, 0.0, step=1, seed=5, eight=False, first=0, **HYPER)
    assert np.array_equal(tp.cpu().numpy(), want[0])
    assert np.array_equal(m[:, 0].cpu().numpy(), want[1]) and np.array_equal(v[:, 0].cpu().numpy(), want[2])
    assert int(m.count_nonzero()) == np.count_nonzero(want[1])


@pytest.mark.parametrize("bits", [32, 8])
def test_a_captured_step_is_that_step_again(bits):
    """What gan.h says of a graph: a replay repeats the step that was captured, its rates and its rounding bits, on the moments and gradients as they are then."""
    torch = U.torch_mod()

    def fresh():
        b = Both([3000, 17], True, bits, seed=6)
        for g in b.g:
            g.copy_(torch.randn(g.shape, generator=torch.Generator().manual_seed(9)) * 1e-2)
        return b

    eager, graphed = fresh(), fresh()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.plan.step(1e-3, 0.9, 0.999, 1e-8, 7, 3, torch.cuda.current_stream().cuda_stream)
    for k in range(3):
        graph.replay()
        eager.plan.step(1e-3, 0.9, 0.999, 1e-8, 7, 3, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        pairs = list(zip(eager.p + eager.c, graphed.p + graphed.c)) + [(eager.m, graphed.m), (eager.v, graphed.v)]
        if bits == 8:
            pairs += [(eager.ms, graphed.ms), (eager.vs, graphed.vs)]
        for a, b in pairs:
            assert np.array_equal(a.float().cpu().numpy(), b.float().cpu().numpy(), equal_nan=True), k
