"""What the operators for label experts refuse, on the host, before anything is launched; and their sizes."""
import ctypes as C

import numpy as np
import pytest

from paper_2102_10485_amd import binding as B
from tests import operators_ref as R

P = 1 << 20                                                         # an address that no refused call touches


def refused(call, status, word):
    with pytest.raises(B.GanError) as e:
        call()
    assert e.value.status == status and word in str(e.value), str(e.value)


def norm(**k):
    a = dict(precision=B.BF16, x=P, x_stride=64, residual=0, residual_stride=0, gain=P, eps=1e-5, rows=4, cols=64, total=0, total_stride=0, y=P, y_stride=64,
             y8=0, y8_scale=0, inv_rms=0)
    a.update(k)
    return lambda: B.rms_norm(**a)


def test_norm():
    for change, word in ((dict(precision=2), "precision"), (dict(x=0), "NULL"), (dict(gain=0), "NULL"), (dict(rows=-1), "negative"), (dict(cols=0), "columns"),
                         (dict(x_stride=63), "x_stride"), (dict(residual=P, residual_stride=63), "residual_stride"), (dict(total=P, total_stride=1), "sum_stride"),
                         (dict(y_stride=0), "y_stride"), (dict(y8=P), "go together"), (dict(y8=P + 4, y8_scale=P), "aligned"), (dict(eps=-1.0), "eps"),
                         (dict(eps=float("nan")), "eps")):
        refused(norm(**change), B.GAN_E_ARG, word)
    refused(norm(rows=1 << 31), B.GAN_E_SHAPE, "2^30")
    norm(rows=0)()

    def back(**k):
        a = dict(precision=B.FP32, dy=P, dy_stride=64, total=P, total_stride=64, gain=P, inv_rms=P, dtotal=0, dtotal_stride=0, rows=4, cols=64, dx=P, dx_stride=64,
                 dgain=P, work=P, work_bytes=B.rms_norm_backward_bytes(4, 64))
        a.update(k)
        return lambda: B.rms_norm_backward(**a)

    for change, word in ((dict(dy=0), "NULL"), (dict(inv_rms=0), "NULL"), (dict(dy_stride=3), "dy_stride"), (dict(dtotal=P), "dsum_stride"), (dict(work=0), "work"),
                         (dict(work_bytes=4), "work"), (dict(work=P + 8), "work"), (dict(precision=-1), "precision")):
        refused(back(**change), B.GAN_E_ARG, word)
    assert B.rms_norm_backward_bytes(0, 5) == 0 and B.rms_norm_backward_bytes(3, 5) == 20 and B.rms_norm_backward_bytes(-1, 5) == 0
    refused(lambda: B.quantize8(B.FP32, P, 3, 4, 5, P, P), B.GAN_E_ARG, "x_stride")
    refused(lambda: B.quantize8(B.FP32, P, 5, 4, 5, P + 1, P), B.GAN_E_ARG, "aligned")


@pytest.mark.parametrize("call", [B.group_linear, B.group_linear_dgrad])
def test_linear(call):
    ok = [B.BF16, P, 64, P, P, 4, 10, 64, 64, P, 64]
    for at, value, status, word in ((0, 5, B.GAN_E_ARG, "precision"), (1, 0, B.GAN_E_ARG, "NULL"), (4, 0, B.GAN_E_ARG, "NULL"), (2, 63, B.GAN_E_ARG, "stride"),
                                    (10, 63, B.GAN_E_ARG, "stride"), (5, -1, B.GAN_E_ARG, "negative"), (6, -1, B.GAN_E_ARG, "negative"),
                                    (7, 0, B.GAN_E_ARG, "inputs"), (5, 65536, B.GAN_E_SHAPE, "65535"), (6, (1 << 30) + 1, B.GAN_E_SHAPE, "2^30")):
        a = list(ok)
        a[at] = value
        refused(lambda: call(*a), status, word)
    ok[6] = 0
    call(*ok)


def test_wgrad_and_eight_bits():
    refused(lambda: B.group_linear_wgrad(B.BF16, P, 64, P, 63, P, 4, 10, 64, 64, P, P, 1 << 40), B.GAN_E_ARG, "dy_stride")
    refused(lambda: B.group_linear_wgrad(B.BF16, P, 64, P, 64, P, 4, 10, 64, 64, P, P + 4, 1 << 40), B.GAN_E_ARG, "work")
    ok = [P, P, P, P, P, 4, 10, 100, 64, B.BF16, P, 64]
    for at, value, word in ((1, 0, "NULL"), (3, 0, "NULL"), (0, P + 8, "aligned"), (2, P + 8, "aligned"), (11, 63, "y_stride"), (9, 7, "precision")):
        a = list(ok)
        a[at] = value
        refused(lambda: B.group_linear8(*a), B.GAN_E_ARG, word)


def test_adamw():
    def make(sizes=(5,), params=(P,), grads=(P,), precision=B.FP32, copies=None, decay=None, bits=32, m=P, v=P, ms=0, vs=0):
        return lambda: B.AdamW(list(sizes), list(params), list(grads), precision, copies, decay, bits, m, v, ms, vs)

    for k, word in ((dict(precision=3), "precision"), (dict(bits=16), "state_bits"), (dict(m=0), "NULL"), (dict(params=(0,)), "NULL"), (dict(ms=P, vs=P), "state_bits 8"),
                    (dict(bits=8, ms=P), "state_bits 8"), (dict(m=P + 4), "aligned"), (dict(sizes=(-1,)), "negative"), (dict(decay=[-1.0]), "decay"),
                    (dict(decay=[float("nan")]), "decay"), (dict(sizes=(), params=(), grads=()), "no tensors"), (dict(params=(P, P)), "one entry")):
        refused(make(**k), B.GAN_E_ARG, word)
    lib = B.load_library()
    assert lib.gan_adamw_step(None, 1e-3, 0.9, 0.999, 1e-8, 1, 0, None) == B.GAN_E_ARG and lib.gan_adamw_destroy(None) == B.GAN_OK
    assert lib.gan_adamw_create(1, None, None, None, 0, None, None, 32, None, None, None, None, None) == B.GAN_E_ARG
    assert B.adamw_blocks([1, 128, 129, 0]) == 4 and lib.gan_adamw_blocks(0, None) == 0 and B.adamw_blocks([-5]) == 0
    assert isinstance(lib.gan_operator_last_error(), bytes) and C.sizeof(C.c_void_p) == 8


def test_chance_rounding_is_fair():
    """The reference's codes rounded by chance: the mean over 2^16 indices is the value, to the deviation of such a mean (five of them)."""
    rng = np.random.default_rng(0)
    x = np.repeat(np.exp(rng.normal(size=16) * 2).astype(np.float32), 128)[None].reshape(16, 128)
    x[:, 0] = 448.0
    s = R.scale_bytes(x)[:, 0]
    total, n = np.zeros((16, 128)), 512
    for t in range(n):
        u = R.mixed(np.arange(x.size), t, 9).reshape(x.shape)
        total += R.decode(R.chance_codes(x, s, u & 0xFFFF, False), s[:, None])
    ulp = np.maximum(np.exp2(np.floor(np.log2(x / np.exp2(s - 127.0)[:, None]))), 2.0 ** -6) / 8 * np.exp2(s - 127.0)[:, None]
    assert np.all(np.abs(total[:, 1:].mean(1) / n - x[:, 1]) <= 5 * 0.5 * ulp[:, 1] / np.sqrt(127 * n))


def test_eight_bits_of_too_many_inputs():
    """2^22 inputs are the most in 8 bits, padded to 128 or not; what is refused for its sizes is refused without rows too."""
    for n_in, rows in (((1 << 22) + 1, 10), ((1 << 22) + 128, 0), (1 << 28, 10)):
        refused(lambda: B.group_linear8(P, P, P, P, P, 4, rows, n_in, 64, B.BF16, P, 64), B.GAN_E_SHAPE, "2^22")
    B.group_linear8(P, P, P, P, P, 4, 0, 1 << 22, 64, B.BF16, P, 64)
