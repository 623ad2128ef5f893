"""Calls without rows, without experts, and optimisers without values (GPU), on empty tensors as a program has them: their address is NULL."""
import numpy as np
import pytest

from paper_2102_10485_amd import binding as B
from tests import gpu_util as U

pytestmark = pytest.mark.gpu


def empty(*shape, dtype=None):
    torch = U.torch_mod()
    t = torch.empty(shape, dtype=dtype or torch.bfloat16, device="cuda")
    assert t.data_ptr() == 0
    return t.data_ptr()


def test_no_rows():
    torch = U.torch_mod()
    u8, f32 = torch.uint8, torch.float32
    gain, offs, w = torch.ones(64, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda"), torch.ones((3, 32, 64), device="cuda").bfloat16()
    w8, ws = torch.zeros((3, 32, 128), dtype=u8, device="cuda"), torch.ones((3, 32, 1), dtype=u8, device="cuda")
    x, y, inv = empty(0, 64), empty(0, 32), empty(0, dtype=f32)
    B.rms_norm(B.BF16, x, 64, x, 64, gain.data_ptr(), 1e-5, 0, 64, x, 64, x, 64, empty(0, 128, dtype=u8), empty(0, 1, dtype=u8), inv)
    dgain = torch.full((64,), float("nan"), device="cuda")
    assert B.rms_norm_backward_bytes(0, 64) == 0
    B.rms_norm_backward(B.BF16, x, 64, x, 64, gain.data_ptr(), inv, x, 64, 0, 64, x, 64, dgain.data_ptr(), 0, 0)
    B.quantize8(B.BF16, x, 64, 0, 64, empty(0, 128, dtype=u8), empty(0, 1, dtype=u8))
    B.group_linear(B.BF16, x, 64, w.data_ptr(), offs.data_ptr(), 3, 0, 64, 32, y, 32)
    B.group_linear_dgrad(B.BF16, y, 32, w.data_ptr(), offs.data_ptr(), 3, 0, 64, 32, x, 64)
    B.group_linear8(empty(0, 128, dtype=u8), empty(0, 1, dtype=u8), w8.data_ptr(), ws.data_ptr(), offs.data_ptr(), 3, 0, 64, 32, B.BF16, y, 32)
    assert not dgain.cpu().numpy().any()
    for precision in (B.BF16, B.FP32):                                # experts without rows: zeros
        dw = torch.full((3, 32, 64), float("nan"), device="cuda")
        assert B.group_linear_wgrad_bytes(3, 0, 64, 32) == 0
        B.group_linear_wgrad(precision, x, 64, y, 32, offs.data_ptr(), 3, 0, 64, 32, dw.data_ptr(), 0, 0)
        assert not dw.cpu().numpy().any()


@pytest.mark.parametrize("bf16", [False, True])
def test_no_experts(bf16):
    """Every row belongs to no expert: zeros; and there is no weight gradient."""
    torch = U.torch_mod()
    kind, precision = (torch.bfloat16, B.BF16) if bf16 else (torch.float32, B.FP32)
    offs, u8 = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.uint8
    x, y, dx = torch.ones((5, 64), device="cuda").to(kind), torch.ones((5, 32), device="cuda").to(kind), torch.ones((5, 64), device="cuda").to(kind)
    w = empty(0, 32, 64)
    B.group_linear_dgrad(precision, y.data_ptr(), 32, w, offs.data_ptr(), 0, 5, 64, 32, dx.data_ptr(), 64)
    B.group_linear(precision, x.data_ptr(), 64, w, offs.data_ptr(), 0, 5, 64, 32, y.data_ptr(), 32)
    assert not dx.float().cpu().numpy().any() and not y.float().cpu().numpy().any()
    B.group_linear_wgrad(precision, x.data_ptr(), 64, y.data_ptr(), 32, offs.data_ptr(), 0, 5, 64, 32, empty(0, 32, 64, dtype=torch.float32), 0, 0)
    y.fill_(1)
    x8, xs = torch.zeros((5, 128), dtype=u8, device="cuda"), torch.ones((5, 1), dtype=u8, device="cuda")
    B.group_linear8(x8.data_ptr(), xs.data_ptr(), empty(0, 32, 128, dtype=u8), empty(0, 32, 1, dtype=u8), offs.data_ptr(), 0, 5, 64, 32, precision, y.data_ptr(), 32)
    assert not y.float().cpu().numpy().any()


@pytest.mark.parametrize("bits", [32, 8])
def test_no_values(bits):
    nothing = empty(0)
    plan = B.AdamW([0, 0], [nothing] * 2, [nothing] * 2, B.BF16, [nothing] * 2, None, bits, nothing, nothing, nothing, nothing)
    plan.step(1e-3, 0.9, 0.999, 1e-8, 1)
    plan.close()


def test_what_has_elements_is_still_wanted():
    p = 1 << 20                                                       # an address that no refused call touches
    for call in (lambda: B.group_linear(B.BF16, 0, 64, p, p, 3, 5, 64, 32, p, 32), lambda: B.group_linear(B.BF16, p, 64, 0, p, 3, 5, 64, 32, p, 32),
                 lambda: B.group_linear(B.BF16, p, 64, p, 0, 3, 5, 64, 32, p, 32), lambda: B.group_linear_dgrad(B.BF16, p, 32, p, p, 3, 5, 64, 32, 0, 64),
                 lambda: B.group_linear_wgrad(B.BF16, p, 64, 0, 32, p, 3, 5, 64, 32, p, 0, 0), lambda: B.group_linear_wgrad(B.BF16, 0, 64, 0, 32, p, 3, 0, 64, 32, 0, 0, 0),
                 lambda: B.group_linear8(p, 0, p, p, p, 3, 5, 64, 32, B.BF16, p, 32), lambda: B.group_linear8(p, p, p, 0, p, 3, 5, 64, 32, B.BF16, p, 32),
                 lambda: B.rms_norm(B.BF16, p, 64, 0, 0, 0, 1e-5, 0, 64, 0, 0, p, 64, 0, 0, 0), lambda: B.quantize8(B.BF16, p, 64, 5, 64, p, 0),
                 lambda: B.rms_norm_backward(B.BF16, p, 64, p, 64, p, 0, 0, 0, 5, 64, p, 64, 0, 0, 0),
                 lambda: B.AdamW([0, 3], [0, p], [0, p], B.BF16, None, None, 32, 0, 0)):
        with pytest.raises(B.GanError) as e:
            call()
        assert e.value.status == B.GAN_E_ARG and "NULL" in str(e.value)
