"""Whose error a call of the operators reports (GPU)."""
import pytest

from paper_2102_10485_amd import binding as B
from tests import gpu_util as U

pytestmark = pytest.mark.gpu


def test_another_calls_error_is_not_the_operators():
    """A HIP call that failed before leaves its error with the thread: an operator that launches is right all the same."""
    torch = U.torch_mod()
    hip = B.load_library()                                            # (the runtime that it is linked with)
    x, gain = torch.ones((3, 64), device="cuda"), torch.ones(64, device="cuda")
    y, q, sc = torch.zeros((3, 64), device="cuda"), torch.zeros((3, 128), dtype=torch.uint8, device="cuda"), torch.zeros((3, 1), dtype=torch.uint8, device="cuda")
    w, offs, dw = torch.ones((1, 64, 64), device="cuda"), torch.tensor([0, 3], dtype=torch.int32, device="cuda"), torch.zeros((1, 64, 64), device="cuda")
    plan = B.AdamW([64], [gain.data_ptr()], [x.data_ptr()], B.FP32, None, None, 32, dw.data_ptr(), dw.data_ptr() + 2048)
    px, py, pw, po, pd = (t.data_ptr() for t in (x, y, w, offs, dw))
    for call in (lambda: B.rms_norm(B.FP32, px, 64, 0, 0, gain.data_ptr(), 0.0, 3, 64, 0, 0, py, 64, 0, 0, 0), lambda: B.quantize8(B.FP32, px, 64, 3, 64, q.data_ptr(), sc.data_ptr()),
                 lambda: B.rms_norm_backward(B.FP32, px, 64, px, 64, gain.data_ptr(), gain.data_ptr(), 0, 0, 3, 64, py, 64, 0, 0, 0),
                 lambda: B.group_linear(B.FP32, px, 64, pw, po, 1, 3, 64, 64, py, 64), lambda: B.group_linear_dgrad(B.FP32, px, 64, pw, po, 1, 3, 64, 64, py, 64),
                 lambda: B.group_linear_wgrad(B.FP32, px, 64, px, 64, po, 1, 3, 64, 64, pd, 0, 0), lambda: plan.step(0.0, 0.9, 0.999, 1e-8, 1)):
        assert hip.hipSetDevice(12345) != 0                           # refused by the host
        call()
    torch.cuda.synchronize()
