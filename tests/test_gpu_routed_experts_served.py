"""The serving path of the example (GPU): its operators in 8 bits chained through hand out and put together, against the same network in bf16."""
import numpy as np
import pytest

from tests import gpu_util as U
from tests.test_gpu_routed_experts import example

pytestmark = pytest.mark.gpu


def test_served_rows():
    """Bound: an e4m3 operand is off by at most 2^-4 of each value, two of them independently by sqrt(2) 2^-4 of a product's outputs, an activation's slope is at most 1.13; the longest chain is
    four products, whose errors are independent: 1.13 sqrt(4) sqrt(2) 2^-4 = 0.20 of a row's norm, and a dozen roundings of bf16 as sqrt(12) 2^-8.  Errors of the logits move some rows with close
    choices to another expert, so that it is the middle row that has to keep the bound; an expert's own part of a row is over half of the residual's."""
    torch = U.torch_mod()
    E = example()
    model = E.Denoiser(3)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    for k in E.Denoiser.BIASES:                                       # (biases of zero would hide theirs)
        model.p[k].copy_(torch.randn(model.p[k].shape, generator=gen, device="cuda") * 0.2)
    _, noisy = E.batch(400, 9)
    model.freeze()
    exact, f = model.forward(noisy, train=False)
    exact, served = exact.double(), model.serve(noisy).double()
    off = ((served - exact).norm(dim=1) / exact.norm(dim=1)).cpu().numpy()
    assert np.isfinite(off).all() and np.median(off) <= 0.20 + np.sqrt(12) * 2.0 ** -8, np.median(off)
    assert 0 < float(f["balance"]) <= E.EXPERTS
