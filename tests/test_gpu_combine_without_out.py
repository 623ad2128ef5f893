"""gan_combine_rows_backward for the rows' gradient alone (GPU): without `out`, the bits that it has with it."""
import numpy as np
import pytest

from paper_2102_10485_amd import binding as B
from tests import experts_ref as E
from tests import gpu_util as U
from tests import operators_ref as R
from tests.test_gpu_expert_rows import SHAPES, problem, sort, unwritten
from tests.test_gpu_rms_norm import matrix

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,cols,k,groups", SHAPES + [(700, 1024, 6, 5)])
def test_rows_gradient_alone(rows, cols, k, groups, bf16):
    torch = U.torch_mod()
    prec = B.BF16 if bf16 else B.FP32
    for pad, offset, weighted in ((0, 0, True), (8, 8, False), (3, 1, True)):
        labels, _, out, _, dy, w = problem(rows, cols, k, groups, bf16, pad)
        st, n = cols + pad, rows * k
        offs, _, place = sort(labels, groups)
        tw = torch.from_numpy(w).cuda()
        md, mo = matrix(dy, bf16, st, offset), matrix(out, bf16, st, offset)
        got = []
        for po, want_dw in ((0, False), (mo[2], False), (mo[2], True)):
            mdo = matrix(np.full((n, cols), 7.0), bf16, st, offset)
            dw = torch.full((n + 4,), float("nan"), device="cuda")
            B.combine_rows_backward(prec, md[2], st, po, st, place.data_ptr(), tw.data_ptr() if weighted else 0, offs.data_ptr(), groups, k, rows, cols, mdo[2], st,
                                    dw.data_ptr() if want_dw else 0)
            torch.cuda.synchronize()
            assert bool(dw[n if want_dw else 0:].isnan().all())
            got.append(unwritten(mdo, offset, n, st, cols))
        assert np.array_equal(got[0], got[1]) and np.array_equal(got[0], got[2])
        want, _, _ = E.combine_backward(dy, out, place.view(rows, k).cpu().numpy(), w if weighted else None, int(offs[groups]))
        assert np.all(np.abs(got[0] - want) <= (R.U32 + (R.UBF if bf16 else 0)) * np.abs(want))
