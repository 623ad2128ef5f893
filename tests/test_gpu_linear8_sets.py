"""8-bit products with an epilogue where two sets of waves share the sums of more than 256 tiles by the count (GPU), and the next sizes, where one has them: tiles of both heights, ragged and empty
experts.  Bounds as in test_gpu_group_act.py."""
import pytest

import tests.test_gpu_group_act as A
from tests.test_gpu_group_linear_large import offsets

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("counts,n_in,n_out", [([30, 33, 0, 64, 65, 20, 1, 40], 2050, 4000), ([64, 0, 70, 63], 2048, 7900), ([30, 33, 0, 64, 65, 20, 1, 40], 2050, 4100)])
def test_sums_of_two_sets(counts, n_in, n_out, bf16):
    """288 tiles by the count, 256 in all; 310 and 248; 297 and 264 (one set)."""
    A.test_eight_bits(offsets(counts), n_in, n_out, bf16)
