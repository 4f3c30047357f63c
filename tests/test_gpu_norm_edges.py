"""Row norms where a row group is not full, there is nothing to sum, or the gate's exponential leaves the middle of its range. Formula, inputs and
tolerances as in test_gpu_norm.py unless a test says otherwise."""
import pytest
import torch

from paper_2606_06034_b200 import binding as gdn
from test_gpu_norm import _check, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("rows,width", [(5, 128), (17, 77), (9, 256), (3, 500), (1, 128), (16, 128), (3, 2056)])
def test_no_eps_and_rows_that_do_not_fill_a_group(dtype, rms, rows, width):
    """With eps = 0 a row of zeros has no norm: the places behind the last row hold such rows, and count for nothing in the weight's gradient."""
    _check(_inputs(rows, width, dtype, seed=rows), rms, eps=0.0)
