"""Row norms where a row group is not full, there is nothing to sum, or the gate's exponential leaves the middle of its range. Formula, inputs and
tolerances as in test_gpu_norm.py unless a test says otherwise."""
import ctypes

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


def test_no_rows_and_no_workspace():
    """Nothing to sum: the library asks for no workspace, and the weight's and the bias's gradients are zero all the same."""
    lib = gdn.load_library()
    assert lib.gdn_layer_norm_backward_workspace(0, 128) == 0
    some = torch.zeros(128, device="cuda")  # (rows of no tensor: an address that is neither read nor written)
    dw, db = torch.full((128,), 7.0, device="cuda"), torch.full((128,), 7.0, device="cuda")
    at = some.data_ptr()
    rc = lib.gdn_layer_norm_backward(at, at, at, at, None, 0, 128, ctypes.c_float(1e-5), gdn.GDN_DTYPE_FP32, gdn.GDN_DTYPE_FP32, at, dw.data_ptr(), db.data_ptr(),
                                     None, None, 0, 0, torch.cuda.current_stream().cuda_stream)
    assert rc == gdn.GDN_OK
    torch.cuda.synchronize()
    assert not dw.any() and not db.any() and not some.any()

@pytest.mark.parametrize("width", [128, 75, 2048])
def test_gates_far_below_zero_keep_fp32_rows_exact(width):
    """y and dgate of fp32 rows, value by value, where silu is small: z from -85 to -40. The rows hold 1 and -1 and their RMS is 1, so no sum is rounded. Off
    by at most, in steps of 2^-24: rsqrt 4, exp(-z) 2, its sum with 1 1, the reciprocal 2, three products 3: 12. dgate: the slope s + z s (1 - s) is z s less a
    fortieth at most, s is off by 5, the product and the sum by 2, both times 41 / 39; rsqrt 4, products 3: 15; 28 leaves a margin into which an exponent
    rounded before exp is taken does not fit (|z| log2(e) = 123, off by 2^-18, is 44 steps by itself, and log2(e) in fp32 17)."""
    gen = torch.Generator().manual_seed(width)
    z = (-85 + 45 * torch.rand(64, width, generator=gen)).cuda()
    x = torch.where(torch.rand(64, width, generator=gen) < 0.5, -1.0, 1.0).cuda()  # (rms: n = x, no sum is rounded)
    w = torch.ones(width, device="cuda")
    z64 = z.double()
    s = torch.sigmoid(z64)
    y = gdn.layer_norm(x, w, gate=z, rms=True, eps=0.0).double()
    off = ((y - x * z64 * s) / (z64 * s)).abs().max().item()
    assert off <= 12 * 2 ** -24, off
    dz = gdn.layer_norm_backward(torch.ones_like(x), x, w, gate=z, rms=True, eps=0.0)[3]
    slope = s * (1 + z64 * (1 - s))
    off = ((dz.double() - x * slope) / slope).abs().max().item()
    assert off <= 28 * 2 ** -24, off
