"""The layer's backward pass where fp32 results show what their operands are held in. Formula, inputs and tolerances as in
test_gpu_layer_backward.py unless a test says otherwise."""
import pytest
import torch

from paper_2606_06034_b200 import binding as gdn
from test_gpu_layer_backward import D, NAMES, _call, _check, _dense, _expected, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("closed", [8, 32, 60])
@pytest.mark.parametrize("open_by", [1.0, 0.01])
def test_gates_that_close_many_times_in_a_chunk(closed, open_by):
    """Decays behind a closed gate are those between the tokens there, whatever the sum of the chunk's gates has come to."""
    x = _inputs(150, 1, 2, 31 + closed)
    x["g"] *= open_by
    x["g"][0:2 * closed:2] = -float("inf")  # every second token from the first on, into the second chunk for 60
    ref, dS = _expected(x, [0, 150])
    _check(_call(_dense(x, 1, 150), x), ref, dS)


@pytest.mark.parametrize("B,T,H_k,H_v", [(8, 34, 8, 8), (4, 64, 4, 8), (1, 253, 6, 24), (1, 500, 2, 4)])
def test_decays_are_accurate_to_their_own_size(B, T, H_k, H_v):
    """dbeta with a gradient from the final states: r of a chunk's last tokens is made of exp(g_C - g_i), a difference of at most a few, of sums that
    reach 50. With a decay off by 2^-24 of the difference (5) and of exp, sums of 128 products (8 accumulations of each of three pieces, 2^-24
    each, in sequence, on random signs: sqrt(24)), twice, and 64 more in the dot products: sqrt(2 x 24 + 64 + 5^2) x 2^-24 = 7e-7; dg
    has one product more and twice the terms, of which some cancel: twice that. Sums rounded at 50 are off by 2^-19 = 1.9e-6 at worst, 1.4e-6 in dbeta."""
    x = _inputs(B * T, H_k, H_v, 41, B)
    ref, _ = _expected(x, [b * T for b in range(B + 1)])
    got = _call(_dense(x, B, T), x)
    for n, tol in (("beta", 7e-7), ("g", 1.4e-6)):
        t = got[NAMES.index(n)].reshape(ref[n].shape).double()
        err = ((t - ref[n]).norm() / ref[n].norm()).item()
        assert err <= tol, (n, err)
