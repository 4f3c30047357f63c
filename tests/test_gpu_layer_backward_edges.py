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


# 1 + 2^-9 + 0.9 x 2^-17: of two bf16 pieces 1 and 2^-9 stay, off by 6.9e-6
HARD = 1 + 2.0 ** -9 + 0.9 * 2.0 ** -17


def test_states_count_with_all_their_bits_in_dg():
    """One token with beta = 0 and values of one sign. dg = exp(g) <D, S>: 32 products in a row, 5 and 16 sums, exp: (32 + 21 + 4) x 2^-24. Without D,
    scale exp(g) <q, S^T dO>: 24 accumulations of 2^-23 each, 11 + 10 additions, exp and rsqrt."""
    x = _inputs(1, 1, 1, 51)
    x["beta"].zero_()
    x["g"].fill_(-0.5)
    x["S"].fill_(HARD)
    x["dS"].fill_(HARD)
    x["Q"].fill_(1)
    x["dO"].zero_()
    dg = _call(_dense(x, 1, 1), x)[4].double().item()
    ref = torch.tensor(-0.5, dtype=torch.float64).exp().item() * D * D * x["S"].double()[0, 0, 0, 0].item() ** 2
    assert abs(dg / ref - 1) <= 57 * 2 ** -24, dg / ref - 1
    x["dS"].zero_()
    x["dO"].fill_(1)
    dg = _call(_dense(x, 1, 1), x)[4].double().item()
    ref = D ** -0.5 * torch.tensor(-0.5, dtype=torch.float64).exp().item() * D * D ** 0.5 * x["S"].double()[0, 0, 0, 0].item()
    assert abs(dg / ref - 1) <= (48 + 21 + 8) * 2 ** -24, dg / ref - 1


def test_bf16_gradients_are_rounded_once():
    """dQ of single tokens with beta = 0, dq = scale exp(g) S^T dO, against the fp64 value's own rounding to bf16: they differ where a border between two bf16
    values lies between the exact value and the kernel's, whose share is the error over the distance of the borders. States of one sign: off by 77 x 2^-24
    at most (see above), borders 2^-7 to 2^-8 of the value apart, 1.4 x 2^-8 on the average of the reciprocals over a mantissa: less than 77 x 2^-24 x 2^8 / 1.4
    = 8.4e-4. Two pieces of a state that is HARD times powers of two are 6.9e-6 off, which gives 1.3e-3 of 262144 values: 5e-4 more, by a scatter of 7e-5."""
    B, H = 128, 16
    x = _inputs(B, H, H, 52, B)
    x["g"].fill_(-0.5)
    x["beta"].zero_()
    gen = torch.Generator(device="cuda").manual_seed(53)
    x["S"] = HARD * 2.0 ** torch.randint(0, 4, x["S"].shape, generator=gen, device="cuda").float()
    x["dO"] = x["dO"].float().abs().bfloat16()
    got = _call(_dense(x, B, 1), x, qk_l2norm=False, with_dS=False)
    ref = D ** -0.5 * x["g"].double().exp()[..., None] * torch.einsum("bhvk,bhv->bhk", x["S"].double(), x["dO"].double())
    share = (got[0].reshape(ref.shape) != ref.bfloat16()).double().mean().item()
    assert share <= 8.4e-4, share


def test_gradient_of_the_state_in_the_place_of_the_next_ones():
    """dS_in may be dS_out: the gradients of a text's pieces are handed down in one tensor."""
    T, n = 200, 2
    x = _inputs(T, 1, 2, 54, n)
    cu = torch.tensor([0, 70, T], dtype=torch.int32, device="cuda")
    ref = _call(x, x, cu_seqlens=[0, 70, T])
    outs = [torch.empty_like(x[k]) for k in NAMES]
    ws = torch.empty(gdn.gdn_gated_delta_layer_backward_workspace(n, T, 2), dtype=torch.uint8, device="cuda")
    flags = gdn.GDN_FLAG_G_RAW | gdn.GDN_FLAG_LAYOUT_BTHD | gdn.GDN_FLAG_K_L2NORM
    gdn.gdn_gated_delta_layer_backward_varlen(x["dO"], *(x[k] for k in NAMES), cu, n, T, 1, 2, 64, D, D, D ** -0.5, x["S"], x["dS"], *outs, x["dS"], ws, flags)
    assert gdn.gdn_device_status() == gdn.GDN_OK
    assert all(torch.equal(p, q) for p, q in zip([*outs, x["dS"]], ref))
