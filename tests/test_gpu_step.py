"""The decoding step (gated_delta_step) against the recurrence in fp64.

Tolerances, relative 2-norms: a result in bf16 carries one rounding, 2^-8 of each value at most; fp32 sums of up to 256 terms, taken 8 to a lane
and in 3 shuffles, lose at most 40 x 2^-24 of the sum of magnitudes, and eight tokens eight times that: 2e-5."""
import pytest
import torch

from oracle import gdn_recurrent as orc
from paper_2606_06034_b200 import binding as gdn

pytestmark = pytest.mark.gpu
TOL = {torch.float32: 2e-5, torch.bfloat16: 2 ** -8 + 2e-5}


def _inputs(B, T, H_k, H_v, d_k, d_v, dtype, seed=0, n_slots=None, state=torch.float32):
    gen = torch.Generator().manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    return [x.cuda() for x in (rn(B, T, H_k, d_k).to(dtype), rn(B, T, H_k, d_k).to(dtype), rn(B, T, H_v, d_v).to(dtype), torch.sigmoid(rn(B, T, H_v)),
                               -torch.nn.functional.softplus(rn(B, T, H_v)), (0.3 * rn(n_slots or B, H_v, d_v, d_k)).to(state))]


def _expected(Q, K, V, beta, g, S, rows, **kw):
    O, S = torch.zeros(V.shape, dtype=torch.float64, device="cuda"), S.double()
    for b, slot in rows:
        O[b], S[slot] = orc.gated_delta_rule(*(x[b].double() for x in (Q, K, V, beta, g)), S[slot], **kw)
    return O, S


def _near(x, ref, tol):
    err, norm = (x.double() - ref).norm().item(), ref.norm().item()
    assert err <= tol * norm, f"{err / max(norm, 1e-300):.3e} > {tol:.1e}"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("state", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,T,H_k,H_v,d_k,d_v", [(1, 1, 1, 1, 128, 128), (3, 1, 2, 4, 128, 128), (5, 3, 3, 3, 64, 96), (2, 8, 1, 4, 256, 256), (7, 2, 2, 2, 8, 16),
                                                 (2, 1, 1, 2, 200, 40), (300, 1, 1, 1, 128, 128)])
def test_step(dtype, state, B, T, H_k, H_v, d_k, d_v):
    x = _inputs(B, T, H_k, H_v, d_k, d_v, dtype, B + T, state=state)
    ref = _expected(*x, [(b, b) for b in range(B)])
    O = gdn.gated_delta_step(*x)
    assert gdn.gdn_device_status() == gdn.GDN_OK
    _near(O, ref[0], TOL[dtype])
    _near(x[5], ref[1], TOL[state])


def test_head_major_raw_keys_and_scale():
    Q, K, V, beta, g, S = _inputs(2, 3, 2, 4, 128, 128, torch.bfloat16, 9)
    Q, K = 0.1 * Q, 0.05 * K
    ref = _expected(Q, K, V, beta, g, S, [(0, 0), (1, 1)], scale=0.7, qk_l2norm=False)
    hm = [t.transpose(1, 2).contiguous() for t in (Q, K, V, beta, g)]
    O = gdn.gated_delta_step(*hm, S, scale=0.7, token_major=False, qk_l2norm=False)
    _near(O.transpose(1, 2), ref[0], TOL[torch.bfloat16])
    _near(S, ref[1], TOL[torch.float32])


def test_slots_padding_and_slots_that_cannot_be():
    Q, K, V, beta, g, S = _inputs(6, 2, 1, 2, 128, 128, torch.bfloat16, 3, n_slots=9)
    Q[2] = V[2] = beta[2] = float("nan")  # a padded row: nothing of it is read
    before = S.clone()
    # rows 0 and 4 ask for the same slot, row 5 for one that is not there
    slots = torch.tensor([7, 0, -1, 3, 7, 9], dtype=torch.int32, device="cuda")
    ref = _expected(Q, K, V, beta, g, S, [(0, 7), (1, 0), (3, 3)])
    out = torch.full_like(V, 5.0)
    O = gdn.gated_delta_step(Q, K, V, beta, g, S, slots, out=out)
    assert O is out
    assert gdn.gdn_device_status() == gdn.GDN_ERR_INVALID_ARG
    assert gdn.gdn_device_status() == gdn.GDN_OK
    assert (O[2] == 0).all() and (O[4] == 0).all() and (O[5] == 0).all()
    _near(O, ref[0], TOL[torch.bfloat16])
    _near(S, ref[1], TOL[torch.float32])
    left = [1, 2, 4, 5, 6, 8]
    assert torch.equal(S[left], before[left])


def test_degenerate_tokens():
    Q, K, V, beta, g, S = _inputs(4, 2, 2, 2, 128, 128, torch.bfloat16, 4)
    K[0, 0], Q[1, 1], beta[2, 0], g[3, 0], g[3, 1] = 0, 0, 0, -float("inf"), 0
    ref = _expected(Q, K, V, beta, g, S, [(b, b) for b in range(4)])
    O = gdn.gated_delta_step(Q, K, V, beta, g, S)
    _near(O, ref[0], TOL[torch.bfloat16])
    _near(S, ref[1], TOL[torch.float32])
    assert (O[1, 1] == 0).all()


def test_nothing_to_do():
    Q, K, V, beta, g, S = _inputs(2, 1, 2, 2, 128, 128, torch.bfloat16)
    before = S.clone()
    assert gdn.gated_delta_step(Q[:0], K[:0], V[:0], beta[:0], g[:0], S).shape == (0, 1, 2, 128)
    assert gdn.gated_delta_step(Q[:, :0], K[:, :0], V[:, :0], beta[:, :0], g[:, :0], S).shape == (2, 0, 2, 128)
    assert torch.equal(S, before)


def test_offsets_past_32_bits():
    """A pool whose last state lies more than 2^31 elements behind the first."""
    n = (1 << 31) // (32 * 128 * 128) + 2
    S = torch.zeros(n, 32, 128, 128, dtype=torch.bfloat16, device="cuda")
    Q, K, V, beta, g, part = _inputs(2, 1, 16, 32, 128, 128, torch.bfloat16, 6, state=torch.bfloat16)
    S[n - 1], S[1] = part[0], part[1]
    ref = _expected(Q, K, V, beta, g, part, [(0, 0), (1, 1)])
    O = gdn.gated_delta_step(Q, K, V, beta, g, S, torch.tensor([n - 1, 1], dtype=torch.int32, device="cuda"))
    _near(O, ref[0], TOL[torch.bfloat16])
    _near(torch.stack([S[n - 1], S[1]]), ref[1], TOL[torch.bfloat16])
    assert not S[0].any() and not S[2].any()


def test_captured_step_replayed_with_new_inputs_on_another_stream():
    x = _inputs(3, 1, 2, 4, 128, 128, torch.bfloat16, 1)
    y = _inputs(3, 1, 2, 4, 128, 128, torch.bfloat16, 2)
    ref1 = _expected(*x, [(b, b) for b in range(3)])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        gdn.gated_delta_step(*(t.clone() for t in x))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            O = gdn.gated_delta_step(*x)
        graph.replay()
        stream.synchronize()
        _near(O, ref1[0], TOL[torch.bfloat16])
        ref2 = _expected(*y[:5], x[5], [(b, b) for b in range(3)])
        for a, b in zip(x[:5], y[:5]):
            a.copy_(b)
        graph.replay()
        stream.synchronize()
    _near(O, ref2[0], TOL[torch.bfloat16])
    _near(x[5], ref2[1], TOL[torch.float32])
