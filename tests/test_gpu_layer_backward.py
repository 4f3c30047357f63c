"""The layer's backward pass (gated_delta_layer_backward) against autograd through the recurrence in fp64, token by token, and against differences.

Tolerances, relative 2-norms. dQ, dK, dV: one rounding to bf16, 2^-8 of each value at most, and operands in two bf16 pieces, 2^-17: 2^-8 + 1e-4.
dbeta, dg, dS_in: fp32 sums of up to 128 terms (128 x 2^-24 = 8e-6 of the sum of magnitudes at worst) on top of each other three deep, and the two-piece
states in two of dg's terms (2^-17 = 8e-6): 4e-5. Keys that are nearly the same, written with beta near 1 behind open gates, let a token's u
cancel against those before it: ten times that."""
import pytest
import torch

from oracle import gdn_recurrent as orc
from paper_2606_06034_b200 import binding as gdn

pytestmark = pytest.mark.gpu
D = 128
TOL16, TOL32 = 2 ** -8 + 1e-4, 4e-5
NAMES = ("Q", "K", "V", "beta", "g")


def _inputs(tokens, H_k, H_v, seed=0, n_state=1):
    """Token-major tensors of `tokens` tokens, states of n_state sequences."""
    gen = torch.Generator().manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    x = {"Q": rn(tokens, H_k, D).bfloat16(), "K": rn(tokens, H_k, D).bfloat16(), "V": rn(tokens, H_v, D).bfloat16(), "beta": torch.sigmoid(rn(tokens, H_v)),
         "g": -torch.nn.functional.softplus(rn(tokens, H_v)), "dO": rn(tokens, H_v, D).bfloat16(), "S": 0.3 * rn(n_state, H_v, D, D), "dS": 0.1 * rn(n_state, H_v, D, D)}
    return {k: v.cuda() for k, v in x.items()}


def _expected(x, bounds, with_S=True, with_dS=True, **kw):
    """Gradients of all inputs; rows that no sequence covers get zeros."""
    out = {n: torch.zeros(x[n].shape, dtype=torch.float64, device="cuda") for n in NAMES}
    dS = torch.zeros(x["S"].shape, dtype=torch.float64, device="cuda")
    for s, (a, b) in enumerate(zip(bounds[:-1], bounds[1:])):
        leaf = [x[n][a:b].double().requires_grad_() for n in NAMES]
        S = (x["S"][s] if with_S else torch.zeros_like(x["S"][s])).double().requires_grad_()
        o, end = orc.gated_delta_rule(*leaf, S, **kw)
        loss = (o * x["dO"][a:b].double()).sum() + (end * (x["dS"][s].double() if with_dS else 0.0)).sum()
        *g, dS[s] = torch.autograd.grad(loss, leaf + [S], allow_unused=True, materialize_grads=True)
        for n, d in zip(NAMES, g):
            out[n][a:b] = d
    return out, dS


def _near(x, ref, tol, what):
    err, norm = (x.double() - ref).norm().item(), ref.norm().item()
    assert err <= tol * norm, f"{what}: {err / max(norm, 1e-300):.3e} > {tol:.1e}"


def _check(got, ref, dS=None, scale=1.0):
    for n, t in zip(NAMES, got):
        _near(t.reshape(ref[n].shape), ref[n], (TOL32 if n in ("beta", "g") else TOL16) * scale, "d" + n)
    if dS is not None:
        _near(got[5], dS, TOL32 * scale, "dS_in")
    assert gdn.gdn_device_status() == gdn.GDN_OK


def _dense(x, B, T):
    return {n: x[n].view(B, T, *x[n].shape[1:]) for n in (*NAMES, "dO")}


def _call(d, x, with_S=True, with_dS=True, **kw):
    return gdn.gated_delta_layer_backward(d["dO"], *(d[n] for n in NAMES), S_in=x["S"] if with_S else None, dS_out=x["dS"] if with_dS else None, **kw)


@pytest.mark.parametrize("B,T,H_k,H_v", [(1, 1, 1, 1), (2, 2, 1, 1), (1, 15, 2, 2), (1, 16, 1, 2), (3, 63, 1, 1), (1, 64, 1, 1), (2, 65, 2, 4), (1, 128, 1, 3), (2, 200, 1, 2), (1, 500, 1, 1)])
@pytest.mark.parametrize("with_S,with_dS", [(False, False), (True, True), (True, False), (False, True)])
def test_dense(B, T, H_k, H_v, with_S, with_dS):
    x = _inputs(B * T, H_k, H_v, B + T, B)
    ref, dS = _expected(x, [b * T for b in range(B + 1)], with_S, with_dS)
    got = _call(_dense(x, B, T), x, with_S, with_dS)
    assert (got[5] is None) == (not with_S)
    _check(got, ref, dS if with_S else None)
    if T == 1 and not with_S:
        assert not got[4].any()  # a first token's gate decays nothing


def test_head_major_raw_keys_and_scale():
    B, T = 2, 100
    x = _inputs(B * T, 2, 4, 7, B)
    for n in ("Q", "K"):
        x[n] *= 0.08
    ref, dS = _expected(x, [0, T, 2 * T], scale=0.3, qk_l2norm=False)
    d = {n: t.transpose(1, 2).contiguous() for n, t in _dense(x, B, T).items()}
    got = _call(d, x, scale=0.3, qk_l2norm=False, token_major=False)
    _check([t.transpose(1, 2).reshape(ref[n].shape) for n, t in zip(NAMES, got)] + [got[5]], ref, dS)


@pytest.mark.parametrize("bounds,T", [([0, 1, 2, 3], 3), ([0, 64, 64, 129, 300], 300), ([5, 70, 71, 71, 200], 230), ([0, 63, 127, 128, 192, 193], 193)])
@pytest.mark.parametrize("token_major", [True, False])
def test_packed(bounds, T, token_major):
    """Sequences of no token, of one, ragged ones, ones that begin inside a tile; rows that none covers hold what must not be read."""
    x = _inputs(T, 2, 4, T, len(bounds) - 1)
    ref, dS = _expected(x, bounds)
    for n in (*NAMES, "dO"):
        x[n][:bounds[0]] = float("nan")
        x[n][bounds[-1]:] = float("nan")
    d = x if token_major else {n: x[n].transpose(0, 1).contiguous() for n in (*NAMES, "dO")}
    got = _call(d, x, cu_seqlens=bounds, token_major=token_major)
    back = got[:5] if token_major else [t.transpose(0, 1) for t in got[:5]]
    _check([*back, got[5]], ref, dS)
    for t in back:
        assert not t[:bounds[0]].any() and not t[bounds[-1]:].any()


def test_packed_is_the_same_as_dense():
    x = _inputs(2 * 192, 2, 2, 11, 2)
    a = _call(_dense(x, 2, 192), x)
    b = _call(x, x, cu_seqlens=[0, 192, 384])
    assert all(torch.equal(p.reshape(q.shape), q) for p, q in zip(a, b))


def test_degenerate_tokens():
    x = _inputs(150, 1, 2, 12)
    x["K"][3], x["Q"][5], x["K"][70], x["beta"][9], x["beta"][64] = 0, 0, 0, 0, 0
    x["g"][20:24], x["g"][80:100] = 0, 0
    x["g"][30], x["g"][110] = -200.0, -1e30
    ref, dS = _expected(x, [0, 150])
    got = _call(_dense(x, 1, 150), x)
    _check(got, ref, dS)
    assert not got[1][0, 3].any() and not got[0][0, 5].any()
    x["g"][110] = -float("inf")
    again = _call(_dense(x, 1, 150), x)
    assert all(torch.isfinite(t).all() for t in again) and all(torch.equal(a, b) for a, b in zip(got, again))


def test_open_gates_and_keys_that_are_nearly_the_same():
    x = _inputs(320, 1, 2, 13)
    x["K"] = (x["K"][:1] + 0.3 * x["K"]).bfloat16().contiguous()
    x["beta"], x["g"] = 0.9 + 0.1 * x["beta"], 1e-3 * x["g"]
    ref, dS = _expected(x, [0, 320])
    _check(_call(_dense(x, 1, 320), x), ref, dS, 10)


def test_small_and_large_gradients():
    """A loss scaled by a power of two scales every gradient by it, down to where the states' pieces would leave bf16's range."""
    x = _inputs(130, 1, 1, 14)
    a = _call(_dense(x, 1, 130), x)
    for e in (-40, 30):
        x2 = {**x, "dO": x["dO"] * 2.0 ** e, "dS": x["dS"] * 2.0 ** e}
        assert all(torch.equal(p, q * 2.0 ** -e) for p, q in zip(a, _call(_dense(x2, 1, 130), x2)))


def test_against_differences():
    """<gradient, direction> against central differences of the fp64 recurrence: h = 1e-4, their own error of order h^2."""
    x = _inputs(90, 1, 2, 15)
    got = _call(_dense(x, 1, 90), x)
    gen = torch.Generator(device="cuda").manual_seed(16)
    base = [x[n].double() for n in NAMES] + [x["S"][0].double()]

    def loss(a):
        o, s = orc.gated_delta_rule(*a)
        return (o * x["dO"].double()).sum() + (s * x["dS"][0].double()).sum()

    for i, g in enumerate(got):
        d = torch.randn(base[i].shape, generator=gen, device="cuda", dtype=torch.float64)
        up, down = ([u + s * 1e-4 * d if j == i else u for j, u in enumerate(base)] for s in (1, -1))
        slope, g = ((loss(up) - loss(down)) / 2e-4).item(), g.reshape(d.shape).double()
        tol = (TOL32 if i > 2 else TOL16) * (g.norm() * d.norm()).item()
        assert abs(slope - (g * d).sum().item()) <= tol + 1e-6 * abs(slope)


def test_repeatable_with_a_workspace_of_the_caller_and_beside_other_calls():
    x, y = _inputs(700, 2, 4, 17), _inputs(700, 2, 4, 18)
    dx, dy = _dense(x, 1, 700), _dense(y, 1, 700)
    a, b = _call(dx, x), _call(dy, y)
    ws = torch.full((gdn.gdn_gated_delta_layer_backward_workspace(1, 700, 4),), 255, dtype=torch.uint8, device="cuda")  # (NaN wherever it is read first)
    again = _call(dx, x, workspace=ws)
    assert all(torch.equal(p, q) for p, q in zip(a, again))
    with pytest.raises(gdn.GdnError):
        _call(dx, x, workspace=ws[:-16])
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    out = [[], []]
    for _ in range(4):
        for i, (d, z) in enumerate(((dx, x), (dy, y))):
            with torch.cuda.stream(streams[i]):
                out[i].append(_call(d, z))
    torch.cuda.synchronize()
    for ref, runs in zip((a, b), out):
        for r in runs:
            assert all(torch.equal(p, q) for p, q in zip(ref, r))


def test_captured_packed_call_replayed_with_other_lengths():
    T, n = 400, 3
    x = _inputs(T, 1, 2, 19, n)
    cu = torch.tensor([0, 100, 229, 400], dtype=torch.int32, device="cuda")
    outs = [torch.zeros_like(x[k]) for k in NAMES] + [torch.empty_like(x["S"])]
    ws = torch.empty(gdn.gdn_gated_delta_layer_backward_workspace(n, T, 2), dtype=torch.uint8, device="cuda")
    flags = gdn.GDN_FLAG_G_RAW | gdn.GDN_FLAG_LAYOUT_BTHD | gdn.GDN_FLAG_K_L2NORM

    def call():
        gdn.gdn_gated_delta_layer_backward_varlen(x["dO"], *(x[k] for k in NAMES), cu, n, T, 1, 2, 64, D, D, D ** -0.5, x["S"], x["dS"], *outs, ws, flags)

    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for bounds in ([0, 100, 229, 400], [0, 300, 301, 400]):
        cu.copy_(torch.tensor(bounds, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        ref, dS = _expected(x, bounds)
        _check(outs, ref, dS)
    with pytest.raises(RuntimeError):  # boundaries from the host cannot be captured
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            _call(x, x, cu_seqlens=[0, T], with_S=False, with_dS=False)


def test_nothing_to_do():
    x = _inputs(64, 1, 2, 20, 2)
    got = _call({n: t[:, :0].contiguous() for n, t in _dense(x, 2, 32).items()}, x)
    assert got[0].shape == (2, 0, 1, D) and torch.equal(got[5], x["dS"])  # no token: the state goes through
    got = gdn.gated_delta_layer_backward(x["dO"][:0], *(x[n][:0] for n in NAMES), cu_seqlens=[0])
    assert got[2].shape == (0, 2, D)


def test_more_chunks_than_one_round_of_the_grid():
    """Every CTA of the last kernel takes several chunks, heads of a group among them."""
    B, T, H_k, H_v = 4, 640, 4, 8
    x = _inputs(B * T, H_k, H_v, 21, B)
    got = _call(_dense(x, B, T), x)
    for b in (0, B - 1):
        part = {n: x[n][b * T:(b + 1) * T] for n in (*NAMES, "dO")} | {"S": x["S"][b:b + 1], "dS": x["dS"][b:b + 1]}
        ref, dS = _expected(part, [0, T])
        _check([t[b] for t in got[:5]] + [got[5][b:b + 1]], ref, dS)
