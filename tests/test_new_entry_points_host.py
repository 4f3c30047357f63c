"""Refusals of the decoding step, the layer's backward pass and the row norm, and the oracle's own gradients: no GPU needed."""

import pytest
import torch

from oracle import gdn_recurrent as orc
from paper_2606_06034_b200 import binding as gdn
from paper_2606_06034_b200 import build as gdn_build

A = 1 << 20  # an aligned address that nothing reads


@pytest.fixture(scope="module")
def lib():
    gdn_build.build()
    return gdn.load_library()


def _step(lib, **kw):
    a = dict(Q=A, K=A, V=A, beta=A, g=A, B=2, H_k=2, H_v=4, T=1, d_k=128, d_v=128, scale=1.0, dtype=1, S=A, state_dtype=0, slots=None, n_slots=2,
             O=A, flags=gdn.GDN_FLAG_LAYOUT_BTHD, stream=None)
    a.update(kw)
    return lib.gdn_recurrent_step(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(Q=None), "NULL"), (dict(S=None), "NULL"), (dict(O=None), "NULL"), (dict(beta=None), "NULL"),
    (dict(B=-1), "INVALID_ARG"), (dict(T=-1), "INVALID_ARG"), (dict(H_v=3), "INVALID_ARG"), (dict(n_slots=1), "INVALID_ARG"), (dict(dtype=7), "INVALID_ARG"),
    (dict(state_dtype=2), "INVALID_ARG"), (dict(flags=gdn.GDN_FLAG_G_RAW), "INVALID_ARG"), (dict(n_slots=-1, slots=A), "INVALID_ARG"),
    (dict(d_k=100), "UNSUPPORTED"), (dict(d_v=264), "UNSUPPORTED"), (dict(V=A + 8), "ALIGN"), (dict(slots=A + 4), "ALIGN")])
def test_step_refuses(lib, kw, status):
    assert _step(lib, **kw) == getattr(gdn, "GDN_ERR_" + status)


def _backward(lib, packed=False, **kw):
    a = dict(dO=A, Q=A, K=A, V=A, beta=A, g=A)
    a.update(dict(cu=A, n_seq=2, T=128) if packed else dict(n_seq=2))
    a.update(dict(H_k=2, H_v=4, T=128, C=64, d_k=128, d_v=128, scale=1.0, S_in=None, dS_out=None, dQ=A, dK=A, dV=A, dbeta=A, dg=A, dS_in=None, ws=A,
                  bytes=1 << 40, flags=gdn.GDN_FLAG_G_RAW, stream=None))
    if packed:
        order = ["dO", "Q", "K", "V", "beta", "g", "cu", "n_seq", "T", "H_k", "H_v", "C", "d_k", "d_v"]
        a = {k: a[k] for k in order + [k for k in a if k not in order]}
    a.update(kw)
    return (lib.gdn_gated_delta_layer_backward_varlen if packed else lib.gdn_gated_delta_layer_backward)(*a.values())


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("kw,status", [
    (dict(dO=None), "NULL"), (dict(dg=None), "NULL"), (dict(ws=None), "NULL"), (dict(n_seq=-1), "INVALID_ARG"), (dict(H_v=3), "INVALID_ARG"),
    (dict(T=-1), "INVALID_ARG"), (dict(bytes=16), "INVALID_ARG"), (dict(flags=gdn.GDN_FLAG_G_RAW | gdn.GDN_FLAG_OUT_FP32), "INVALID_ARG"),
    (dict(flags=0), "UNSUPPORTED"), (dict(C=32), "UNSUPPORTED"), (dict(d_k=64), "UNSUPPORTED"), (dict(dQ=A + 4), "ALIGN"), (dict(S_in=A + 8), "ALIGN")])
def test_backward_refuses(lib, packed, kw, status):
    assert _backward(lib, packed, **kw) == getattr(gdn, "GDN_ERR_" + status)


def test_backward_without_boundaries_is_refused(lib):
    assert _backward(lib, True, cu=None) == gdn.GDN_ERR_NULL


def test_workspace_sizes(lib):
    per_chunk = lib.gdn_gated_delta_layer_backward_workspace(1, 63, 1)
    assert per_chunk > 0
    assert lib.gdn_gated_delta_layer_backward_workspace(1, 64, 3) == 2 * 3 * per_chunk  # a packed sequence may begin in any row
    assert lib.gdn_gated_delta_layer_backward_workspace(8, 8 * 65536, 32) == (8 * 1024 + 8) * 32 * per_chunk  # past 32 bits
    assert lib.gdn_gated_delta_layer_backward_workspace(0, 0, 4) == 0
    assert lib.gdn_layer_norm_backward_workspace(0, 128) == 0 < lib.gdn_layer_norm_backward_workspace(1, 128)


def _norm(lib, backward=False, **kw):
    if backward:
        a = dict(dy=A, x=A, weight=A, bias=A, gate=A, rows=4, width=128, eps=1e-5, dtype=1, param=0, dx=A, dweight=A, dbias=A, dgate=A, ws=A, bytes=1 << 30,
                 flags=0, stream=None)
    else:
        a = dict(x=A, weight=A, bias=A, gate=A, rows=4, width=128, eps=1e-5, dtype=1, param=0, y=A, flags=0, stream=None)
    a.update(kw)
    return (lib.gdn_layer_norm_backward if backward else lib.gdn_layer_norm)(*a.values())


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("kw,status", [
    (dict(x=None), "NULL"), (dict(rows=-1), "INVALID_ARG"), (dict(width=0), "INVALID_ARG"), (dict(eps=-1.0), "INVALID_ARG"), (dict(eps=float("nan")), "INVALID_ARG"),
    (dict(dtype=3), "INVALID_ARG"), (dict(param=9), "INVALID_ARG"), (dict(flags=2), "INVALID_ARG"), (dict(width=16385), "UNSUPPORTED"), (dict(gate=A + 2), "ALIGN")])
def test_norm_refuses(lib, backward, kw, status):
    assert _norm(lib, backward, **kw) == getattr(gdn, "GDN_ERR_" + status)


@pytest.mark.parametrize("kw,status", [(dict(dweight=None), "NULL"), (dict(weight=None), "NULL"), (dict(dbias=None), "NULL"), (dict(dgate=None), "NULL"),
                                       (dict(gate=None), "NULL"), (dict(ws=None), "NULL"), (dict(bytes=8), "INVALID_ARG")])
def test_norm_backward_wants_gradients_for_what_it_has(lib, kw, status):
    assert _norm(lib, True, **kw) == getattr(gdn, "GDN_ERR_" + status)


def test_binding_refuses(lib):
    z = torch.zeros
    q, v, b = z(2, 1, 2, 128, dtype=torch.bfloat16), z(2, 1, 4, 128, dtype=torch.bfloat16), z(2, 1, 4)
    with pytest.raises(ValueError):  # host tensors
        gdn.gated_delta_step(q, q, v, b, b, z(2, 4, 128, 128))
    with pytest.raises(ValueError):  # another shape of beta
        gdn.gated_delta_step(q, q, v, z(2, 4, 1), b, z(2, 4, 128, 128))
    with pytest.raises(TypeError):
        gdn.gated_delta_step(q, q, v.float(), b, b, z(2, 4, 128, 128))
    with pytest.raises(ValueError):
        gdn.gated_delta_step(q, q, v, b, b, z(4, 128, 128))
    with pytest.raises(TypeError):
        gdn.gated_delta_step(q, q, v, b, b, z(2, 4, 128, 128), z(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        gdn.gated_delta_layer_backward(v, q, q, v, b, b)
    with pytest.raises(ValueError):  # boundaries that fall
        gdn.gated_delta_layer_backward(v[0], q[0], q[0], v[0], b[0], b[0], cu_seqlens=[0, 1, 0])
    with pytest.raises(ValueError):
        gdn.gated_delta_layer_backward(v[0], q[0], q[0], v[0], b[0], b[0], cu_seqlens=[0, 2])
    with pytest.raises(TypeError):
        gdn.gated_delta_layer_backward(v.float(), q.float(), q.float(), v.float(), b, b)
    with pytest.raises(ValueError):
        gdn.layer_norm(z(3, 128), z(64))
    with pytest.raises(ValueError):
        gdn.layer_norm(z(3, 128), z(128))
    with pytest.raises(TypeError):
        gdn.layer_norm(z(3, 128), z(128), gate=z(3, 128, dtype=torch.bfloat16))


def test_oracle_gradients_against_differences():
    """The oracle's gradients (autograd, fp64) against central differences along random directions: their error is of order h^2."""
    gen = torch.Generator().manual_seed(5)
    rn = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)  # noqa: E731
    x = [rn(5, 1, 8), rn(5, 1, 8), rn(5, 2, 8), torch.sigmoid(rn(5, 2)), -torch.nn.functional.softplus(rn(5, 2)), 0.3 * rn(2, 8, 8)]
    wo, ws = rn(5, 2, 8), rn(2, 8, 8)

    def loss(a):
        o, s = orc.gated_delta_rule(*a)
        return (o * wo).sum() + (s * ws).sum()

    leaves = [t.clone().requires_grad_() for t in x]
    grads = torch.autograd.grad(loss(leaves), leaves)
    for i, t in enumerate(x):
        d, h = rn(*t.shape), 1e-5
        up, down = ([u + s * h * d if j == i else u for j, u in enumerate(x)] for s in (1, -1))
        assert abs((loss(up) - loss(down)) / (2 * h) - (grads[i] * d).sum()) < 1e-7 * (1 + (grads[i] * d).abs().sum())
