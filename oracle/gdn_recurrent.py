"""The gated delta rule and the row norm by their definitions, in the precision of what they are given (the tests give fp64), differentiable."""
from __future__ import annotations

import torch


def unit_rows(x):
    """Rows of unit length; rows of zeros stay zero (and have no gradient)."""
    n2 = x.square().sum(-1, keepdim=True)
    return torch.where(n2 > 0, x * torch.where(n2 > 0, n2, 1.0).rsqrt(), 0.0)


def gated_delta_rule(q, k, v, beta, g, S=None, scale=None, qk_l2norm=True):
    """Token by token. q, k [T,H_k,d_k], v [T,H_v,d_v], beta, g [T,H_v], S [H_v,d_v,d_k]. Returns (o [T,H_v,d_v], S)."""
    T, H_v, d_v = v.shape
    H_k, d_k = k.shape[1:]
    scale = d_k ** -0.5 if scale is None else scale
    if qk_l2norm:
        q, k = unit_rows(q), unit_rows(k)
    q, k = (x.repeat_interleave(H_v // H_k, 1) for x in (q, k))
    S = torch.zeros(H_v, d_v, d_k, dtype=v.dtype, device=v.device) if S is None else S
    out = []
    for t in range(T):
        S = S * g[t].exp()[:, None, None]
        u = beta[t][:, None] * (v[t] - (S @ k[t][..., None])[..., 0])
        S = S + u[..., None] * k[t][:, None, :]
        out.append(scale * (S @ q[t][..., None])[..., 0])
    return (torch.stack(out) if out else torch.zeros_like(v)), S


def row_norm(x, weight=None, bias=None, gate=None, rms=False, eps=1e-5):
    x = x if rms else x - x.mean(-1, keepdim=True)
    h = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    h = h if weight is None else h * weight
    h = h if bias is None else h + bias
    return h if gate is None else h * gate * torch.sigmoid(gate)
