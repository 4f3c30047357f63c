"""Performance cases of the layer's operators around the chunk-wise forward pass: what decoding and training have them do.

A case is a dict of plain values. Kinds:

  step       `gated_delta_step`: one or a few new tokens per sequence on a pool of states, updated in place
  grad       `gated_delta_layer_backward` on dense [B,T,H,d] tensors
  packed     the same on sequences of different lengths laid end to end (`cu_seqlens`)
  norm       `layer_norm`: the rows of the layer's output normalised and gated, or a block's plain layer norm
  norm_grad  `layer_norm_backward` of the same, with the gradients of weight and bias

`run` computes them from elementary torch operations in fp32, or with `own` through the library's binding.
"""
from __future__ import annotations

import math
import random

import torch

own = False

D = 128  # feature size of the layer's heads
C = 64   # chunk size
EPS = 1e-6


def _step(name, B, H_k, H_v, T, pool, pad, state):
    return {"name": name, "kind": "step", "B": B, "H_k": H_k, "H_v": H_v, "T": T, "pool": pool, "pad": pad, "state": state}


def _grad(name, B, H_k, H_v, T, carry):
    return {"name": name, "kind": "grad", "B": B, "H_k": H_k, "H_v": H_v, "T": T, "carry": carry}


def _packed(name, H_k, H_v, T, n_seq, pattern):
    return {"name": name, "kind": "packed", "B": 1, "H_k": H_k, "H_v": H_v, "T": T, "n_seq": n_seq, "pattern": pattern, "carry": False}


def _norm(name, kind, rows, width, rms, gated, bias, dtype):
    return {"name": name, "kind": kind, "rows": rows, "width": width, "rms": rms, "gated": gated, "bias": bias, "dtype": dtype}


def listed():
    return [
        # one conversation: the next token of a single sequence, where a launch's latency is what counts
        _step("step_one", 1, 16, 32, 1, 1, 0, "fp32"),
        # a serving batch: 256 sequences in a pool of 320 states, a few rows of the batch padded
        _step("step_batch", 256, 16, 32, 1, 320, 5, "fp32"),
        # four drafted tokens for each of 32 sequences, states kept in bf16
        _step("step_draft", 32, 16, 32, 4, 48, 0, "bf16"),
        # fine-tuning on one short text
        _grad("grad_short", 1, 16, 32, 200, False),
        # a training batch
        _grad("grad_batch", 8, 32, 32, 4096, False),
        # one long document, with a state carried in from the text before it
        _grad("grad_long", 1, 16, 32, 32768, True),
        # a training batch of texts of very different lengths packed end to end, none of them a multiple of the chunk
        _packed("grad_packed", 16, 32, 16411, 61, 7),
        # the layer's output of one decoded token of a batch of 16
        _norm("norm_token", "norm", 16 * 32, D, True, True, False, "bf16"),
        # the layer's output over a prompt of 32768 tokens
        _norm("norm_prefill", "norm", 32768 * 32, D, True, True, False, "bf16"),
        # its backward pass over the training batch
        _norm("norm_grad_batch", "norm_grad", 8 * 4096 * 32, D, True, True, False, "bf16"),
        # a block's layer norm at the model's width: training, fp32 rows of a ragged batch
        _norm("norm_wide", "norm", 4099, 4096, False, False, True, "fp32"),
        _norm("norm_grad_wide", "norm_grad", 8 * 2048, 4096, False, False, True, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["step", "step", "step", "grad", "grad", "packed", "packed", "norm", "norm_grad"])
    H_k = rng.choice([1, 2, 3, 4, 6, 8, 12, 16, 24, 32])
    H_v = H_k * rng.choice([1, 1, 2, 4])
    if kind == "step":
        T = rng.choice([1, 1, 1, 2, 3, 5, 8])
        B = max(1, _log_int(rng, 1, 8192 // T) // H_v)
        return _step("", B, H_k, H_v, T, B + rng.randrange(0, B + 1), rng.randrange(0, B // 4 + 1), rng.choice(["fp32", "fp32", "bf16"]))
    if kind == "grad":
        B = rng.choice([1, 1, 1, 2, 3, 4, 8])
        T = max(1, _log_int(rng, 256, 1 << 19) // (B * H_v))
        return _grad("", B, H_k, H_v, T, rng.random() < 0.5)
    if kind == "packed":
        T = max(8, _log_int(rng, 512, 1 << 19) // H_v)
        return _packed("", H_k, H_v, T, min(T, _log_int(rng, 1, 128)), rng.randrange(1 << 16))
    values = _log_int(rng, 1 << 12, 1 << 26)
    if rng.random() < 0.5:  # rows of a head's features
        width, rms, gated, bias = rng.choice([64, 96, 128, 128, 200, 256]), True, True, False
    else:
        width, rms, gated, bias = _log_int(rng, 3, 8192), rng.random() < 0.5, rng.random() < 0.3, rng.random() < 0.5
    return _norm("", kind, max(1, values // width), width, rms, gated, bias, rng.choice(["bf16", "bf16", "fp32"]))


def _boundaries(case):
    """Sequence boundaries of a packed case: lengths log-normal around their mean (a few long texts, many short ones)."""
    r = random.Random(case["pattern"])
    w = [r.lognormvariate(0.0, 1.0) for _ in range(case["n_seq"])]
    spare = case["T"] - case["n_seq"]  # every sequence has at least one token
    total, acc, cu = sum(w), 0.0, [0]
    for i, x in enumerate(w):
        acc += x
        cu.append(i + 1 + int(spare * acc / total))
    cu[-1] = case["T"]
    return cu


def _chunk_plan(cu):
    """Chunks of the sequences [cu[s], cu[s+1]) for the plain form, the sequences from the longest down: the n-th chunks of all
    sequences that have one are neighbours, and belong to the first sequences of that order."""
    order = sorted(range(len(cu) - 1), key=lambda s: cu[s] - cu[s + 1])
    first, size, steps, t0 = [], [], [0], 0
    while True:
        alive = [s for s in order if cu[s] + t0 < cu[s + 1]]
        if not alive:
            break
        first += [cu[s] + t0 for s in alive]
        size += [min(C, cu[s + 1] - cu[s] - t0) for s in alive]
        steps.append(len(first))
        t0 += C
    first, size = torch.tensor(first, device="cuda"), torch.tensor(size, device="cuda")
    row = torch.arange(C, device="cuda")
    ok = row < size[:, None]
    at = torch.where(ok, first[:, None] + row, first[:, None])
    return {"at": at, "ok": ok, "tokens": at[ok], "steps": steps, "order": torch.tensor(order, device="cuda")}


def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device=dev, dtype=torch.float32)

    kind = case["kind"]
    if kind in ("norm", "norm_grad"):
        rows, width = case["rows"], case["width"]
        dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        st = {"case": case, "x": (0.7 * randn(rows, width) + 0.1).to(dtype), "weight": 1 + 0.2 * randn(width),
              "bias": 0.1 * randn(width) if case["bias"] else None, "gate": randn(rows, width).to(dtype) if case["gated"] else None}
        if kind == "norm_grad":
            st["dy"] = randn(rows, width).to(dtype)
        return st
    B, T, H_k, H_v = case["B"], case["T"], case["H_k"], case["H_v"]
    lead = (T,) if kind == "packed" else (B, T)
    st = {"case": case, "Q": randn(*lead, H_k, D).bfloat16(), "K": randn(*lead, H_k, D).bfloat16(), "V": randn(*lead, H_v, D).bfloat16(),
          "beta": torch.sigmoid(randn(*lead, H_v)), "g": -torch.nn.functional.softplus(randn(*lead, H_v))}
    if kind == "step":
        st["S"] = (0.3 * randn(case["pool"], H_v, D, D)).to(torch.bfloat16 if case["state"] == "bf16" else torch.float32)
        live = B - case["pad"]
        slots = torch.randperm(case["pool"], generator=gen, device=dev)[:B].to(torch.int32)
        slots[live:] = -1  # the batch is padded to a fixed size
        st["slots"], st["live"] = slots, slots[:live].long()
        return st
    st["dO"] = randn(*lead, H_v, D).bfloat16()
    st["S_in"] = 0.3 * randn(B, H_v, D, D) if case["carry"] else None
    st["dS_out"] = 0.1 * randn(B, H_v, D, D) if case["carry"] else None
    st["cu"] = _boundaries(case) if kind == "packed" else [b * T for b in range(B + 1)]
    st["plan"] = _chunk_plan(st["cu"])
    return st


# ---------------------------------------------------------------- plain forms, fp32
def _unit(x):
    """Rows of unit length, and one over their lengths."""
    r = x.square().sum(-1, keepdim=True).rsqrt()
    return x * r, r


def _plain_step(st):
    case = st["case"]
    group, n = case["H_v"] // case["H_k"], st["live"].numel()
    q, k = (_unit(st[x][:n].float())[0].repeat_interleave(group, 2) for x in ("Q", "K"))
    v, beta, a = st["V"][:n].float(), st["beta"][:n], st["g"][:n].exp()
    S = st["S"][st["live"]].float()
    O = torch.zeros_like(st["V"])
    for t in range(case["T"]):
        S = S * a[:, t, :, None, None]
        u = beta[:, t, :, None] * (v[:, t] - (S @ k[:, t, :, :, None])[..., 0])
        S = S + u[..., None] * k[:, t, :, None, :]
        O[:n, t] = (D ** -0.5 * (S @ q[:, t, :, :, None])[..., 0]).to(O.dtype)
    st["S"][st["live"]] = S.to(st["S"].dtype)
    return O, st["S"]


def _plain_grad(st):
    case, plan = st["case"], st["plan"]
    H_k, H_v = case["H_k"], case["H_v"]
    group, scale = H_v // H_k, D ** -0.5
    at, ok, steps = plan["at"], plan["ok"], plan["steps"]
    dense = case["kind"] == "grad"

    def chunks(name):  # [chunks, heads, tokens, ...], zeros behind a sequence's end
        x = st[name].flatten(0, 1) if dense else st[name]
        x = x[at].float()
        return torch.where(ok.view(ok.shape + (1,) * (x.dim() - 2)), x, 0.0).transpose(1, 2)

    def unit(x):
        r = torch.where(ok[:, None, :, None], x.square().sum(-1, keepdim=True).rsqrt(), 0.0)
        return (x * r).repeat_interleave(group, 1), r

    (q, rq), (k, rk) = unit(chunks("Q")), unit(chunks("K"))
    v, dO, beta, g = chunks("V"), chunks("dO"), chunks("beta")[..., None], chunks("g").cumsum(-1)
    gl = g[..., -1:, None]
    gam = (g[..., :, None] - g[..., None, :]).tril().exp().tril()
    low = gam.tril(-1)
    g = g[..., None]
    eg, ec = g.exp(), (gl - g).exp()
    kk = (k @ k.transpose(-1, -2)) * low
    X = -beta * kk
    T = torch.eye(C, device=X.device) + X
    for _ in range(5):  # (I - X)^-1 = (I + X)(I + X^2)(I + X^4)...: X^64 = 0
        X = X @ X
        T = T + X @ T
    qk = scale * gam * (q @ k.transpose(-1, -2))
    # the states, forward
    n_seq = steps[1] if len(steps) > 1 else 0
    order = plan["order"]
    S = torch.zeros(n_seq, H_v, D, D, device=v.device) if st["S_in"] is None else st["S_in"][order]
    S0, u = torch.empty(v.shape[:2] + (D, D), device=v.device), torch.empty_like(v)
    for lo, hi in zip(steps[:-1], steps[1:]):
        s = S[:hi - lo]
        S0[lo:hi] = s
        u[lo:hi] = T[lo:hi] @ (beta[lo:hi] * (v[lo:hi] - eg[lo:hi] * (k[lo:hi] @ s.transpose(-1, -2))))
        S[:hi - lo] = gl[lo:hi].exp() * s + u[lo:hi].transpose(-1, -2) @ (ec[lo:hi] * k[lo:hi])
    # their gradients, backward
    G = torch.zeros_like(S) if st["dS_out"] is None else st["dS_out"][order]
    G1, r = torch.empty_like(S0), torch.empty_like(v)
    for lo, hi in zip(reversed(steps[:-1]), reversed(steps[1:])):
        d = G[:hi - lo]
        G1[lo:hi] = d
        du = qk[lo:hi].transpose(-1, -2) @ dO[lo:hi] + (ec[lo:hi] * k[lo:hi]) @ d.transpose(-1, -2)
        r[lo:hi] = T[lo:hi].transpose(-1, -2) @ du
        G[:hi - lo] = (gl[lo:hi].exp() * d + dO[lo:hi].transpose(-1, -2) @ (scale * eg[lo:hi] * q[lo:hi])
                       - r[lo:hi].transpose(-1, -2) @ (beta[lo:hi] * eg[lo:hi] * k[lo:hi]))
    # the chunks' own
    p = (dO @ u.transpose(-1, -2)) * gam * scale
    dq_state, dk_end = scale * eg * (dO @ S0), ec * (u @ G1)
    kS = eg * (k @ S0.transpose(-1, -2))
    ru = -(r @ u.transpose(-1, -2)).tril(-1)
    m = beta * low * ru
    dq = dq_state + p @ k
    dk = p.transpose(-1, -2) @ q + dk_end - beta * eg * (r @ S0) + m @ k + m.transpose(-1, -2) @ k
    dv = beta * r
    dbeta = (r * (v - kS)).sum(-1) + (ru * kk).sum(-1)
    pair = p * (q @ k.transpose(-1, -2)) + ru * beta * kk
    end = (dk_end * k).sum(-1)
    dg = pair.sum(-1) - pair.sum(-2) + (dq_state * q).sum(-1) - (beta * r * kS).sum(-1) - end
    dg[..., -1] += end.sum(-1) + gl[..., 0, 0].exp() * (G1 * S0).sum((-1, -2))
    dg = dg.flip(-1).cumsum(-1).flip(-1)

    def shared(d, x, inv):  # heads of a group summed, then through the norm of the row
        d = d.unflatten(1, (H_k, group)).sum(2)
        x = x[:, ::group]
        return inv * (d - x * (x * d).sum(-1, keepdim=True))

    def tokens(x, like):
        out = torch.empty(like.shape, dtype=like.dtype, device=like.device)
        (out.flatten(0, 1) if dense else out)[plan["tokens"]] = x.transpose(1, 2)[ok].to(like.dtype)
        return out

    back = torch.empty_like(G)
    back[order] = G
    return {"dQ": tokens(shared(dq, q, rq), st["Q"]), "dK": tokens(shared(dk, k, rk), st["K"]), "dV": tokens(dv, st["V"]),
            "dbeta": tokens(dbeta, st["beta"]), "dg": tokens(dg, st["g"]), "dS_in": back if st["S_in"] is not None else None}


def _plain_norm(st):
    x, rms = st["x"].float(), st["case"]["rms"]
    x = x if rms else x - x.mean(-1, keepdim=True)
    n = x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
    h = n * st["weight"] if st["bias"] is None else n * st["weight"] + st["bias"]
    if st["gate"] is not None:
        z = st["gate"].float()
        h = h * z / (1 + (-z).exp())
    return h.to(st["x"].dtype)


def _plain_norm_grad(st):
    x, rms, dh = st["x"].float(), st["case"]["rms"], st["dy"].float()
    x = x if rms else x - x.mean(-1, keepdim=True)
    inv = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
    n = x * inv
    out = {}
    if st["gate"] is not None:
        z = st["gate"].float()
        s = 1 / (1 + (-z).exp())
        h = n * st["weight"] if st["bias"] is None else n * st["weight"] + st["bias"]
        out["dgate"] = (dh * h * s * (1 + z * (1 - s))).to(st["gate"].dtype)
        dh = dh * z * s
    out["dweight"] = (dh * n).sum(0, dtype=torch.float64).float()
    if st["bias"] is not None:
        out["dbias"] = dh.sum(0, dtype=torch.float64).float()
    dn = dh * st["weight"]
    dx = dn - n * (dn * n).mean(-1, keepdim=True)
    out["dx"] = (inv * (dx if rms else dx - dn.mean(-1, keepdim=True))).to(st["x"].dtype)
    return out


# ---------------------------------------------------------------- the library's operators
def _own(st):
    from paper_2606_06034_b200 import binding as gdn

    kind = st["case"]["kind"]
    if kind == "step":
        return gdn.gated_delta_step(st["Q"], st["K"], st["V"], st["beta"], st["g"], st["S"], st["slots"]), st["S"]
    if kind in ("grad", "packed"):
        got = gdn.gated_delta_layer_backward(st["dO"], st["Q"], st["K"], st["V"], st["beta"], st["g"], S_in=st["S_in"], dS_out=st["dS_out"],
                                             cu_seqlens=st["cu"] if kind == "packed" else None)
        return dict(zip(("dQ", "dK", "dV", "dbeta", "dg", "dS_in"), got))
    if kind == "norm":
        return gdn.layer_norm(st["x"], st["weight"], st["bias"], st["gate"], rms=st["case"]["rms"], eps=EPS)
    got = gdn.layer_norm_backward(st["dy"], st["x"], st["weight"], st["bias"], st["gate"], rms=st["case"]["rms"], eps=EPS)
    return {n: x for n, x in zip(("dx", "dweight", "dbias", "dgate"), got) if x is not None}


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind == "step":
        return _plain_step(state)
    if kind in ("grad", "packed"):
        return _plain_grad(state)
    return _plain_norm(state) if kind == "norm" else _plain_norm_grad(state)


def work(case):
    """Every input read once, every output written once; multiply-adds of the recurrence (step), or of the chunked form's products
    on the triangles it needs, forward states and backward (grad)."""
    kind = case["kind"]
    if kind in ("norm", "norm_grad"):
        n = case["rows"] * case["width"]
        e = 2 if case["dtype"] == "bf16" else 4
        tensors = 2 + case["gated"] if kind == "norm" else 3 + 2 * case["gated"]
        params = (1 + case["bias"]) * (1 if kind == "norm" else 2)
        return {"bytes": e * n * tensors + 4 * case["width"] * params, "flops": n * (8 if kind == "norm" else 20)}
    B, T, H_k, H_v = case["B"], case["T"], case["H_k"], case["H_v"]
    keys, vals = B * T * H_k, B * T * H_v
    if kind == "step":
        e = 2 if case["state"] == "bf16" else 4
        live = B - case["pad"]
        return {"bytes": 2 * e * live * H_v * D * D + 2 * D * (2 * keys + 2 * vals) + 8 * vals, "flops": 7 * live * T * H_v * D * D}
    states = 4 * D * D * H_v * B * (3 if case["carry"] else 0)
    # full products: k S, u k, k D, dO q, r k, dO S, u D, r S; on triangles: k k, q k, the inverse, T R, P dO, T r, dO u, its two, r u, its two
    return {"bytes": 2 * D * (4 * keys + 3 * vals) + 16 * vals + states,
            "flops": vals * (16 * D * D + 9 * C * D + C * C / 3) + 2 * keys * C * D}


# ---------------------------------------------------------------- the definitions in 64 bits
def _exact_step(case, st):
    group, n = case["H_v"] // case["H_k"], case["B"] - case["pad"]
    S = st["S"].double()
    O = torch.zeros(st["V"].shape, dtype=torch.float64, device="cuda")
    key = torch.arange(case["H_v"], device="cuda") // group
    for b in range(n):
        s = S[st["slots"][b].long()]
        for t in range(case["T"]):
            q, k = (torch.nn.functional.normalize(st[x][b, t].double(), dim=-1, eps=1e-300)[key] for x in ("Q", "K"))
            s *= st["g"][b, t].double().exp()[:, None, None]
            u = st["beta"][b, t].double()[:, None] * (st["V"][b, t].double() - torch.einsum("hvk,hk->hv", s, k))
            s += torch.einsum("hv,hk->hvk", u, k)
            O[b, t] = torch.einsum("hvk,hk->hv", s, q) * D ** -0.5
        S[st["slots"][b].long()] = s
    return O, S


def _forward64(q, k, v, beta, g, S):
    """The layer in fp64 on sequences of one length: q, k, v [n, H, T, d], beta, g [n, H, T]; outputs and the last state."""
    out = []
    for t0 in range(0, v.shape[2], C):
        qc, kc, vc, bc, gc = (x[:, :, t0:t0 + C] for x in (q, k, v, beta, g))
        gc = gc.cumsum(-1)
        diff = gc[..., :, None] - gc[..., None, :]
        keep = torch.ones_like(diff[0, 0], dtype=torch.bool).tril()
        gam = torch.where(keep, diff, -torch.inf).exp()
        L = bc[..., None] * gam.tril(-1) * (kc @ kc.transpose(-1, -2)) + torch.eye(vc.shape[2], dtype=vc.dtype, device=vc.device)
        e = gc.exp()[..., None]
        u = torch.linalg.solve_triangular(L, bc[..., None] * (vc - e * (kc @ S.transpose(-1, -2))), upper=False, unitriangular=True)
        out.append(D ** -0.5 * (e * (qc @ S.transpose(-1, -2)) + ((qc @ kc.transpose(-1, -2)) * gam) @ u))
        last = gc[..., -1:]
        S = last[..., None].exp() * S + (u * (last - gc).exp()[..., None]).transpose(-1, -2) @ kc
    return torch.cat(out, 2), S


def _exact_grad(case, st):
    H_k, H_v = case["H_k"], case["H_v"]
    dense = case["kind"] == "grad"
    names = ("Q", "K", "V", "beta", "g")
    flat = {n: (st[n].flatten(0, 1) if dense else st[n]) for n in names + ("dO",)}
    got = {n: torch.empty(flat[n].shape, dtype=torch.float64, device="cuda") for n in names}
    dS = torch.empty(len(st["cu"]) - 1, H_v, D, D, dtype=torch.float64, device="cuda")
    for s in range(len(st["cu"]) - 1):
        a, b = st["cu"][s], st["cu"][s + 1]
        with torch.enable_grad():
            leaf = {n: flat[n][a:b].double().requires_grad_() for n in names}
            q, k = (torch.nn.functional.normalize(leaf[n], dim=-1, eps=1e-300).repeat_interleave(H_v // H_k, 1).transpose(0, 1)[None] for n in ("Q", "K"))
            v, beta, g = (leaf[n].transpose(0, 1)[None] for n in ("V", "beta", "g"))
            S = (torch.zeros(H_v, D, D, dtype=torch.float64, device="cuda") if st["S_in"] is None else st["S_in"][s].double()).requires_grad_()
            o, end = _forward64(q, k, v, beta, g, S[None])
            loss = (o[0] * flat["dO"][a:b].double().transpose(0, 1)).sum()
            if st["dS_out"] is not None:
                loss = loss + (end[0] * st["dS_out"][s].double()).sum()
            grads = torch.autograd.grad(loss, [leaf[n] for n in names] + [S])
        for n, d in zip(names, grads):
            got[n][a:b] = d
        dS[s] = grads[-1]
    out = {"d" + n: got[n].view(st[n].shape) for n in names}
    out["dS_in"] = dS if st["S_in"] is not None else None
    return out


def _exact_norm(case, st, grad):
    names = [n for n in ("x", "weight", "bias", "gate") if st[n] is not None]
    parts, sums = [], {}
    rows = max(1, (1 << 24) // case["width"])
    for a in range(0, case["rows"], rows):
        with torch.enable_grad():
            leaf = {n: (st[n][a:a + rows] if n in ("x", "gate") else st[n]).double().requires_grad_() for n in names}
            x = leaf["x"]
            if case["rms"]:
                h = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
            else:
                h = (x - x.mean(-1, keepdim=True)) / torch.sqrt(x.var(-1, unbiased=False, keepdim=True) + EPS)
            h = h * leaf["weight"]
            if "bias" in leaf:
                h = h + leaf["bias"]
            if "gate" in leaf:
                h = h * leaf["gate"] * torch.sigmoid(leaf["gate"])
            if not grad:
                parts.append(h.detach())
                continue
            got = dict(zip(names, torch.autograd.grad((h * st["dy"][a:a + rows].double()).sum(), [leaf[n] for n in names])))
        parts.append([got.get("x"), got.get("gate")])
        for n in ("weight", "bias"):
            if n in got:
                sums[n] = sums.get(n, 0) + got[n]
    if not grad:
        return torch.cat(parts)
    out = {"dx": torch.cat([p[0] for p in parts]), "dweight": sums["weight"]}
    if "bias" in sums:
        out["dbias"] = sums["bias"]
    if case["gated"]:
        out["dgate"] = torch.cat([p[1] for p in parts])
    return out


def exact(case, seed):
    """What `run` returns for these inputs, from the definitions in fp64: the recurrence token by token, autograd through the
    chunks' triangular systems, autograd through the norm's formula."""
    st = prepare(case, seed)
    if case["kind"] == "step":
        return _exact_step(case, st)
    if case["kind"] in ("grad", "packed"):
        return _exact_grad(case, st)
    return _exact_norm(case, st, case["kind"] == "norm_grad")
