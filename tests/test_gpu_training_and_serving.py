"""The operators together, as a model uses them: a training step of the layer with its output norm, and a prompt followed by decoded tokens."""
import pytest
import torch

from oracle import gdn_recurrent as orc
from paper_2606_06034_b200 import binding as gdn

pytestmark = pytest.mark.gpu
D = 128


def _near(x, ref, tol, what):
    err, norm = (x.double() - ref).norm().item(), ref.norm().item()
    assert err <= tol * norm, f"{what}: {err / norm:.3e} > {tol:.1e}"


def _inputs(B, T, H_k, H_v, seed):
    gen = torch.Generator().manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    return [t.cuda() for t in (rn(B, T, H_k, D).bfloat16(), rn(B, T, H_k, D).bfloat16(), rn(B, T, H_v, D).bfloat16(), torch.sigmoid(rn(B, T, H_v)),
                               -torch.nn.functional.softplus(rn(B, T, H_v)))]


def test_training_step():
    """Layer, gated RMS norm, and back. O and dO pass through bf16 (2^-8 each), W and U of the forward pass too: four roundings, 2^-6."""
    B, T, H_k, H_v = 2, 192, 1, 2
    x = _inputs(B, T, H_k, H_v, 1)
    gen = torch.Generator().manual_seed(2)
    weight, gate, dy = (1 + 0.2 * torch.randn(D, generator=gen)).cuda(), torch.randn(B, T, H_v, D, generator=gen).bfloat16().cuda(), torch.randn(B, T, H_v, D, generator=gen).bfloat16().cuda()
    O, _ = gdn.gated_delta_layer(*x, want_state=False)
    y = gdn.layer_norm(O, weight, gate=gate, rms=True, eps=1e-6)
    dO, dweight, _, dgate = gdn.layer_norm_backward(dy, O, weight, gate=gate, rms=True, eps=1e-6)
    got = gdn.gated_delta_layer_backward(dO, *x)
    leaf = [t.double().requires_grad_() for t in x]
    w, z = weight.double().requires_grad_(), gate.double().requires_grad_()
    o = torch.stack([orc.gated_delta_rule(*(t[b] for t in leaf))[0] for b in range(B)])
    ref = orc.row_norm(o, w, None, z, rms=True, eps=1e-6)
    grads = torch.autograd.grad((ref * dy.double()).sum(), leaf + [w, z])
    _near(y, ref.detach(), 2 ** -6, "y")
    for n, a, b in zip(("dQ", "dK", "dV", "dbeta", "dg", "dweight", "dgate"), (*got[:5], dweight, dgate), grads):
        _near(a, b, 2 ** -6, n)


def test_prompt_then_decoded_tokens():
    """The state that the chunk-wise layer leaves goes on in the decoding step's pool; outputs pass the norm."""
    B, T, new, H_k, H_v = 3, 128, 5, 2, 4
    x = _inputs(B, T + new, H_k, H_v, 3)
    head, tail = [t[:, :T].contiguous() for t in x], [t[:, T:].contiguous() for t in x]
    _, S = gdn.gated_delta_layer(*head)
    pool = torch.zeros(8, H_v, D, D, device="cuda")
    slots = torch.tensor([6, 1, 4], dtype=torch.int32, device="cuda")
    pool[slots.long()] = S
    out = [gdn.layer_norm(gdn.gated_delta_step(*(t[:, i:i + 1].contiguous() for t in tail), pool, slots), rms=True) for i in range(new - 2)]
    out.append(gdn.layer_norm(gdn.gated_delta_step(*(t[:, new - 2:].contiguous() for t in tail), pool, slots), rms=True))  # two at once
    got = torch.cat(out, 1)
    for b in range(B):
        o, end = orc.gated_delta_rule(*(t[b].double() for t in x))
        _near(got[b], orc.row_norm(o[T:], rms=True), 2 ** -7 + 5e-3, "tokens")  # (two roundings, and the prompt's state: W and U in bf16)
        _near(pool[slots[b].long()], end, 5e-3, "state")
