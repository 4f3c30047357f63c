"""What the binding refuses before it asks where the tensors live, by the words it refuses it with. No GPU needed: the tensors are on the host."""
import pytest
import torch

from paper_2606_06034_b200 import binding as gdn

z = torch.zeros
H, D = 4, 128


def _tokens(T=2, lead=()):
    q, v, b = z(*lead, T, 2, D, dtype=torch.bfloat16), z(*lead, T, H, D, dtype=torch.bfloat16), z(*lead, T, H)
    return {"Q": q, "K": q, "V": v, "beta": b, "g_raw": b}


@pytest.mark.parametrize("change,error,words", [
    (dict(beta=z(3, H, 2)), ValueError, "beta"),
    (dict(g_raw=z(3, 2, H + 1)), ValueError, "g_raw"),
    (dict(beta=z(3, 2, H, dtype=torch.bfloat16)), TypeError, "fp32"),
    (dict(V=z(3, 2, H, D)), TypeError, "share a dtype"),
    (dict(Q=z(3, 3, 2, D, dtype=torch.bfloat16)), ValueError, "do not belong together"),
    (dict(V=z(2, 2, H, D, dtype=torch.bfloat16)), ValueError, "do not belong together"),
    (dict(S=z(H, D, D)), ValueError, "n_slots,H_v,d_v,d_k"),
    (dict(S=z(3, H, D, 64)), ValueError, "S has shape"),
    (dict(S=z(3, H, D, D, dtype=torch.float16)), TypeError, "S is"),
    (dict(slots=z(2, dtype=torch.int32)), ValueError, "slots has shape"),
    (dict(slots=z(3, dtype=torch.int64)), TypeError, "slots is"),
    (dict(out=z(3, 2, H, D)), TypeError, "out is"),
    (dict(out=z(3, 2, D, H, dtype=torch.bfloat16)), ValueError, "out has shape"),
    (dict(), ValueError, "CUDA device")])
def test_step(change, error, words):
    with pytest.raises(error, match=words):
        gdn.gated_delta_step(**{**_tokens(lead=(3,)), "S": z(3, H, D, D), **change})


@pytest.mark.parametrize("change,error,words", [
    (dict(cu_seqlens=[0, 2, 1, 2]), ValueError, "non-decreasing"),
    (dict(cu_seqlens=[-1, 2]), ValueError, "non-decreasing, from 0"),
    (dict(cu_seqlens=[0, 3]), ValueError, "up to the number of tokens"),
    (dict(cu_seqlens=[]), ValueError, "non-decreasing"),
    (dict(S_in=z(2, H, D, D)), ValueError, "S_in has shape"),
    (dict(dS_out=z(1, H, D, D, dtype=torch.bfloat16)), TypeError, "dS_out is"),
    (dict(dO=z(2, H, D)), TypeError, "dO is"),
    (dict(dO=z(1, H, D, dtype=torch.bfloat16)), ValueError, "dO has shape"),
    (dict(beta=z(H, 2)), ValueError, "beta"),
    (dict(cu_seqlens=None), ValueError, "4 dimensions"),
    (dict(), ValueError, "CUDA device")])
def test_backward(change, error, words):
    x = _tokens()
    with pytest.raises(error, match=words):
        gdn.gated_delta_layer_backward(**{"dO": x["V"], **x, "cu_seqlens": [0, 2], **change})


@pytest.mark.parametrize("change,error,words", [
    (dict(weight=z(64)), ValueError, "weight has shape"),
    (dict(bias=z(D, 1)), ValueError, "bias has shape"),
    (dict(weight=z(D, dtype=torch.float16)), TypeError, "weight is"),
    (dict(weight=z(D), bias=z(D, dtype=torch.bfloat16)), TypeError, "weight and bias share"),
    (dict(gate=z(3, D, dtype=torch.bfloat16)), TypeError, "gate is"),
    (dict(gate=z(2, D)), ValueError, "gate has shape"),
    (dict(x=z(3, D, dtype=torch.float16)), TypeError, "bf16 or fp32"),
    (dict(), ValueError, "CUDA device")])
def test_norm(change, error, words):
    with pytest.raises(error, match=words):
        gdn.layer_norm(**{"x": z(3, D), **change})
    with pytest.raises(error, match=words):
        gdn.layer_norm_backward(**{"dy": change.get("x", z(3, D)), "x": z(3, D), **change})
