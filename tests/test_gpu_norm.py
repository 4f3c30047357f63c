"""Row norms (layer_norm, layer_norm_backward) against their formula in fp64, the gradients by autograd and by differences.

Tolerances, relative 2-norms: one rounding, 2^-8 of each value at most, for bf16 results; for fp32 ones 2e-5: sums with at most 40 additions in a row
(40 x 2^-24 = 2.4e-6 of the sum of magnitudes), the exponential's argument rounded at |z| <= 6 (6 x 2^-23 = 7e-7), its 2 ulp, and the two
subtractions of dx, which cancel by no more than a few times here."""
import pytest
import torch

from oracle import gdn_recurrent as orc
from paper_2606_06034_b200 import binding as gdn

pytestmark = pytest.mark.gpu
TOL = {torch.float32: 2e-5, torch.bfloat16: 2 ** -8 + 2e-5}


def _inputs(rows, width, dtype, weight=True, bias=True, gate=True, params=torch.float32, seed=0):
    gen = torch.Generator().manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    x = {"x": (0.7 * rn(rows, width) + 0.2).to(dtype), "weight": (1 + 0.3 * rn(width)).to(params) if weight else None,
         "bias": (0.2 * rn(width)).to(params) if bias else None, "gate": rn(rows, width).to(dtype) if gate else None, "dy": rn(rows, width).to(dtype)}
    return {k: None if v is None else v.cuda() for k, v in x.items()}


def _near(x, ref, tol, what="", more=0.0):
    err, norm = (x.double() - ref).norm().item(), ref.norm().item()
    assert err <= tol * norm + more, f"{what} {err / max(norm, 1e-300):.3e} > {tol:.1e}"


def _check(s, rms, eps=1e-5):
    names = [n for n in ("x", "weight", "bias", "gate") if s[n] is not None]
    leaf = {n: s[n].double().requires_grad_() for n in names}
    y = orc.row_norm(**{n: leaf.get(n) for n in ("x", "weight", "bias", "gate")}, rms=rms, eps=eps)
    grads = dict(zip(names, torch.autograd.grad((y * s["dy"].double()).sum(), [leaf[n] for n in names])))
    args = [s[n] for n in ("x", "weight", "bias", "gate")]
    dtype = s["x"].dtype
    # dx = rstd (dn - mean(dn) - n mean(dn n)): with two features and a mean nothing but eps is left of it (a row of two values, of mean 0 and norm
    # sqrt(2), has no freedom), so its error is measured by its terms: three of at most rstd ||dn|| each, n and rstd off by 4 x 2^-24 and four more
    # roundings: 3 x 8 x 2^-24
    h = s["dy"].double() * (1 if s["gate"] is None else s["gate"].double() * torch.sigmoid(s["gate"].double())) * (1 if s["weight"] is None else s["weight"].double())
    x = s["x"].double()
    rstd = ((x if rms else x - x.mean(-1, keepdim=True)).square().mean(-1, keepdim=True) + eps).rsqrt()
    terms = 24 * 2 ** -24 * (rstd * h).norm().item()
    _near(gdn.layer_norm(*args, rms=rms, eps=eps), y.detach(), TOL[dtype], "y")
    got = dict(zip(("x", "weight", "bias", "gate"), gdn.layer_norm_backward(s["dy"], *args, rms=rms, eps=eps)))
    for n in ("x", "weight", "bias", "gate"):
        assert (got[n] is None) == (s[n] is None)
        if n in names:
            _near(got[n], grads[n], TOL[torch.float32] if n in ("weight", "bias") else TOL[dtype], n, terms if n == "x" else 0.0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("rows,width", [(1, 2), (5, 3), (1000, 128), (33, 77), (17, 200), (9, 256), (50, 504), (21, 1000), (8, 1024), (5, 2048), (700, 2056), (3, 4099),
                                        (300, 4096), (11, 8192), (2, 16384), (3, 12345)])
def test_norm(dtype, rms, rows, width):
    _check(_inputs(rows, width, dtype, seed=width), rms)


@pytest.mark.parametrize("weight,bias,gate", [(False, False, False), (True, False, False), (False, True, False), (False, False, True), (True, False, True), (False, True, True)])
@pytest.mark.parametrize("width", [128, 75, 1500])
def test_missing_parts(weight, bias, gate, width):
    _check(_inputs(40, width, torch.float32, weight, bias, gate, seed=3), True)
    _check(_inputs(40, width, torch.bfloat16, weight, bias, gate, torch.bfloat16, seed=4), False)


def test_one_feature_and_no_rows():
    s = _inputs(7, 1, torch.float32, gate=False)
    assert torch.equal(gdn.layer_norm(s["x"], s["weight"], s["bias"]), s["bias"].expand(7, 1))  # (x - mean = 0)
    s = _inputs(0, 128, torch.bfloat16)
    assert gdn.layer_norm(s["x"], s["weight"], s["bias"], s["gate"]).shape == (0, 128)
    dx, dw, db, dz = gdn.layer_norm_backward(s["dy"], s["x"], s["weight"], s["bias"], s["gate"])
    assert dx.shape == dz.shape == (0, 128) and not dw.any() and not db.any()


def test_leading_dimensions_in_place_and_large_gates():
    s = _inputs(6, 128, torch.float32)
    s["gate"] *= 30  # beyond where the exponential over- and underflows
    s["gate"][0, :4] = torch.tensor([100.0, -100.0, 1000.0, -1000.0], device="cuda")
    ref = orc.row_norm(*(s[n].double() for n in ("x", "weight", "bias", "gate")), rms=True)
    x = s["x"].view(2, 3, 128).clone()
    y = gdn.layer_norm(x, s["weight"], s["bias"], s["gate"].view(2, 3, 128), rms=True, out=x)
    assert y is x
    # (the exponential's argument is rounded at |z| <= 1000, where the result is 0 or z: 90 x 2^-23 where it matters)
    _near(y.view(6, 128), ref, 4e-5)


def test_a_row_that_is_not_finite_stays_alone():
    s = _inputs(64, 128, torch.bfloat16)
    clean = gdn.layer_norm(s["x"], s["weight"], s["bias"], s["gate"])
    s["x"][5, 3], s["x"][9, 0] = float("nan"), float("inf")
    y = gdn.layer_norm(s["x"], s["weight"], s["bias"], s["gate"])
    others = [i for i in range(64) if i not in (5, 9)]
    assert torch.equal(y[others], clean[others]) and y[5].isnan().all() and not y[9].isfinite().all()


def test_constant_rows():
    x = torch.full((3, 256), 7.0, device="cuda")
    assert not gdn.layer_norm(x).any()
    _near(gdn.layer_norm(x, rms=True), torch.ones(3, 256, dtype=torch.float64, device="cuda"), 2e-5)


def test_repeatable_and_captured():
    s = _inputs(20000, 128, torch.bfloat16)
    args = (s["dy"], s["x"], s["weight"], s["bias"], s["gate"])
    a, b = gdn.layer_norm_backward(*args), gdn.layer_norm_backward(*args)
    assert all(torch.equal(x, y) for x, y in zip(a, b))  # the order of every sum depends on the shape alone
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c = gdn.layer_norm_backward(*args)
    s["dy"].mul_(2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(c[1], 2 * a[1]) and torch.equal(c[0], 2 * a[0])  # (a factor of two changes no rounding)


def test_many_rows_and_few_bytes_past_32_bits():
    rows = (1 << 31) // 8 + 3
    x = torch.zeros(rows, 8, dtype=torch.bfloat16, device="cuda")
    x[-1] = torch.arange(8)
    y = gdn.layer_norm(x, out=x)
    ref = orc.row_norm(torch.arange(8, dtype=torch.float64, device="cuda")[None])[0]
    _near(y[-1], ref, TOL[torch.bfloat16])
    assert not y[:-1:65537].any()
