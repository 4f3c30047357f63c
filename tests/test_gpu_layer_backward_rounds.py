"""The last kernel's loop over (chunk, key head) units, 148 CTAs taking every 148th: units beyond a CTA's second one, full chunks behind short ones, places
of a packed layout that hold no chunk. Tolerances as in test_gpu_layer_backward.py; a sequence's gradients do not depend on what else is in
the call, bit for bit."""
import random

import pytest
import torch

from paper_2606_06034_b200 import binding as gdn
from test_gpu_layer_backward import NAMES, _call, _check, _dense, _expected, _inputs

pytestmark = pytest.mark.gpu


def test_more_than_three_rounds_with_short_chunks_and_groups_of_three():
    B, T, H_k, H_v = 5, 500, 12, 36
    assert B * (T // 64 + 1) * H_k > 3 * 148 and T % 64
    x = _inputs(B * T, H_k, H_v, 61, B)
    got = _call(_dense(x, B, T), x)
    assert gdn.gdn_device_status() == gdn.GDN_OK
    for b in range(B):
        part = {n: x[n][b * T:(b + 1) * T] for n in (*NAMES, "dO")} | {"S": x["S"][b:b + 1], "dS": x["dS"][b:b + 1]}
        alone = _call(_dense(part, 1, T), part)
        assert all(torch.equal(p[b], q[0]) for p, q in zip(got, alone))
        if b in (0, B - 1):
            ref, dS = _expected(part, [0, T])
            _check([t[b] for t in got[:5]] + [got[5][b:b + 1]], ref, dS)


@pytest.mark.parametrize("token_major", [True, False])
def test_many_short_sequences_and_empty_ones(token_major):
    """Sequence s starts at place cu[s] / 64 + s of the workspace: with sequences shorter than a chunk, and empty ones, most places hold no chunk."""
    r, n, H_k, H_v = random.Random(62), 170, 4, 4
    bounds = [3]
    for s in range(n):
        bounds.append(bounds[-1] + (0 if s % 5 == 2 else r.randrange(1, 40) if s % 7 else r.randrange(60, 140)))
    T = bounds[-1] + 2
    assert (T // 64 + n) * H_k > 3 * 148 and max(b - a for a, b in zip(bounds, bounds[1:])) > 128
    x = _inputs(T, H_k, H_v, 63, n)
    d = x if token_major else {k: x[k].transpose(0, 1).contiguous() for k in (*NAMES, "dO")}
    got = _call(d, x, cu_seqlens=bounds, token_major=token_major)
    assert gdn.gdn_device_status() == gdn.GDN_OK
    rows = got[:5] if token_major else [t.transpose(0, 1) for t in got[:5]]
    for s, (a, b) in enumerate(zip(bounds, bounds[1:])):
        if a == b:
            assert torch.equal(got[5][s], x["dS"][s])  # no token: the gradient goes through
            continue
        part = {k: x[k][a:b] for k in (*NAMES, "dO")} | {"S": x["S"][s:s + 1], "dS": x["dS"][s:s + 1]}
        alone = _call(_dense(part, 1, b - a), part)
        assert all(torch.equal(p[a:b], q[0]) for p, q in zip(rows, alone)) and torch.equal(got[5][s], alone[5][0]), s
        if s in (0, n // 2, n - 1):
            ref, dS = _expected(part, [0, b - a])
            _check([t[a:b] for t in rows] + [got[5][s:s + 1]], ref, dS)
    for t in rows:
        assert not t[:bounds[0]].any() and not t[bounds[-1]:].any()
