"""The decoding step at its edges: two errors at once, outputs that lie on inputs, slots far apart in a large batch. Formula and tolerances as in
test_gpu_step.py."""
import pytest
import torch

from paper_2606_06034_b200 import binding as gdn
from test_gpu_step import TOL, _expected, _inputs, _near

pytestmark = pytest.mark.gpu


def test_an_unusable_slot_does_not_hide_a_wait_that_ran_out():
    """Both are reported, the wait first."""
    Q, K, V, beta, g, S = _inputs(2, 1, 1, 2, 128, 128, torch.bfloat16, 5)
    assert gdn.gdn_selftest_bounded_wait() == gdn.GDN_OK
    gdn.gated_delta_step(Q, K, V, beta, g, S, torch.tensor([0, 2], dtype=torch.int32, device="cuda"))
    assert gdn.gdn_device_status() == gdn.GDN_ERR_TIMEOUT
    assert gdn.gdn_device_status() == gdn.GDN_ERR_INVALID_ARG
    assert gdn.gdn_device_status() == gdn.GDN_OK

def test_outputs_that_lie_on_inputs():
    """Slices of a head store outputs while others still read Q and K: refused. V's rows are read by the threads that store O's: allowed."""
    Q, K, V, beta, g, S = _inputs(3, 2, 2, 2, 128, 128, torch.bfloat16, 6)
    for out in (Q, K):
        with pytest.raises(gdn.GdnError):
            gdn.gated_delta_step(Q, K, V, beta, g, S, out=out)
    both = torch.cat([V.flatten(), V.flatten()])
    with pytest.raises(gdn.GdnError):  # O a row behind V
        gdn.gated_delta_step(Q, K, both[:V.numel()].view_as(V), beta, g, S, out=both[128:128 + V.numel()].view_as(V))
    ref = _expected(Q, K, V, beta, g, S, [(b, b) for b in range(3)])
    beside = gdn.gated_delta_step(Q, K, both[:V.numel()].view_as(V), beta, g, S.clone(), out=both[V.numel():].view_as(V))  # side by side
    _near(beside, ref[0], TOL[torch.bfloat16])
    assert gdn.gated_delta_step(Q, K, V, beta, g, S, out=V) is V
    _near(V, ref[0], TOL[torch.bfloat16])
    _near(S, ref[1], TOL[torch.float32])


def test_a_twin_more_than_one_cta_of_rows_away():
    B, n = 700, 800
    Q, K, V, beta, g, S = _inputs(B, 1, 1, 1, 128, 128, torch.bfloat16, 7, n_slots=n)
    slots = torch.randperm(n, generator=torch.Generator().manual_seed(8))[:B].int()
    slots[650], slots[699], slots[300] = slots[3], slots[400], -1
    before = S.clone()
    ref = _expected(Q, K, V, beta, g, S, [(b, int(s)) for b, s in enumerate(slots) if b not in (650, 699, 300)])
    O = gdn.gated_delta_step(Q, K, V, beta, g, S, slots.cuda())
    assert gdn.gdn_device_status() == gdn.GDN_ERR_INVALID_ARG
    assert not O[650].any() and not O[699].any() and not O[300].any()
    _near(O, ref[0], TOL[torch.bfloat16])
    _near(S, ref[1], TOL[torch.float32])
    left = sorted(set(range(n)) - set(slots.tolist()))
    assert torch.equal(S[left], before[left])
