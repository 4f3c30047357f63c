"""The decoding step at its edges: two errors at once, outputs that lie on inputs, slots far apart in a large batch. Formula and tolerances as in
test_gpu_step.py."""
import pytest
import torch

from paper_2606_06034_b200 import binding as gdn
from test_gpu_step import _inputs

pytestmark = pytest.mark.gpu


def test_an_unusable_slot_does_not_hide_a_wait_that_ran_out():
    """Both are reported, the wait first."""
    Q, K, V, beta, g, S = _inputs(2, 1, 1, 2, 128, 128, torch.bfloat16, 5)
    assert gdn.gdn_selftest_bounded_wait() == gdn.GDN_OK
    gdn.gated_delta_step(Q, K, V, beta, g, S, torch.tensor([0, 2], dtype=torch.int32, device="cuda"))
    assert gdn.gdn_device_status() == gdn.GDN_ERR_TIMEOUT
    assert gdn.gdn_device_status() == gdn.GDN_ERR_INVALID_ARG
    assert gdn.gdn_device_status() == gdn.GDN_OK
