"""Registers and spills of the decoding, backward and norm kernels, from the compiler's report that the build keeps."""
import re

from paper_2606_06034_b200 import build as gdn_build


def test_spills_are_no_more_than_were_measured():
    """chunk_grads_kernel holds 32 values of dQ and dK and 32 of a state in 96 registers (17 warps of one CTA per SM): 140 bytes; its neighbours 36 at most. The
    step and the norms' rows of up to 4096 features: none that matters (40 bytes where a width is no multiple of 8)."""
    gdn_build.build()
    res = gdn_build.kernel_resources("chunk_backward.cu")
    most = {"chunk_system_kernel": 0, "chunk_states_kernel": 0, "chunk_state_grads_kernel": 36, "chunk_grads_kernel": 140}
    for kernel, spill in most.items():
        hits = [v for k, v in res.items() if kernel in k]
        assert len(hits) == 1 and hits[0]["spill_stores"] <= spill, (kernel, hits)
        assert hits[0]["registers"] <= 96
    assert all(v["spill_stores"] == 0 for v in gdn_build.kernel_resources("recurrent_step.cu").values())
    for name, v in gdn_build.kernel_resources("row_norm.cu").items():
        m = re.search(r"norm_(?:forward|backward)_kernelI\w+Li(\d)ELi(\d+)ELb(\d)", name)
        if m and int(m[1]) * int(m[2]) * 8 <= 4096:
            assert v["spill_stores"] <= (4 if m[3] == "1" else 40), (name, v)
