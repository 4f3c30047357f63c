"""The decoding step and the norms refuse outputs that lie on what other threads still read. No GPU needed: every call here is refused before the device is asked for."""
import pytest

from paper_2606_06034_b200 import binding as gdn
from paper_2606_06034_b200 import build as gdn_build

MB = 1 << 20
# addresses that nothing reads, 16 MB apart
AT = {n: (i + 1) * 16 * MB for i, n in enumerate(("Q", "K", "V", "beta", "g", "S", "slots", "O"))}
B, H_k, H_v, T, D = 2, 2, 4, 3, 128
SIZE = {"Q": B * T * H_k * D * 2, "K": B * T * H_k * D * 2, "V": B * T * H_v * D * 2, "beta": B * T * H_v * 4, "g": B * T * H_v * 4, "S": 5 * H_v * D * D * 4, "slots": B * 4,
        "O": B * T * H_v * D * 2}


@pytest.fixture(scope="module")
def lib():
    gdn_build.build()
    return gdn.load_library()


def _step(lib, **kw):
    a = {**AT, **kw}
    return lib.gdn_recurrent_step(a["Q"], a["K"], a["V"], a["beta"], a["g"], B, H_k, H_v, T, D, D, 1.0, gdn.GDN_DTYPE_BF16, a["S"], gdn.GDN_DTYPE_FP32, a["slots"], 5, a["O"],
                                  gdn.GDN_FLAG_LAYOUT_BTHD, None)


@pytest.mark.parametrize("out,other", [("O", "S")] + [(out, other) for out in ("O", "S") for other in ("Q", "K", "V", "beta", "g", "slots")])
def test_one_byte_in_common_is_refused(lib, out, other):
    up = (SIZE[other] + 15) // 16 * 16  # the first 16-byte boundary behind the other one
    for at in (AT[other] + up - 16, AT[other] - SIZE[out] + 16):
        assert _step(lib, **{out: at}) == gdn.GDN_ERR_INVALID_ARG


def test_v_that_is_q_too_may_not_be_written_over(lib):
    assert _step(lib, O=AT["V"], Q=AT["V"]) == gdn.GDN_ERR_INVALID_ARG


ROWS, W = 64, 256
X = {n: (i + 1) * 16 * MB for i, n in enumerate(("dy", "x", "weight", "bias", "gate", "out", "dgate", "dweight", "dbias", "ws"))}
BYTES = ROWS * W * 2


def _norm(lib, backward, **kw):
    a = {**X, **kw}
    if backward:
        return lib.gdn_layer_norm_backward(a["dy"], a["x"], a["weight"], a["bias"], a["gate"], ROWS, W, 1e-5, gdn.GDN_DTYPE_BF16, gdn.GDN_DTYPE_FP32, a["out"], a["dweight"], a["dbias"],
                                           a["dgate"], a["ws"], 1 << 30, 0, None)
    return lib.gdn_layer_norm(a["x"], a["weight"], a["bias"], a["gate"], ROWS, W, 1e-5, gdn.GDN_DTYPE_BF16, gdn.GDN_DTYPE_FP32, a["out"], 0, None)


@pytest.mark.parametrize("backward,out,other", [(False, "out", n) for n in ("x", "gate")] + [(True, out, n) for out in ("out", "dgate") for n in ("dy", "x", "gate")])
def test_rows_that_are_moved_are_refused(lib, backward, out, other):
    for by in (16, W * 2, BYTES - 16, -16, 16 - BYTES):
        assert _norm(lib, backward, **{out: X[other] + by}) == gdn.GDN_ERR_INVALID_ARG


@pytest.mark.parametrize("backward,out", [(False, "out"), (True, "out"), (True, "dgate")])
def test_rows_on_parameters_or_on_each_other_are_refused(lib, backward, out):
    for other in ("weight", "bias"):
        for by in (0, W * 4 - 16, 16 - BYTES):
            assert _norm(lib, backward, **{out: X[other] + by}) == gdn.GDN_ERR_INVALID_ARG
    if backward:
        assert _norm(lib, True, out=X["dgate"] + 32) == gdn.GDN_ERR_INVALID_ARG
        assert _norm(lib, True, out=X["dgate"]) == gdn.GDN_ERR_INVALID_ARG
