"""Flags that KV8_APPEND, ATTN_DEC8 and LOGPROBS do not know are refused, not passed over; on the CPU."""
import pytest

from paper_2504_15465_amd import binding as B
from test_quant_step_refusals import A16, append, dec8, grad, lp, plan

FLAGS = [getattr(B, "F_" + n) for n in ("TRANS_A", "TRANS_B", "BIAS", "GELU", "RESIDUAL", "OUT_F32", "IN_F32", "SPLIT_A", "OUT_SPLIT", "NORM_LN", "NORM_RMS", "GLU", "E4M3")] + [1 << 13, 1 << 31]


def dec8_with(flags):
    op = dec8()
    op.flags = flags
    return op


@pytest.mark.parametrize("flag", FLAGS)
@pytest.mark.parametrize("make,known,name", [
    (lambda f: append(flags=f), B.F_IN_F32 | B.F_E4M3, b"kv8_append"),
    (dec8_with, B.F_IN_F32 | B.F_OUT_F32 | B.F_E4M3, b"attn_dec8"),
    (lambda f: lp(flags=f), B.F_IN_F32, b"logprobs"),
    (lambda f: lp(B.OP_LOGPROBS_MERGE, splits=2, flags=f), B.F_IN_F32, b"logprobs"),
    (lambda f: grad(flags=f), B.F_IN_F32 | B.F_OUT_F32, b"logprobs")])
def test_flags(make, known, name, flag):
    rc, _ = plan(make(flag))
    if flag & known:
        assert rc == B.OK
    else:
        assert rc == B.EINVAL and name in B.lib().lithos_last_error()
