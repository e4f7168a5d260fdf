"""LOGPROBS' scale: what its arithmetic in powers of two cannot hold is refused, on the CPU."""
import pytest

from paper_2504_15465_amd import binding as B
from test_quant_step_refusals import grad, lp, plan

MOST = 2.0 ** 127                                                    # 2^127 log2(e) is below 2^128


@pytest.mark.parametrize("make", [lambda s: lp(scale=s), lambda s: lp(B.OP_LOGPROBS_MERGE, splits=3, scale=s), lambda s: grad(scale=s)])
@pytest.mark.parametrize("scale,taken", [(1e-30, True), (1e30, True), (MOST, True), (1.3 * MOST, True), (1.4 * MOST, False), (3.4e38, False)])
def test_scale(make, scale, taken):
    rc, _ = plan(make(scale))
    assert rc == (B.OK if taken else B.EINVAL)
    assert taken or b"logprobs" in B.lib().lithos_last_error()
