"""DecoderChain with an 8-bit cache: a step's answer depends on its input alone, whatever the steps before it were given."""
import numpy as np
import pytest
import torch

from paper_2504_15465_amd import inputs
from paper_2504_15465_amd.models import run_ops
from gpu_util import bits_equal, ctx
from test_gpu_quant_chain import D, H, N_KV, N_Q, build

pytestmark = pytest.mark.gpu


def state(chain):
    return [t.clone().view(torch.uint8) for t in chain.kc + chain.vc] + [s.clone().view(torch.uint8) for s in chain.kv_scales]


@pytest.mark.parametrize("batch,pos", [(1, 64), (3, 200), (2, 33), (16, 127), (1, 1), (2, 0)])
@pytest.mark.parametrize("kw", [dict(kv8_block=32), dict(q4_group=64, kv8_block=32, kv8_e4m3=True), dict(q4_group=128, kv8_block=128), dict(kv8_block=16, splits=3)])
@pytest.mark.parametrize("before", ["large", "nan"])
def test_a_step_does_not_depend_on_the_steps_before(batch, pos, kw, before):
    fresh, params, *_ = build(batch, pos, **kw)
    mine = inputs.decoder_hidden(batch, H, seed=90)
    fresh.set_input(mine)
    run_ops(ctx(), fresh.ops())
    used = build(batch, pos, **kw)[0]
    ops = used.ops()
    # along the weights of a key's and a value's element, which become 14 where the prompt's are of N(0, 1): the scales grow
    w = inputs.bits_to_torch(np.ascontiguousarray(params[0]["w_qkv"])).float().numpy()
    other = np.repeat((w[:, N_Q * D + 5] + w[:, (N_Q + N_KV) * D + 9])[None], batch, 0)
    if before == "nan":
        other[0, 5] = np.nan
    used.set_input(other)
    run_ops(ctx(), ops)
    if before == "large" and pos % kw["kv8_block"]:
        assert bool((used.kv_scales[0][:, :, -1] > 2 * fresh.kv_scales[0][:, :, -1]).any())
    used.set_input(mine)
    run_ops(ctx(), ops)
    for a, b in zip((used.out, used.logits, used.stats), (fresh.out, fresh.logits, fresh.stats)):
        assert bits_equal(a, b) and bool(torch.isfinite(a).all())
    for a, b in zip(state(used), state(fresh)):
        assert torch.equal(a, b)
