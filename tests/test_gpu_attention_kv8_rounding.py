"""ATTN_DEC8 with a bf16 output: what reaches the output's one rounding is right to far more bits than that keeps."""
import pytest
import torch

from paper_2504_15465_amd import binding as B
from gpu_util import nan_like
from test_gpu_quant_step import BF, E4M3, F32, U, half_step, launch, make_cache, rnd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("keys", [1, 3, 40])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [4, 7, 16])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("splits", [1, 2])
def test_weighted_values_are_not_cut_off(keys, d, G, e4m3, splits):
    """Queries of zeros weigh every key alike: the output is the mean of the values."""
    batch, n_kv, block = 4, 8, 16
    codes, scales = make_cache(batch, keys, n_kv, d, block, e4m3, 70)
    codes[1].view(torch.uint8).bitwise_and_(0x7F)                    # no values below zero, which cancel
    scales[1] = (1.0 + 2.0 ** -8 + 2.0 ** -15 - 2.0 ** -23) * torch.exp2(torch.randint(-3, 4, scales[1].shape, generator=rnd(71)).float())
    o = nan_like((batch, n_kv * G * d), BF)
    ws = nan_like((B.attn_workspace_floats(batch, n_kv * G, d, splits),), F32) if splits > 1 else None
    q = torch.zeros(batch, n_kv * G * d, dtype=BF, device="cuda")
    ops = [B.attn_dec8_op(q, codes[0].cuda(), codes[1].cuda(), scales.cuda(), o, batch, n_kv * G, n_kv, d, keys, keys, block, 1.0, splits=splits, workspace=ws)]
    if splits > 1:
        ops.append(B.attn_merge_op(ws, o, batch, n_kv * G, n_kv, d, splits))
    launch(*ops)
    v = codes[1].float().double() * scales[1].double().repeat_interleave(block, 1)[:, :keys, :, None]       # b, key, h, d
    want = v.mean(1)[:, :, None].expand(batch, n_kv, G, d).reshape(batch, -1)
    # a weighted scale is two bf16 numbers, the second the first's error, rounded: 2^-9 of 2^-9; the rest is fp32
    inner = (2.0 ** -18 + (2 * keys + 16) * U) * want
    off = (o.cpu().double() - want).abs()
    assert bool((off <= half_step(BF) * (want + inner) + inner).all()), "off by %g of the value" % (off / want.clamp(min=1e-30)).max()
