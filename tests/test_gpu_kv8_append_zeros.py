"""KV8_APPEND of zeros of both signs and of values too small for a code: the codes are those of the definition to the bit."""
import pytest
import torch

from paper_2504_15465_amd import binding as B
from test_gpu_quant_step import BF, F32, append_plain, launch, make_cache, rnd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("tokens,pos", [(1, 0), (1, 9), (40, 9), (40, 32)])
@pytest.mark.parametrize("peak", [4.0, 1e-20])
def test_zeros_and_small_values(e4m3, dt, d, tokens, pos, peak):
    batch, n_kv, block, cap = 2, 2, 32, pos + tokens
    codes, scales = make_cache(batch, cap, n_kv, d, block, e4m3, 80)
    codes.view(torch.uint8)[torch.rand(codes.shape, generator=rnd(81)) < 0.3] = 0x80 if e4m3 else 0          # held zeros below
    scales *= peak / 4.0                                             # earlier codes are rounded to a larger scale
    small = torch.tensor([0.0, -0.0, 1e-42, -1e-42, 1e-30, -1e-30, 1e-9, -1e-9]) * peak
    x = small[torch.randint(0, 8, (2, batch, tokens, n_kv, d), generator=rnd(82))]
    x[..., 0, :, 5] = peak                                           # of a block's first token at least
    x[:, :, ::7, :, 5] = -peak
    x = x.to(dt)
    kc, vc, sc, xd = codes[0].cuda(), codes[1].cuda(), scales.cuda(), x.cuda()
    launch(B.kv8_append_op(xd[0], xd[1], kc, vc, sc, batch, tokens, n_kv, d, pos, cap, block))
    append_plain(x.float(), codes, scales, [pos] * batch, block, e4m3)
    assert torch.equal(sc.cpu(), scales)
    for got, want in ((kc, codes[0]), (vc, codes[1])):
        assert torch.equal(got.cpu().view(torch.uint8), want.view(torch.uint8))
