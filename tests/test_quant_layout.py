"""Weights in 4 bits: quantisation error and layout, on the CPU."""
import pytest
import torch

from paper_2504_15465_amd import quant


@pytest.mark.parametrize("n,k", [(1, 8), (16, 128), (33, 264), (5, 1000)])
def test_packing_is_a_bijection_of_the_codes(n, k):
    q = torch.randint(0, 16, (n, k), dtype=torch.uint8, generator=torch.Generator().manual_seed(n))
    packed = quant.pack_q4(q)
    assert packed.shape == (-(-n // 16), -(-k // 128), 4, 16, 16) and packed.is_contiguous()
    assert torch.equal(quant.unpack_q4(packed, n, k), q)


def test_a_code_lies_where_the_header_says():
    n, k = 40, 400
    q = torch.randint(0, 16, (n, k), dtype=torch.uint8, generator=torch.Generator().manual_seed(3))
    packed = quant.pack_q4(q)
    for row, kk in ((0, 0), (17, 37), (39, 399), (8, 260)):
        c, r = kk // 128, kk % 128
        t, p, j = r // 32, r % 32 // 8, r % 8
        byte = int(packed[row // 16, c, p, row % 16, 4 * t + j % 4])
        assert (byte >> (4 * (j // 4))) & 15 == int(q[row, kk])
    s = torch.randn(n, 7, generator=torch.Generator().manual_seed(4)).bfloat16()
    assert quant.pack_q4_groups(s)[2, 5, 7] == s[39, 5]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("symmetric", [False, True])
def test_weights_come_back_within_half_a_step(group, symmetric):
    n, k = 24, 456
    w = torch.randn(n, k, generator=torch.Generator().manual_seed(5)) * 0.02 + 0.003
    w[3] = 0.0
    w[4] = 0.7
    q, s, z = quant.quantize_q4(w, group, symmetric)
    assert q.dtype == torch.uint8 and int(q.max()) <= 15 and (z is None) == symmetric
    wide = lambda t: t.double().repeat_interleave(group, 1)[:, :k]  # noqa: E731
    back = (q.double() - (8.0 if symmetric else wide(z))) * wide(s)
    # half a step inside the range; at its ends the scale (2^-8) and the zero point (2^-8 of at most 16) as bf16 rounds
    # them cut off up to 15 * 2^-8 + 16 * 2^-8 of a step more.  Groups of equal weights have a zero point of -1, 1 or 0.
    step = wide(s).abs()
    assert ((back - w.double()).abs() <= step * (0.5 + 31 * 2.0 ** -8) + 1e-12)[[i for i in range(n) if i != 4]].all()
    assert ((back[4] - 0.7).abs() <= 0.7 * 2.0 ** -7 + (step[4] * 0.5 if symmetric else 0)).all()
