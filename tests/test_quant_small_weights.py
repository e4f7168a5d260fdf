"""Weights at the lower end of their type: quantised to finite scales and zero points, on the CPU."""
import pytest
import torch

from paper_2504_15465_amd import quant


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("symmetric", [False, True])
@pytest.mark.parametrize("size", [2.0 ** -126, 2.0 ** -130, 2.0 ** -133, 2.0 ** -136, 2.0 ** -140, 2.0 ** -149])
def test_small_weights_come_back_as_small_numbers(group, symmetric, size):
    n, k = 6, 256
    w = torch.randn(n, k, generator=torch.Generator().manual_seed(1)) * size
    w[1], w[2], w[3] = size, -size, 0.0                              # equal weights
    w[4] = w[4].abs() + 4 * size                                     # away from zero
    w[5, ::2] = 0.0
    q, s, z = quant.quantize_q4(w, group, symmetric)
    assert bool(torch.isfinite(s).all()) and (z is None or bool(torch.isfinite(z).all()))
    wide = lambda t: t.double().repeat_interleave(group, 1)  # noqa: E731
    back = (q.double() - (8.0 if symmetric else wide(z))) * wide(s)
    # the scale is bf16, whose steps are 2^-133 down there: half a code's step, and 15 codes times half a step of the scale
    top = w.double().abs().amax(1, keepdim=True)
    assert bool(((back - w.double()).abs() <= 0.6 * wide(s) + top * 2.0 ** -3 + 16 * 2.0 ** -134).all())
