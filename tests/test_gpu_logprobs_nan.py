"""LOGPROBS of rows with a NaN or an infinity above: every statistic says so, also where a logit of -infinity stands beside it."""
import math

import pytest
import torch

from test_gpu_quant_step import BF, F32, check_lp, logits, lp_run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows_more,vocab,splits", [(0, 3000, 1), (0, 3000, 3), (300, 6001, 1), (0, 40001, 1), (0, 70001, 1), (0, 70001, 5)])
@pytest.mark.parametrize("dt", [F32, BF])
def test_rows_that_hold_no_numbers(rows_more, vocab, splits, dt):
    top = 5
    x = logits(8 + rows_more, vocab, dt)
    x[1, vocab - 3], x[1, 4] = math.nan, -math.inf                   # the given token is forbidden
    x[2, 11], x[2, 4] = math.inf, -math.inf
    x[3] = math.nan                                                  # nothing else
    x[4] = -math.inf                                                 # fewer numbers than are asked for
    x[4, 70], x[4, 71] = math.nan, 1.0
    x[5] = -math.inf
    x[5, 9] = math.inf
    x[6] = -math.inf                                                 # nothing is allowed, but everything is a number
    tokens = [4] * x.shape[0]
    stats, ids = lp_run(x, vocab, tokens, top, splits=splits)
    assert bool(torch.isnan(stats[1:6, :3 + top]).all())
    assert bool(((ids[:, :top] >= 0) & (ids[:, :top] < vocab)).all())
    good = [0, 6, 7]
    check_lp(stats[good], ids[good], x[good], [4] * 3, top, 1.0)
    stats, _ = lp_run(x, vocab, [-1] * x.shape[0], top, splits=splits)      # no given token: 0 whatever the row holds
    assert bool((stats[:, 0] == 0).all()) and bool(torch.isnan(stats[1:6, 1:3 + top]).all())
