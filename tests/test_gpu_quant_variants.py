"""Kernel variants of the quantised decode step that only larger launches choose, and roundings that sums of many terms hide,
against plain definitions in 64 bits.  U = 2^-24, the rounding of fp32 arithmetic."""
import math

import pytest
import torch

from paper_2504_15465_amd import binding as B
from paper_2504_15465_amd import quant
from gpu_util import bits_equal, ctx, nan_like
from test_gpu_quant_step import BF, E4M3, F32, F64, U, append_plain, attn_case, check, half_step, launch, make_cache, rnd

pytestmark = pytest.mark.gpu


# ---- products with weights in 4 bits: column blocks of a workgroup ----------------------------------

def column_blocks(op, n, glu):
    """16-column blocks of a workgroup as the plan has them; x of the grid is blocks of rows, y of columns."""
    (_, gy, _), _ = B.lithos_op_grid(ctx(), op)
    nb = 1
    while -(-n // (16 * nb // (2 if glu else 1) or 8)) != gy:
        nb *= 2
        assert nb <= 16, "grid of %d column blocks for %d columns" % (gy, n)
    return nb


def wide_case(m, n, k, group, a_dt, glu, seed=0):
    """As many columns as it takes, on the GPU, also the definition."""
    g = torch.Generator(device="cuda").manual_seed(seed + 31 * m + n + 7 * k)
    rows = 2 * n if glu else n
    q = torch.randint(0, 16, (rows, k), dtype=torch.uint8, generator=g, device="cuda")
    groups = -(-k // group)
    s = (0.01 * torch.randn(rows, groups, generator=g, device="cuda")).to(BF)
    z = (8 + 3 * torch.randn(rows, groups, generator=g, device="cuda")).to(BF)
    a = torch.randn(m, k, generator=g, device="cuda").to(a_dt)
    c = nan_like((m, n + 3), F32)
    op = B.gemm_q4_op(a, quant.pack_q4(q), quant.pack_q4_groups(s), c, m, n, k, group, zeros=quant.pack_q4_groups(z), glu=glu, ldc=n + 3)
    wide = lambda t: t.double().repeat_interleave(group, 1)[:, :k]  # noqa: E731
    x = a.double()
    y = (x @ ((q.double() - wide(z)) * wide(s)).t().contiguous()).cpu()
    # |rounding| <= (number of additions and products behind one value) u * sum of magnitudes
    tol = (k + 3 * groups + 16) * U * (x.abs() @ ((q.double() + wide(z).abs()) * wide(s).abs()).t().contiguous()).cpu()
    if glu:
        gt, up, tg, tu = y[:, :n], y[:, n:], tol[:, :n], tol[:, n:]
        y = gt * torch.sigmoid(gt) * up
        tol = 1.1 * tg * up.abs() + (gt.abs() + 1.1 * tg) * tu + 16 * U * y.abs()      # |silu'| < 1.1
    return op, c, y, tol + 4 * U * y.abs()


# rows, type of A, tiles of 16 columns for 1, 2, 4 and 8 blocks (none where as many are never chosen); last tiles are partial
SHAPES = [(1, F32, (75, 399, 999, None)), (3, F32, (75, 399, 999, None)), (7, F32, (75, 399, 999, 1901)), (13, F32, (75, 399, 999, 1901)),
          (27, F32, (75, 199, 499, 999)), (3, BF, (75, 399, 999, None)), (9, BF, (75, 399, 999, 1901)), (27, BF, (75, 399, 999, None))]
CASES = [(m, dt, t, 1 << i) for m, dt, tiles in SHAPES for i, t in enumerate(tiles) if t is not None]


@pytest.mark.parametrize("m,a_dt,tiles,blocks", CASES)
@pytest.mark.parametrize("group,k", [(32, 264), (64, 264), (128, 264), (32, 4104), (128, 4104)])
def test_q4_column_blocks(m, a_dt, tiles, blocks, group, k):
    n = 16 * tiles - 11
    op, c, y, tol = wide_case(m, n, k, group, a_dt, False)
    assert column_blocks(op, n, False) == blocks
    launch(op)
    check(c, y, tol)


@pytest.mark.parametrize("m,a_dt,tiles,blocks", [c for c in CASES if c[3] > 1])
@pytest.mark.parametrize("group,k", [(32, 264), (64, 264), (128, 264), (64, 4104)])
def test_q4_column_blocks_gated(m, a_dt, tiles, blocks, group, k):
    n = tiles // 2 * 16                                              # 499 and 950 tiles of gates: no multiples of 2 and 4
    op, c, y, tol = wide_case(m, n, k, group, a_dt, True)
    assert column_blocks(op, n, True) == blocks
    launch(op)
    check(c, y, tol)


@pytest.mark.parametrize("m", [257, 1000])
@pytest.mark.parametrize("a_dt", [F32, BF])
@pytest.mark.parametrize("n,glu", [(301, False), (304, True), (4111, False)])
def test_q4_rows_of_a_prompt(m, a_dt, n, glu):
    op, c, y, tol = wide_case(m, n, 712, 64, a_dt, glu)
    launch(op)
    check(c, y, tol)


@pytest.mark.parametrize("m,tiles,blocks", [c[:1] + c[2:] for c in CASES if c[1] == F32])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_q4_every_bit_of_fp32_rows_counts(m, tiles, blocks, group):
    """One live k per row, 24 significant bits: the lowest plane is 2^-16 of the value and more."""
    n, k = 16 * tiles - 11, 264
    g = torch.Generator(device="cuda").manual_seed(m + tiles)
    q = torch.randint(0, 16, (n, k), dtype=torch.uint8, generator=g, device="cuda")
    s = torch.ones(n, -(-k // group), device="cuda")
    a = torch.zeros(m, k, device="cuda")
    at = (37 * torch.arange(m, device="cuda") + 5) % k
    a[torch.arange(m, device="cuda"), at] = 2.0 - 2.0 ** -23 - torch.randint(0, 128, (m,), generator=g, device="cuda") * 2.0 ** -22
    c = nan_like((m, n), F32)
    op = B.gemm_q4_op(a, quant.pack_q4(q), quant.pack_q4_groups(s), c, m, n, k, group)
    assert column_blocks(op, n, False) == blocks
    launch(op)
    live, v = q[:, at].t().double(), a.amax(1, keepdim=True).double()
    # two sums of three products, planes and groups joined, two fused steps: eight additions at most that are not of zeros, each
    # off by a unit of the last place of v (q + 8)
    check(c, (v * (live - 8)).cpu(), (16 * U * v * (live + 8)).cpu())


# ---- the cache: four wavefronts, several heads a key/value head ------------------------------------------

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [4, 7, 16])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("q_dt,o_dt", [(F32, F32), (F32, BF), (BF, F32), (BF, BF)])
def test_attention_of_many_blocks(d, G, e4m3, q_dt, o_dt):
    ops, o, want, tol = attn_case(32, 8, G, d, 333, 32, e4m3, q_dt, o_dt, lens=[(97 * b) % 334 for b in range(32)])
    assert B.lithos_op_grid(ctx(), ops[0])[0][0] * 32 >= 256         # four wavefronts from as many on
    launch(*ops)
    check(o, want, tol)


@pytest.mark.parametrize("d,G,e4m3,dt", [(64, 7, False, BF), (64, 16, True, F32), (128, 5, True, BF), (128, 16, False, F32)])
def test_attention_of_many_blocks_split(d, G, e4m3, dt):
    ops, o, want, tol = attn_case(8, 8, G, d, 1500, 48, e4m3, dt, dt, lens=[1500, 0, 33, 1499, 700, 1, 1024, 64], splits=4)
    launch(*ops)
    whole = o.clone()
    check(o, want, tol)
    o.fill_(float("nan"))
    launch(*ops, atom_blocks=37)
    assert bits_equal(o, whole)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("block,tokens,pos", [(128, 300, 0), (128, 300, 77), (256, 613, 0), (256, 613, 250), (1024, 2100, 0), (1024, 1301, 1000), (1024, 700, 5)])
def test_append_of_blocks_longer_than_the_registers(d, dt, e4m3, block, tokens, pos):
    batch, n_kv, cap = 2, 2, pos + tokens + 3
    codes, scales = make_cache(batch, cap, n_kv, d, block, e4m3, 60)
    x = (torch.randn(2, batch, tokens, n_kv, d, generator=rnd(61)) * torch.tensor([3.0, 0.2])[None, None, None, :, None]).to(dt)     # one head's scales grow, the other's stay
    kc, vc, sc, xd = codes[0].cuda(), codes[1].cuda(), scales.cuda(), x.cuda()
    launch(B.kv8_append_op(xd[0], xd[1], kc, vc, sc, batch, tokens, n_kv, d, pos, cap, block))
    append_plain(x.float(), codes, scales, [pos] * batch, block, e4m3)
    assert torch.equal(sc.cpu(), scales)
    for got, want in ((kc, codes[0]), (vc, codes[1])):
        assert torch.equal(got.cpu().view(torch.uint8), want.view(torch.uint8))
