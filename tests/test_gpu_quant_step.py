"""The quantised decode step's operators through the C ABI against plain definitions in 64 bits.

Tolerances count roundings: u = 2^-24 for fp32 arithmetic, half a step of the output type (2^-8 relative for bf16)."""
import math

import pytest
import torch

from paper_2504_15465_amd import binding as B
from paper_2504_15465_amd import quant
from gpu_util import bits_equal, counters, ctx, nan_like

pytestmark = pytest.mark.gpu

U, BF, F32, F64 = 2.0 ** -24, torch.bfloat16, torch.float32, torch.float64
E4M3 = torch.float8_e4m3fn


def rnd(seed):
    return torch.Generator().manual_seed(seed)


def launch(*ops, atom_blocks=0, part=None):
    """The operators in order on one queue; with atoms, every block of the first exactly once."""
    torch.cuda.synchronize()
    grid, _ = B.lithos_op_grid(ctx(), ops[0])
    n = grid[0] * grid[1] * grid[2]
    for i, op in enumerate(ops):
        if i == 0 and atom_blocks:
            cnt = counters(n)
            torch.cuda.synchronize()
            B.lithos_debug_block_counters(ctx(), cnt)
            try:
                B.lithos_launch_atomized(ctx(), op, (0, 0, 0), atom_blocks, part, None)
                B.lithos_partition_sync(ctx(), part)
            finally:
                B.lithos_debug_block_counters(ctx(), None)
            assert cnt.cpu().tolist() == [1] * n
        else:
            B.lithos_launch_atomized(ctx(), op, (0, 0, 0), 0, part, None)
    B.lithos_partition_sync(ctx(), part)


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


# ---- products with weights in 4 bits ------------------------------------------------------

def q4_case(m, n, k, group, zeros, a_dt, c_dt, glu=False, epi=(), lda_pad=0, ldc_pad=0, ldr_pad=0, seed=0):
    g = rnd(seed + 31 * m + n + 7 * k)
    rows = 2 * n if glu else n
    q = torch.randint(0, 16, (rows, k), dtype=torch.uint8, generator=g)
    groups = -(-k // group)
    s = (0.01 * torch.randn(rows, groups, generator=g)).to(BF)
    z = (8 + 3 * torch.randn(rows, groups, generator=g)).to(BF) if zeros else None
    a = torch.randn(m, k + lda_pad, generator=g).to(a_dt)
    bias = torch.randn(n, generator=g) if "bias" in epi else None
    res = torch.randn(m, n + ldr_pad, generator=g) if "residual" in epi else None
    wide = lambda t: t.double().repeat_interleave(group, 1)[:, :k]  # noqa: E731
    qz = q.double() - (wide(z) if zeros else 8.0)
    x = a[:, :k].double()
    y = x @ (qz * wide(s)).t()
    # |rounding| <= (number of additions and products behind one value) u * sum of magnitudes
    mag = x.abs() @ ((q.double() + (wide(z).abs() if zeros else 8.0)) * wide(s).abs()).t()
    tol = (k + 3 * groups + 16) * U * mag
    if glu:
        gt, up, tg, tu = y[:, :n], y[:, n:], tol[:, :n], tol[:, n:]
        y = gt * torch.sigmoid(gt) * up
        tol = 1.1 * tg * up.abs() + (gt.abs() + 1.1 * tg) * tu + 16 * U * y.abs()      # |silu'| < 1.1
    if bias is not None:
        y = y + bias.double()
    if "gelu" in epi:
        y = y * torch.special.ndtr(y)
        tol = 1.13 * tol + 64 * U * (y.abs() + 1)                                          # |gelu'| < 1.13
    if res is not None:
        y = y + res[:, :n].double()
    tol = tol + 4 * U * y.abs() + (half_step(c_dt) * (y.abs() + tol) if c_dt == BF else 0)
    c = nan_like((m, n + ldc_pad), c_dt)
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    pack = lambda t: None if t is None else quant.pack_q4_groups(t).cuda()  # noqa: E731
    op = B.gemm_q4_op(dev(a), quant.pack_q4(q).cuda(), pack(s), c, m, n, k, group, zeros=pack(z), bias=dev(bias), gelu="gelu" in epi,
                      residual=dev(res), glu=glu, lda=k + lda_pad, ldc=n + ldc_pad, ldr=n + ldr_pad)
    return op, c, y, tol


def check(c, y, tol):
    got = c[:, :y.shape[1]].double().cpu()
    off = (got - y).abs()
    assert bool((off <= tol).all()), "off by %g, %g allowed" % (off.max(), tol[off > tol].min())
    assert bool(torch.isnan(c[:, y.shape[1]:]).all()), "columns beyond the matrix were written"


@pytest.mark.parametrize("m", [1, 2, 4, 5, 8, 9, 16, 17, 31, 32, 33, 70])
@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True)])
@pytest.mark.parametrize("a_dt", [F32, BF])
def test_q4_rows(m, group, zeros, a_dt):
    op, c, y, tol = q4_case(m, 100, 1160, group, zeros, a_dt, F32, lda_pad=8, ldc_pad=3)
    launch(op)
    check(c, y, tol)


@pytest.mark.parametrize("n,k", [(1, 8), (15, 64), (16, 128), (17, 136), (33, 1032), (300, 2048), (1000, 4096), (64, 14336)])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_q4_sizes(n, k, group):
    op, c, y, tol = q4_case(3, n, k, group, True, F32, F32)
    launch(op)
    check(c, y, tol)


@pytest.mark.parametrize("epi", [(), ("bias",), ("residual",), ("bias", "gelu"), ("gelu", "residual"), ("bias", "gelu", "residual")])
@pytest.mark.parametrize("c_dt", [F32, BF])
@pytest.mark.parametrize("m", [3, 20])
def test_q4_epilogues(epi, c_dt, m):
    op, c, y, tol = q4_case(m, 75, 520, 64, True, F32, c_dt, epi=epi, ldc_pad=5, ldr_pad=1)
    launch(op)
    check(c, y, tol)


@pytest.mark.parametrize("m", [1, 7, 16, 17, 40])
@pytest.mark.parametrize("n,k", [(16, 128), (208, 712)])
@pytest.mark.parametrize("a_dt,c_dt", [(F32, F32), (BF, BF)])
def test_q4_gated(m, n, k, a_dt, c_dt):
    op, c, y, tol = q4_case(m, n, k, 64, True, a_dt, c_dt, glu=True, ldc_pad=2)
    launch(op)
    check(c, y, tol)


@pytest.mark.parametrize("m", [1, 8, 20, 50])
def test_q4_in_atoms_is_the_whole_launch(m):
    op, c, y, tol = q4_case(m, 700, 1024, 128, True, F32, F32)
    launch(op, atom_blocks=3)
    atoms = c.clone()
    c.fill_(float("nan"))
    launch(op)
    check(c, y, tol)
    assert bits_equal(atoms, c)


def test_q4_codes_beyond_the_matrix_and_their_scales_do_not_matter():
    m, n, k, group = 5, 21, 200, 64
    op, c, y, tol = q4_case(m, n, k, group, True, F32, F32)
    codes, scales, zeros = (op._keep[0][i] for i in (1, 4, 5))
    launch(op)
    first = c.clone()
    q = quant.unpack_q4(codes.cpu(), 32, 256)
    q[n:], q[:, k:] = 15, 9
    codes.copy_(quant.pack_q4(q))
    for t in (scales, zeros):
        t[1, :, n - 16:] = float("nan")
    launch(op)
    assert bits_equal(first, c)


def test_q4_weights_quantised_and_packed_by_the_framework():
    m, n, k, group = 4, 192, 640, 64
    w = 0.02 * torch.randn(n, k, generator=rnd(1))
    a = torch.randn(m, k, generator=rnd(2))
    q, s, z = quant.quantize_q4(w, group)
    c = nan_like((m, n), F32)
    launch(B.gemm_q4_op(a.cuda(), quant.pack_q4(q).cuda(), quant.pack_q4_groups(s).cuda(), c, m, n, k, group, zeros=quant.pack_q4_groups(z).cuda()))
    y = a.double() @ w.double().t()
    # 15 steps over the range of 64 normal weights (about 4.7 sigma): an error of 0.09 sigma per weight
    assert float((c.double().cpu() - y).norm() / y.norm()) < 0.12


# ---- the cache of 8 bits ------------------------------------------------------------------

def nearest(y, e4m3):
    return y.clamp(-448, 448).to(E4M3) if e4m3 else y.round().clamp(-127, 127).to(torch.int8)


def append_plain(x, codes, scales, starts, block, e4m3):
    """fp32 steps of the definition, one block and head after another; x [2, b, t, h, d] fp32, the cache in place."""
    qmax = torch.tensor(448.0 if e4m3 else 127.0)
    cap = codes.shape[2]
    over = lambda a, s: torch.where(s > 0, a / s, torch.zeros(()))  # noqa: E731
    for i in range(2):
        for b, p0 in enumerate(starts):
            if p0 < 0:
                continue
            for j in range(p0 // block, (p0 + x.shape[2] - 1) // block + 1):
                lo, hi = max(p0, j * block), min(p0 + x.shape[2], (j + 1) * block, cap)
                if lo >= hi:
                    continue
                for h in range(x.shape[3]):
                    new = x[i, b, lo - p0:hi - p0, h]
                    s = new.abs().max() / qmax
                    if lo > j * block:
                        old = scales[i, b, j, h].clone()
                        if bool(s > old):
                            held = codes[i, b, j * block:lo, h]
                            held.copy_(nearest(over(held.float() * old, s), e4m3))
                        s = torch.maximum(s, old)
                    scales[i, b, j, h] = s
                    codes[i, b, lo:hi, h] = nearest(over(new, s), e4m3)


def make_cache(batch, cap, n_kv, d, block, e4m3, seed):
    g = rnd(seed)
    qmax = 448.0 if e4m3 else 127.0
    codes = nearest(torch.randn(2, batch, cap, n_kv, d, generator=g) * qmax / 4, e4m3)
    scales = (1.0 + 2.0 * torch.rand(2, batch, -(-cap // block), n_kv, generator=g)) / qmax
    return codes, scales


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("d,n_kv,block,tokens,pos", [(128, 2, 32, 1, 0), (128, 8, 32, 1, 37), (64, 3, 16, 1, 15), (128, 1, 64, 70, 60), (64, 2, 128, 300, 0),
                                                     (128, 3, 48, 97, 5), (64, 1, 32, 400, 31)])
def test_append(e4m3, dt, d, n_kv, block, tokens, pos):
    batch, cap, pad = 3, pos + tokens + 9, 16
    codes, scales = make_cache(batch, cap, n_kv, d, block, e4m3, 5)
    x = (torch.randn(batch * tokens, 2 * n_kv * d + pad, generator=rnd(6)) * torch.exp(torch.randn(batch * tokens, 1, generator=rnd(7)))).to(dt)
    x[0] = 0                                                        # a token of zeros, alone in its block: scale 0
    kc, vc, sc, xd = codes[0].cuda(), codes[1].cuda(), scales.cuda(), x.cuda()
    launch(B.kv8_append_op(xd[:, pad:pad + n_kv * d], xd[:, pad + n_kv * d:], kc, vc, sc, batch, tokens, n_kv, d, pos, cap, block, ldx=xd.stride(0)), atom_blocks=2)
    rows = x[:, pad:].float().reshape(batch, tokens, 2, n_kv, d).permute(2, 0, 1, 3, 4)
    append_plain(rows, codes, scales, [pos] * batch, block, e4m3)
    assert torch.equal(sc.cpu(), scales)
    for got, want in ((kc, codes[0]), (vc, codes[1])):
        assert torch.equal(got.cpu().view(torch.uint8), want.view(torch.uint8))


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("tokens", [1, 5, 60])
def test_append_at_positions_of_their_own(e4m3, tokens):
    batch, cap, n_kv, d, block = 6, 130, 2, 128, 32
    starts = [0, -1, 31, 129, 96, 70]                               # one takes no part, some reach beyond the cache
    codes, scales = make_cache(batch, cap, n_kv, d, block, e4m3, 8)
    x = 3 * torch.randn(2, batch, tokens, n_kv, d, generator=rnd(9))
    kc, vc, sc = codes[0].cuda(), codes[1].cuda(), scales.cuda()
    guard = sc.clone()
    xd = x.cuda()
    op = B.kv8_append_op(xd[0], xd[1], kc, vc, sc, batch, tokens, n_kv, d, 0, cap, block, positions=torch.tensor(starts, dtype=torch.int32).cuda())
    launch(op)
    append_plain(x, codes, scales, starts, block, e4m3)
    assert torch.equal(sc.cpu(), scales) and not torch.equal(sc, guard)
    assert torch.equal(kc.cpu().view(torch.uint8), codes[0].view(torch.uint8)) and torch.equal(vc.cpu().view(torch.uint8), codes[1].view(torch.uint8))
    launch(op)                                                      # the same tokens again: nothing changes
    assert torch.equal(sc.cpu(), scales) and torch.equal(kc.cpu().view(torch.uint8), codes[0].view(torch.uint8))


@pytest.mark.parametrize("e4m3", [False, True])
def test_append_token_by_token_is_close_to_the_whole_prompt(e4m3):
    batch, t, n_kv, d, block = 2, 50, 2, 64, 16
    x = torch.randn(2, batch, t, n_kv, d, generator=rnd(10)).cuda()
    kc, vc = (torch.zeros(batch, t, n_kv, d, dtype=E4M3 if e4m3 else torch.int8, device="cuda") for _ in range(2))
    sc = torch.full((2, batch, -(-t // block), n_kv), float("nan"), device="cuda")      # a fresh block's scale is not read
    for p in range(t):
        step = x[:, :, p].contiguous()
        launch(B.kv8_append_op(step[0], step[1], kc, vc, sc, batch, 1, n_kv, d, p, t, block))
    back = torch.stack([kc, vc]).float() * sc.repeat_interleave(block, 2)[:, :, :t, :, None]
    peak = torch.nn.functional.pad(x.abs(), (0, 0, 0, 0, 0, 64 - t)).reshape(2, batch, 4, block, n_kv, d).amax((3, 5)).repeat_interleave(block, 2)[:, :, :t, :, None]
    # a code is rounded at its own scale and once at each larger one, at most 15 times; the steps grow by what the scale
    # grows, so the sum is largest if all are the last: 16 half steps (int8: peak / 254, e4m3: 2^-4 of the value or 2^-10 * peak / 448)
    half = torch.maximum(x.abs() * 2.0 ** -4, peak * 2.0 ** -10 / 448) if e4m3 else peak / 254
    assert bool(((back - x).abs() <= 16.5 * half).all())
    assert float((back - x).norm() / x.norm()) < (0.06 if e4m3 else 0.02)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("e4m3", [False, True])
def test_a_block_with_a_value_that_is_no_number_reads_as_nan(bad, e4m3):
    cap, block, d = 64, 32, 64
    kc, vc = (torch.zeros(1, cap, 1, d, dtype=E4M3 if e4m3 else torch.int8, device="cuda") for _ in range(2))
    sc = torch.zeros(2, 1, 2, 1, device="cuda")
    x = torch.randn(40, d, generator=rnd(11)).cuda()
    y = x.clone()
    y[35, 7] = bad
    launch(B.kv8_append_op(y, x, kc, vc, sc, 1, 40, 1, d, 0, cap, block))
    s = sc.cpu()[:, 0, :, 0]
    assert bool(torch.isfinite(s[1]).all()) and bool(torch.isfinite(s[0, 0])) and not bool(torch.isfinite(s[0, 1]))
    back = kc.float()[0, 32:40, 0] * sc[0, 0, 1, 0]
    assert bool(torch.isnan(back).all())
    launch(B.kv8_append_op(x[:1], x[:1], kc, vc, sc, 1, 1, 1, d, 40, cap, block))       # and stays so
    assert not bool(torch.isfinite(sc[0, 0, 1, 0])) and bool(torch.isfinite(sc[1]).all())


# ---- decode attention ------------------------------------------------------------------------

def attn_case(batch, n_kv, G, d, keys, block, e4m3, q_dt, o_dt, lens=None, splits=1, ldq_pad=0, seed=20, qstd=1.0):
    cap = keys + 5
    codes, scales = make_cache(batch, cap, n_kv, d, block, e4m3, seed)
    q = (qstd * torch.randn(batch, n_kv * G * d + ldq_pad, generator=rnd(seed + 1))).to(q_dt)
    scale = 1 / math.sqrt(d)
    o = nan_like((batch, n_kv * G * d), o_dt)
    want, tol = torch.zeros(batch, n_kv, G, d, dtype=F64), torch.zeros(batch, n_kv, G, d, dtype=F64)
    blocks = torch.arange(cap) // block
    for b in range(batch):
        n = keys if lens is None else max(0, min(lens[b], keys))
        if n == 0:
            continue
        k, v = ((codes[i, b].float().double() * scales[i, b].double()[blocks][:, :, None])[:n].permute(1, 2, 0) for i in range(2))    # h, d, n
        qq = q[b, :n_kv * G * d].double().reshape(n_kv, G, d)
        s, mag = qq @ k * scale, qq.abs() @ k.abs() * scale
        p = torch.softmax(s, 2)
        want[b] = p @ v.transpose(1, 2)
        # a score is off by at most (d + 4) roundings of its terms; its exponential by that, the subtraction and 2 more; sums of n terms
        delta = 2 * (d + 4) * U * mag.amax(2, keepdim=True) + 4 * U * (s.amax(2, keepdim=True) - s.amin(2, keepdim=True)) + (n + 80) * U
        planes = 2.0 ** -15 if o_dt == BF else 0.0
        tol[b] = (delta + planes) * (p @ v.abs().transpose(1, 2))
    want, tol = want.reshape(batch, -1), tol.reshape(batch, -1)
    tol = tol + (half_step(BF) * (want.abs() + tol) if o_dt == BF else 4 * U * want.abs())
    ws = nan_like((B.attn_workspace_floats(batch, n_kv * G, d, splits),), F32) if splits > 1 else None
    ld = torch.tensor(lens, dtype=torch.int32).cuda() if lens is not None else None
    ops = [B.attn_dec8_op(q.cuda(), codes[0].cuda(), codes[1].cuda(), scales.cuda(), o, batch, n_kv * G, n_kv, d, keys, cap, block, scale, lens=ld,
                          ldq=q.shape[1], splits=splits, workspace=ws)]
    if splits > 1:
        ops.append(B.attn_merge_op(ws, o, batch, n_kv * G, n_kv, d, splits))
    return ops, o, want, tol


@pytest.mark.parametrize("keys", [1, 2, 15, 16, 17, 31, 32, 33, 127, 129, 300, 1025])
@pytest.mark.parametrize("d,block,e4m3", [(128, 32, False), (64, 16, True), (128, 64, True), (64, 48, False)])
def test_attention_lengths(keys, d, block, e4m3):
    ops, o, want, tol = attn_case(2, 2, 4, d, keys, block, e4m3, F32, F32)
    launch(*ops)
    check(o, want, tol)


@pytest.mark.parametrize("G", [1, 2, 3, 5, 7, 8, 13, 16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("splits", [1, 3])
def test_attention_head_groups(G, d, splits):
    ops, o, want, tol = attn_case(2, 3, G, d, 200, 32, G % 2 == 0, F32, F32, splits=splits)
    launch(*ops)
    check(o, want, tol)


@pytest.mark.parametrize("q_dt", [F32, BF])
@pytest.mark.parametrize("o_dt", [F32, BF])
@pytest.mark.parametrize("d,e4m3", [(64, False), (64, True), (128, False), (128, True)])
def test_attention_types(q_dt, o_dt, d, e4m3):
    ops, o, want, tol = attn_case(3, 2, 4, d, 333, 128, e4m3, q_dt, o_dt, splits=2, ldq_pad=24, qstd=2.0)
    launch(*ops, atom_blocks=5)
    check(o, want, tol)


@pytest.mark.parametrize("splits", [1, 2, 7, 64])
def test_attention_lengths_of_their_own(splits):
    lens = [0, 1, 500, 31, 33, -3, 501, 100000, 250]               # none, a few, all, more than the cache is said to hold
    ops, o, want, tol = attn_case(len(lens), 2, 4, 128, 500, 32, False, F32, F32, lens=lens, splits=splits)
    launch(*ops)
    check(o, want, tol)
    assert bool((o[[0, 5]] == 0).all())


@pytest.mark.parametrize("splits", [1, 4])
def test_attention_in_atoms_is_the_whole_launch_on_any_partition(splits):
    ops, o, want, tol = attn_case(4, 8, 4, 128, 700, 32, True, F32, F32, splits=splits, lens=[700, 3, 0, 401])
    launch(*ops)
    whole = o.clone()
    check(o, want, tol)
    part = B.lithos_create_partition(ctx(), B.lithos_make_mask(ctx(), 40))
    try:
        o.fill_(float("nan"))
        launch(*ops, atom_blocks=7, part=part)
    finally:
        B.lithos_destroy_partition(part)
    assert bits_equal(o, whole)


def test_attention_keys_behind_the_length_are_not_read():
    lens = [70, 10]
    ops, o, want, tol = attn_case(2, 2, 4, 128, 96, 32, True, F32, F32, lens=lens)
    kc, vc, sc = (ops[0]._keep[0][i] for i in (1, 2, 4))
    for b, n in enumerate(lens):
        kc.view(torch.uint8)[b, n:], vc.view(torch.uint8)[b, n:] = 0x7F, 0x7F            # e4m3 NaN
        sc[:, b, -(-n // 32):] = float("nan")
    launch(*ops)
    check(o, want, tol)


def test_attention_passes_on_what_is_no_number():
    ops, o, want, tol = attn_case(2, 2, 2, 64, 50, 16, False, F32, F32, splits=2)
    q = ops[0]._keep[0][0]
    q[1, 64 + 5] = float("nan")                                    # query head 1 of sequence 1
    launch(*ops)
    got = o.cpu().reshape(2, 4, 64)
    assert bool(torch.isnan(got[1, 1]).all())
    got[1, 1] = want.reshape(2, 4, 64)[1, 1].float()
    check(got.reshape(2, -1).cuda(), want, tol)


def test_attention_offsets_beyond_32_bits():
    # one sequence of 2^21 positions x 8 heads x 128 = 2^31 bytes of keys, and as many values; the last keys alone matter
    cap, n_kv, d, block, n = 1 << 21, 8, 128, 1024, 65
    kc, vc = (torch.zeros(1, cap, n_kv, d, dtype=torch.int8, device="cuda") for _ in range(2))
    sc = torch.ones(2, 1, cap // block, n_kv, device="cuda")
    q = torch.zeros(1, n_kv * d, device="cuda")
    q[0, 7 * d:] = 1.0
    kc[0, -n:, 7], vc[0, -n:, 7] = 1, torch.arange(n * d, device="cuda").reshape(n, d).remainder(100).to(torch.int8)
    o = nan_like((1, n_kv * d), F32)
    ws = nan_like((B.attn_workspace_floats(1, n_kv, d, 64),), F32)
    launch(B.attn_dec8_op(q, kc, vc, sc, o, 1, n_kv, n_kv, d, cap, cap, block, 1.0, splits=64, workspace=ws), B.attn_merge_op(ws, o, 1, n_kv, n_kv, d, 64))
    # scores 128 against 0: the other 2^21 positions weigh exp(-128)
    want = vc[0, -n:, 7].double().mean(0)
    assert bool(((o[0, 7 * d:].double() - want).abs() <= (n + 80) * U * 100).all())
    assert bool((o[0, :7 * d] == 0).all())
    # and an append at the far end
    x = torch.randn(1, n_kv * d, generator=rnd(12)).cuda()
    launch(B.kv8_append_op(x, x, kc, vc, sc, 1, 1, n_kv, d, cap - block, cap, block))
    s = (x.reshape(n_kv, d).abs().amax(1).cpu() / torch.tensor(127.0))
    assert torch.equal(sc[0, 0, -1].cpu(), s) and torch.equal(kc[0, cap - block].cpu(), nearest(x.cpu().reshape(n_kv, d) / s[:, None], False))


# ---- log probabilities -------------------------------------------------------------------------

def logits(rows, vocab, dt, pad=0, masked=0.0, std=3.0, seed=40):
    g = rnd(seed + rows + vocab)
    x = (std * torch.randn(rows, vocab + pad, generator=g)).to(dt)
    if masked:
        x[torch.rand(rows, vocab + pad, generator=g) < masked] = -math.inf
    return x


def lp_plain(x, tokens, top, scale):
    """stats, ids and a bound on the rounding of the stats."""
    rows, vocab = x.shape
    z = x.double() * scale
    lse = torch.logsumexp(z, 1)
    lp = z - lse[:, None]
    none = torch.isneginf(lse)
    lp[none] = -math.inf
    p = lp.exp()
    ent = -torch.where(p > 0, p * lp, 0.0).sum(1)
    given = torch.zeros(rows, dtype=F64)
    for r, t in enumerate(tokens):
        if 0 <= t < vocab:
            given[r] = lp[r, t]
    ids = torch.stack([torch.argsort(x[r].float() + 0.0, descending=True, stable=True)[:top] for r in range(rows)]) if top else torch.zeros(rows, 0, dtype=torch.int64)
    stats = torch.cat([given[:, None], ent[:, None], lse[:, None], lp.gather(1, ids)], 1)
    # a lane adds 16 values of every fourth tile of 1024, then 6 + 3 + 64 partial sums; every exponent is off by 3 roundings of |z|
    zmax = torch.where(torch.isfinite(z), z.abs(), 0.0).amax(1)
    rel = (16 * math.ceil(vocab / 4096) + 96) * U + 8 * U * zmax
    tol = rel[:, None] * (1 + 2 * math.log(vocab + 1)) + 8 * U * (zmax[:, None] + stats.abs().nan_to_num(posinf=0.0))
    return stats, ids, tol


def check_lp(stats, ids, x, tokens, top, scale):
    want, wids, tol = lp_plain(x, tokens, top, scale)
    got = stats.cpu().double()[:, :3 + top]
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf])
    off = torch.where(inf, 0.0, got - want).abs()
    assert bool((off <= tol).all()), "off by %g" % off.max()
    assert torch.equal(ids.cpu()[:, :top].long(), wids)
    assert bool(torch.isnan(stats[:, 3 + top:]).all()) and bool((ids[:, top:] == -7).all())


def lp_run(x, vocab, tokens, top, scale=1.0, splits=1, atom_blocks=0, pad=2):
    rows = x.shape[0]
    xd = x.cuda()
    td = torch.tensor(tokens, dtype=torch.int32).cuda() if tokens is not None else None
    stats, ids = nan_like((rows, 3 + top + pad), F32), torch.full((rows, top + pad), -7, dtype=torch.int32, device="cuda")
    args, kw = (xd, td, stats, ids, rows, vocab, top), dict(scale=scale, ldx=xd.stride(0), lds=3 + top + pad, ldi=top + pad)
    if splits == 1:
        launch(B.logprobs_op(*args, **kw), atom_blocks=atom_blocks)
    else:
        ws = nan_like((B.logprobs_workspace_floats(rows, top, splits),), F32)
        launch(B.logprobs_op(*args, **kw, splits=splits, workspace=ws), B.logprobs_merge_op(ws, *args, splits, **kw), atom_blocks=atom_blocks)
    return stats, ids


@pytest.mark.parametrize("vocab", [1, 2, 31, 33, 63, 1000, 1023, 1024, 1025, 4097, 20011])
@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("splits", [1, 3])
def test_logprobs_vocabularies(vocab, dt, splits):
    top, rows = min(20, vocab), 5
    tokens = [0, vocab - 1, -1, vocab, vocab // 2]
    x = logits(rows, vocab, dt, pad=3)
    stats, ids = lp_run(x, vocab, tokens, top, splits=splits, scale=0.8)
    check_lp(stats, ids, x[:, :vocab], tokens, top, 0.8)


@pytest.mark.parametrize("top", [0, 1, 2, 5, 8, 31, 32])
@pytest.mark.parametrize("splits", [1, 2, 64])
def test_logprobs_top(top, splits):
    rows, vocab = 6, 9001
    tokens = list(range(rows))
    x = logits(rows, vocab, F32)
    stats, ids = lp_run(x, vocab, tokens, top, splits=splits, atom_blocks=5)
    check_lp(stats, ids, x, tokens, top, 1.0)


@pytest.mark.parametrize("kind", ["rising", "falling", "equal", "two_values", "signed_zeros", "last"])
@pytest.mark.parametrize("splits", [1, 5])
def test_logprobs_order(kind, splits):
    """Rows where many elements have to pass through the list, or where only the index decides."""
    vocab, top = 12345, 32
    ramp = torch.arange(vocab) / 1000.0
    x = {"rising": ramp, "falling": -ramp, "equal": torch.full((vocab,), 1.5), "two_values": (torch.arange(vocab) % 7 == 3).float(),
         "signed_zeros": torch.where(torch.arange(vocab) % 2 == 0, -0.0, 0.0), "last": torch.where(torch.arange(vocab) >= vocab - 40, 2.0, -1.0)}[kind]
    x = x[None].repeat(3, 1)
    for dt in (F32, BF):
        stats, ids = lp_run(x.to(dt), vocab, [0, 5, vocab - 1], top, splits=splits)
        check_lp(stats, ids, x.to(dt), [0, 5, vocab - 1], top, 1.0)


@pytest.mark.parametrize("splits", [1, 4])
@pytest.mark.parametrize("dt", [F32, BF])
def test_logprobs_of_forbidden_tokens(splits, dt):
    rows, vocab, top = 7, 5003, 8
    x = logits(rows, vocab, dt, masked=0.9)
    x[1] = -math.inf                                                # nothing is allowed
    x[2] = -math.inf
    x[2, 4000] = 1.0                                                # one token is
    x[3] = torch.finfo(dt).min                                      # masked by the type's lowest value
    x[3, 17] = 0.0
    x[4] = torch.finfo(dt).min                                      # everywhere
    tokens = [int(torch.isneginf(x[0]).nonzero()[0]), 5, 4000, 17, 9, 3, 1]
    stats, ids = lp_run(x, vocab, tokens, top, splits=splits)
    keep = [0, 1, 2, 3, 5, 6]
    check_lp(stats[keep], ids[keep], x[keep], [tokens[i] for i in keep], top, 1.0)
    # equal logits: whatever their value, uniform
    got = stats[4].cpu()
    assert abs(float(got[0]) + math.log(vocab)) < 1e-5 and abs(float(got[1]) - math.log(vocab)) < 1e-5 and ids[4, :top].cpu().tolist() == list(range(top))


@pytest.mark.parametrize("splits", [1, 3])
def test_logprobs_of_rows_with_what_is_no_number(splits):
    rows, vocab, top = 5, 3000, 4
    x = logits(rows, vocab, F32)
    x[1, 2500], x[3, 7] = math.nan, math.inf
    stats, ids = lp_run(x, vocab, [1] * rows, top, splits=splits)
    good = [0, 2, 4]
    check_lp(stats[good], ids[good], x[good], [1] * 3, top, 1.0)
    assert bool(torch.isnan(stats[[1, 3], :3]).all())
    assert bool(((ids[:, :top] >= 0) & (ids[:, :top] < vocab)).all())


def test_logprobs_without_tokens_and_with_large_logits():
    rows, vocab = 3, 2000
    x = logits(rows, vocab, F32, std=300.0)                         # far apart: one token carries the row
    stats, ids = lp_run(x, vocab, None, 3, splits=2)
    check_lp(stats, ids, x, [-1] * rows, 3, 1.0)
    x = logits(rows, vocab, BF) + 2000.0
    stats, ids = lp_run(x, vocab, [5, 6, 7], 3)
    check_lp(stats, ids, x, [5, 6, 7], 3, 1.0)


@pytest.mark.parametrize("rows,vocab,splits", [(3, 16385, 1), (3, 32768, 1), (3, 32769, 1), (2, 65536, 1), (2, 65537, 1), (2, 140003, 1), (2, 140003, 2), (2, 140003, 5),
                                               (2, 140003, 64), (257, 5003, 1), (300, 9001, 1), (120, 9001, 3)])
@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("masked", [0.0, 0.9])
def test_logprobs_long_rows_and_many_rows(rows, vocab, splits, dt, masked):
    x = logits(rows, vocab, dt, pad=3, masked=masked)
    tokens = [(7919 * r) % vocab for r in range(rows)]
    for top in (0, 7, 32):
        stats, ids = lp_run(x, vocab, tokens, top, scale=0.8, splits=splits)
        check_lp(stats, ids, x[:, :vocab], tokens, top, 0.8)


@pytest.mark.parametrize("kind", ["rising", "falling", "equal", "two_values", "none"])
@pytest.mark.parametrize("rows,vocab", [(1, 50001), (1, 65536), (1, 100003), (300, 6001)])
def test_logprobs_order_of_long_rows_and_many_rows(kind, rows, vocab):
    i = torch.arange(vocab).float()
    row = {"rising": i / vocab, "falling": -i / vocab, "equal": 0 * i + 1.5, "two_values": (torch.arange(vocab) % 7 == 3).float(), "none": 0 * i - math.inf}[kind]
    x = row[None].repeat(rows, 1)
    for top in (1, 32):
        stats, ids = lp_run(x, vocab, [vocab - 1] * rows, top)
        check_lp(stats[-1:], ids[-1:], x[-1:], [vocab - 1], top, 1.0)
        assert bits_equal(stats, stats[-1:].repeat(rows, 1)) and torch.equal(ids, ids[-1:].repeat(rows, 1))


def test_logprobs_in_atoms_is_the_whole_launch():
    x = logits(9, 7001, BF, masked=0.3)
    for splits in (1, 3):
        a = lp_run(x, 7001, list(range(9)), 6, splits=splits)
        b = lp_run(x, 7001, list(range(9)), 6, splits=splits, atom_blocks=2)
        assert torch.equal(a[0].nan_to_num(), b[0].nan_to_num()) and torch.equal(a[1], b[1])


def test_logprobs_offsets_beyond_32_bits():
    rows, vocab = 3, (1 << 30) // 2 + 5                             # the third row begins behind 2^31 bytes
    x = torch.zeros(rows, vocab, dtype=BF, device="cuda")
    x[2, vocab - 1], x[2, 77] = 30.0, 29.0
    stats, ids = nan_like((rows, 5), F32), torch.zeros(rows, 2, dtype=torch.int32, device="cuda")
    ws = nan_like((B.logprobs_workspace_floats(rows, 2, 64),), F32)
    t = torch.tensor([1, 2, vocab - 1], dtype=torch.int32, device="cuda")
    args = (x, t, stats, ids, rows, vocab, 2)
    launch(B.logprobs_op(*args, splits=64, workspace=ws), B.logprobs_merge_op(ws, *args, 64))
    e30, e29 = math.exp(30), math.exp(29)
    lse = math.log(e30 + e29 + vocab - 2)
    assert ids.cpu().tolist() == [[0, 1], [0, 1], [vocab - 1, 77]]
    assert abs(float(stats[2, 2]) - lse) < 1e-4 and abs(float(stats[2, 0]) - (30 - lse)) < 1e-4 and abs(float(stats[0, 2]) - math.log(vocab)) < 1e-5


# ---- their gradient -------------------------------------------------------------------------------

def grad_run(x, vocab, tokens, stats, glp, gent, scale, d_dt, pad=0, atom_blocks=0):
    rows = x.shape[0]
    dx = nan_like((rows, vocab + pad), d_dt)
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    td = torch.tensor(tokens, dtype=torch.int32).cuda() if tokens is not None else None
    launch(B.logprobs_grad_op(dev(x), td, dev(stats), dev(glp), dev(gent), dx, rows, vocab, scale=scale, ldx=x.shape[1], ldd=vocab + pad), atom_blocks=atom_blocks)
    return dx


def grad_plain(x, tokens, stats, glp, gent, scale):
    """The formula with the given statistics, and a bound on its rounding."""
    H, lse = stats[:, 1:2].double(), stats[:, 2:3].double()
    lp = x.double() * scale - lse
    p = lp.exp()
    g, ge = glp.double()[:, None].clone(), gent.double()[:, None]
    hot = torch.zeros_like(p)
    for r, t in enumerate(tokens):
        if 0 <= t < x.shape[1]:
            hot[r, t] = 1.0
        else:
            g[r] = 0.0
    lph = torch.where(p > 0, lp + H, 0.0)
    dx = scale * (g * (hot - p) - ge * p * lph)
    arg = 4 * U * (lp.abs() + lse.abs()).nan_to_num(posinf=0.0)              # of an exponent; 8 roundings of the rest
    tol = scale * ((arg + 8 * U) * p * (g.abs() + ge.abs() * (lph.abs() + 1)) + 4 * U * g.abs() * hot + ge.abs() * p * 4 * U * (lp.abs().nan_to_num(posinf=0.0) + H.abs()))
    return dx, tol


@pytest.mark.parametrize("vocab", [1, 7, 8, 9, 2047, 2048, 2049, 5003])
@pytest.mark.parametrize("x_dt,d_dt", [(F32, F32), (BF, BF), (BF, F32), (F32, BF)])
def test_grad(vocab, x_dt, d_dt):
    rows, scale = 5, 0.7
    tokens = [0, vocab - 1, -1, vocab, vocab // 2]
    x = logits(rows, vocab, x_dt, pad=1)
    stats, _, _ = lp_plain(x[:, :vocab], tokens, 0, scale)
    stats = stats.float()
    glp, gent = torch.randn(rows, generator=rnd(50)), torch.randn(rows, generator=rnd(51))
    dx = grad_run(x, vocab, tokens, stats, glp, gent, scale, d_dt, pad=3, atom_blocks=4)
    want, tol = grad_plain(x[:, :vocab], tokens, stats, glp, gent, scale)
    check(dx, want, tol + (half_step(BF) * (want.abs() + tol) if d_dt == BF else 2 * U * want.abs()) + 1e-38)


def test_grad_against_differences_of_the_definition():
    rows, vocab, scale = 2, 40, 0.9
    x = logits(rows, vocab, F32, masked=0.2)
    tokens = [int((~torch.isneginf(x[r])).nonzero()[3]) for r in range(rows)]
    stats, _ = lp_run(x, vocab, tokens, 0, scale=scale, pad=0)
    glp, gent = torch.tensor([0.8, -1.1]), torch.tensor([0.5, 0.9])
    dx = grad_run(x, vocab, tokens, stats, glp, gent, scale, F32).cpu().double()

    def total(z):
        s, _, _ = lp_plain(z, tokens, 0, scale)
        return (glp.double() * s[:, 0] + gent.double() * s[:, 1]).sum()

    h = 1e-4
    for r in range(rows):
        for i in range(vocab):
            if torch.isneginf(x[r, i]):
                assert dx[r, i] == 0.0
                continue
            a, b = x.double(), x.double()
            a[r, i] += h
            b[r, i] -= h
            # third derivatives of both are below 10: h^2 / 6 * 10, and the fp32 arithmetic
            assert abs(float(dx[r, i]) - float(total(a) - total(b)) / (2 * h)) < 5e-7 + 2e-5 * 0.1


@pytest.mark.parametrize("which", ["logprob", "entropy", "neither", "no_tokens"])
def test_grad_with_gradients_left_out(which):
    rows, vocab = 3, 500
    x, tokens = logits(rows, vocab, F32), [3, 4, 5]
    stats = lp_plain(x, tokens, 0, 1.0)[0].float()
    one, zero = torch.ones(rows), torch.zeros(rows)
    glp, gent = (one if which == "logprob" else None), (one if which in ("entropy", "no_tokens") else None)
    dx = grad_run(x, vocab, None if which == "no_tokens" else tokens, stats, glp, gent, 1.0, F32)
    want, tol = grad_plain(x, tokens, stats, zero if glp is None else glp, zero if gent is None else gent, 1.0)
    check(dx, want, tol + 2 * U * want.abs() + 1e-38)


@pytest.mark.parametrize("dt", [F32, BF])
def test_grad_of_forbidden_tokens_and_in_place(dt):
    rows, vocab = 4, 3001
    x = logits(rows, vocab, dt, masked=0.5)
    x[1] = -math.inf
    x[:, 11] = torch.tensor([0.5, -math.inf, 0.25, 1.0]).to(dt)
    tokens = [11, 11, -1, 11]
    stats, _ = lp_run(x, vocab, tokens, 0, pad=0)
    glp, gent = torch.randn(rows, generator=rnd(52)), torch.randn(rows, generator=rnd(53))
    dx = grad_run(x, vocab, tokens, stats, glp, gent, 1.0, dt)
    assert bool(torch.isfinite(dx).all()) and bool((dx[1] == 0).all()) and bool((dx[torch.isneginf(x).cuda()] == 0).all())
    keep = [0, 2, 3]
    want, tol = grad_plain(x[keep], [tokens[i] for i in keep], stats[keep].cpu(), glp[keep], gent[keep], 1.0)
    check(dx[keep], want, tol + (half_step(BF) * (want.abs() + tol) if dt == BF else 2 * U * want.abs()) + 1e-38)
    own = x.cuda()
    launch(B.logprobs_grad_op(own, torch.tensor(tokens, dtype=torch.int32).cuda(), stats, glp.cuda(), gent.cuda(), own, rows, vocab))
    assert bits_equal(own, dx)




@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("scale", [1.0, 2.0])
def test_grad_of_tokens_masked_by_the_lowest_value(dt, scale):
    rows, vocab = 4, 2500
    x = logits(rows, vocab, dt)
    x[torch.rand(rows, vocab, generator=rnd(54)) < 0.4] = torch.finfo(dt).min
    x[:, 5], x[3, 6] = 1.0, torch.finfo(dt).min
    tokens = [5, 5, -1, 6]
    stats, _ = lp_run(x, vocab, tokens, 0, scale=scale, pad=0)
    glp, gent = torch.tensor([0.7, 0.0, -1.3, 0.4]), torch.tensor([3.0, -2.5, 1.5, 0.0])
    dx = grad_run(x, vocab, tokens, stats, glp, gent, scale, dt)
    want, tol = grad_plain(x, tokens, stats.cpu(), glp, gent, scale)
    check(dx, want, tol + (half_step(BF) * (want.abs() + tol) if dt == BF else 2 * U * want.abs()) + 1e-38)


def test_grad_of_rows_with_what_is_no_number():
    rows, vocab = 3, 700
    x = logits(rows, vocab, F32)
    x[1, 300], x[2, 7] = math.nan, math.inf
    stats, _ = lp_run(x, vocab, [1] * rows, 0, pad=0)
    for glp, gent in ((torch.ones(rows), None), (None, torch.ones(rows))):
        dx = grad_run(x, vocab, [1] * rows, stats, glp, gent, 1.0, F32)
        assert bool(torch.isfinite(dx[0]).all()) and bool(torch.isnan(dx[1:]).all())
