"""Descriptors of the quantised decode step's operators that are refused, and their plans, on the CPU: the validators launch nothing."""
import ctypes

import pytest

from paper_2504_15465_amd import binding as B

A16 = (1 << 20, 2 << 20, 3 << 20, 4 << 20, 5 << 20, 6 << 20)        # aligned addresses that nothing reads


class _Plan(ctypes.Structure):
    _fields_ = [("grid", ctypes.c_uint32 * 3), ("total", ctypes.c_uint32), ("threads", ctypes.c_uint32),
                ("wg_per_cu", ctypes.c_uint32), ("variant", ctypes.c_int)]


def plan(op):
    p = _Plan()
    rc = B.lib()["_ZN6lithos7op_planERK9lithos_opPNS_6OpPlanE"](ctypes.byref(op), ctypes.byref(p))
    return rc, p


def q4(m=4, n=100, k=256, group=64, flags=0, ld=None, inp=(A16[0], A16[1], None, None, A16[2], None), out=A16[3]):
    return B.make_op(B.OP_GEMM_Q4, (m, n, k, group), flags, ld=ld or (k, 0, n, n), inputs=inp, outputs=(out,))


def append(batch=2, t=1, n_kv=2, d=128, pos=5, cap=64, block=32, flags=0, ld=None, inp=(A16[0], A16[1], None, A16[2]), out=(A16[3], A16[4])):
    return B.make_op(B.OP_KV8_APPEND, (batch, t, n_kv, d, pos, cap, block), flags, ld=(n_kv * d if ld is None else ld,), inputs=inp, outputs=out)


def dec8(batch=2, n_q=8, n_kv=2, d=128, keys=33, cap=64, splits=1, block=32, ld=None, inp=(A16[0], A16[1], A16[2], A16[3], A16[4], None), out=A16[5]):
    return B.make_op(B.OP_ATTN_DEC8, (batch, n_q, n_kv, d, keys, cap, splits, block), 0, ld=(n_q * d if ld is None else ld,), fparam=(1.0,), inputs=inp, outputs=(out,))


def lp(kind=B.OP_LOGPROBS, rows=3, vocab=1000, top=5, splits=1, scale=1.0, ld=None, inp=(A16[0], A16[1], A16[2]), out=(A16[3], A16[4]), flags=0):
    return B.make_op(kind, (rows, vocab, top, splits), flags, ld=ld or (vocab, 3 + top, top), fparam=(scale,), inputs=inp, outputs=out)


def grad(rows=3, vocab=1000, scale=1.0, ld=None, inp=(A16[0], A16[1], A16[2], A16[3], None), out=A16[4], flags=0):
    return B.make_op(B.OP_LOGPROBS_GRAD, (rows, vocab), flags, ld=ld or (vocab, 3, vocab), fparam=(scale,), inputs=inp, outputs=(out,))


@pytest.mark.parametrize("op,blocks", [
    (append(), 2), (append(t=40, pos=20), 16), (dec8(), 4), (dec8(splits=3), 12), (dec8(n_q=32), 4),
    (lp(), 3), (lp(splits=4), 12), (lp(B.OP_LOGPROBS_MERGE, splits=4), 3), (lp(top=0, out=(A16[0], None), ld=(1000, 3, 0)), 3), (grad(vocab=2049), 6)])
def test_plans(op, blocks):
    rc, p = plan(op)
    assert rc == 0 and p.total == blocks == p.grid[0] * p.grid[1] * p.grid[2] and p.threads in (256, 512)


@pytest.mark.parametrize("op", [q4(), q4(m=33), q4(m=1, n=1, k=8, group=32), q4(n=96, flags=B.F_GLU), q4(flags=B.F_IN_F32, ld=(260, 0, 100, 100))])
def test_q4_descriptors_that_are_taken(op):
    rc, p = plan(op)
    assert rc == 0 and p.total > 0


def _with(t, i, v):
    return t[:i] + (v,) + t[i + 1:]


Q4_IN, AP_IN, D8_IN, LP_IN, GR_IN = q4.__defaults__[6], append.__defaults__[9], dec8.__defaults__[9], lp.__defaults__[7], grad.__defaults__[4]

REFUSED = [
    q4(m=0), q4(n=0), q4(k=0), q4(k=260), q4(k=12), q4(group=16), q4(group=0), q4(group=256), q4(ld=(248, 0, 100, 100)), q4(ld=(257, 0, 100, 100)), q4(ld=(256, 0, 99, 100)),
    q4(flags=B.F_IN_F32, ld=(258, 0, 100, 100)), q4(flags=B.F_BIAS), q4(flags=B.F_RESIDUAL), q4(flags=B.F_RESIDUAL, inp=_with(Q4_IN, 3, A16[4]), ld=(256, 0, 100, 99)),
    q4(flags=B.F_GLU), q4(n=96, flags=B.F_GLU | B.F_GELU), q4(n=96, flags=B.F_GLU | B.F_BIAS, inp=_with(Q4_IN, 2, A16[4])), q4(flags=B.F_TRANS_B), q4(flags=B.F_OUT_SPLIT),
    q4(flags=B.F_NORM_RMS), q4(inp=_with(Q4_IN, 0, None)), q4(inp=_with(Q4_IN, 1, None)), q4(inp=_with(Q4_IN, 4, None)), q4(inp=_with(Q4_IN, 0, A16[0] + 8)),
    q4(inp=_with(Q4_IN, 1, A16[0] + 8)), q4(inp=_with(Q4_IN, 4, A16[0] + 2)), q4(inp=_with(Q4_IN, 5, A16[0] + 2)), q4(out=None),
    append(batch=0), append(t=0), append(t=65), append(n_kv=0), append(d=96), append(d=256), append(pos=-1), append(pos=64), append(t=2, pos=63), append(cap=0), append(block=0), append(block=8),
    append(block=40), append(block=2048), append(ld=248), append(ld=260), append(flags=B.F_IN_F32, ld=258), append(out=(None, A16[0])), append(out=(A16[0], None)), append(out=(A16[0], A16[1] + 8)),
    *[append(inp=_with(AP_IN, i, None)) for i in (0, 1, 3)], append(inp=_with(AP_IN, 0, A16[0] + 2)), append(inp=_with(AP_IN, 2, A16[0] + 2)), append(inp=_with(AP_IN, 3, A16[0] + 2)),
    dec8(batch=0), dec8(n_q=7), dec8(n_q=0), dec8(n_q=34), dec8(n_kv=0), dec8(d=80), dec8(keys=0), dec8(keys=65), dec8(splits=65), dec8(block=24), dec8(ld=1000), dec8(ld=1028),
    *[dec8(inp=_with(D8_IN, i, None)) for i in (0, 1, 2, 4)], dec8(inp=_with(D8_IN, 1, A16[0] + 8)), dec8(inp=_with(D8_IN, 4, A16[0] + 2)), dec8(inp=_with(D8_IN, 5, A16[0] + 2)),
    dec8(splits=2, inp=_with(D8_IN, 3, None)), dec8(splits=2, inp=_with(D8_IN, 3, A16[0] + 4)), dec8(out=None), dec8(out=A16[0] + 1),
    lp(rows=0), lp(vocab=0), lp(top=-1), lp(top=33), lp(vocab=4, top=5, ld=(4, 8, 5)), lp(scale=0.0), lp(scale=-1.0), lp(scale=float("inf")), lp(scale=float("nan")), lp(splits=65),
    lp(ld=(999, 8, 5)), lp(ld=(1000, 7, 5)), lp(ld=(1000, 8, 4)), lp(inp=_with(LP_IN, 0, None)), lp(inp=_with(LP_IN, 0, A16[0] + 1)), lp(inp=_with(LP_IN, 0, A16[0] + 2), flags=B.F_IN_F32),
    lp(inp=_with(LP_IN, 1, A16[0] + 2)), lp(splits=2, inp=_with(LP_IN, 2, None)), lp(splits=2, inp=_with(LP_IN, 2, A16[0] + 4)), lp(B.OP_LOGPROBS_MERGE, inp=_with(LP_IN, 2, None)),
    lp(out=(None, A16[0])), lp(out=(A16[0], None)), lp(out=(A16[0] + 2, A16[1])), lp(out=(A16[0], A16[1] + 2)),
    grad(rows=0), grad(scale=0.0), grad(ld=(999, 3, 1000)), grad(ld=(1000, 2, 1000)), grad(ld=(1000, 3, 999)), grad(inp=_with(GR_IN, 0, None)), grad(inp=_with(GR_IN, 1, None)),
    grad(inp=_with(GR_IN, 2, None)), grad(inp=_with(GR_IN, 2, A16[0] + 2)), grad(inp=_with(GR_IN, 3, A16[0] + 2)), grad(inp=_with(GR_IN, 4, A16[0] + 2)), grad(out=None), grad(out=A16[0] + 1),
    grad(out=A16[0], flags=B.F_OUT_F32), grad(out=A16[0], ld=(1008, 3, 1000)),
]


@pytest.mark.parametrize("i", range(len(REFUSED)))
def test_refused(i):
    rc, _ = plan(REFUSED[i])
    assert rc == B.EINVAL
    assert b"gemm_q4" in B.lib().lithos_last_error() or b"kv8" in B.lib().lithos_last_error() or b"attn_dec8" in B.lib().lithos_last_error() or b"logprobs" in B.lib().lithos_last_error()


def test_split_hint():
    big = lambda batch, n_kv, keys: dec8(batch=batch, n_q=4 * n_kv, n_kv=n_kv, keys=keys, cap=keys)  # noqa: E731
    for op in (big(1, 8, 1), big(1, 8, 512), big(64, 8, 32768), lp(rows=1, vocab=1000), lp(rows=4096, vocab=100000), lp(rows=100, vocab=50000)):
        assert B.lithos_split_hint(op, 256) == 1
    for op, most in ((big(1, 8, 513), 5), (big(4, 8, 4096), 16), (big(1, 1, 1 << 20), 64), (lp(rows=1, vocab=131072), 64), (lp(rows=100, vocab=131072), 33)):
        for cus in (8, 64, 256):
            assert 1 <= B.lithos_split_hint(op, cus) <= most
        assert B.lithos_split_hint(op, 256) > 1
    split = dec8(splits=9, inp=_with(D8_IN, 3, None), keys=4000, cap=4000)       # its own splits and workspace are not looked at
    assert B.lithos_split_hint(split, 256) == B.lithos_split_hint(dec8(keys=4000, cap=4000), 256)
    for bad in (dec8(keys=0), lp(vocab=0), q4(), B.make_op(B.OP_ATTN_DEC, (1,))):
        with pytest.raises(B.LithosError) as e:
            B.lithos_split_hint(bad, 256)
        assert e.value.code == B.EINVAL
    with pytest.raises(B.LithosError):
        B.lithos_split_hint(dec8(), 0)
