"""Arguments of the quantised decode step's operators that the library would misread: refused where the descriptor is made, on the CPU."""
import pytest
import torch

from paper_2504_15465_amd import binding as B

F32, BF, F16, I8, U8, I32, I64, E4M3 = torch.float32, torch.bfloat16, torch.float16, torch.int8, torch.uint8, torch.int32, torch.int64, torch.float8_e4m3fn
t = lambda dtype, *shape: torch.zeros(shape or (64,), dtype=dtype)  # noqa: E731

Q4 = dict(a=F32, codes=U8, scales=BF, c=F32, zeros=BF, bias=F32, residual=F32)
APPEND = dict(k=BF, v=BF, kcodes=I8, vcodes=I8, scales=F32, positions=I32)
DEC8 = dict(q=F32, kcodes=E4M3, vcodes=E4M3, scales=F32, o=BF, lens=I32, workspace=F32)
LP = dict(logits=BF, tokens=I32, stats=F32, ids=I32, workspace=F32)
GRAD = dict(logits=BF, tokens=I32, stats=F32, g_logprob=F32, g_entropy=F32, dlogits=F32)
CALLS = [(B.gemm_q4_op, Q4, dict(m=1, n=16, k=64, group=32)),
         (B.kv8_append_op, APPEND, dict(batch=1, tokens=1, n_kv=1, d=64, pos=0, cap=16, block=16)),
         (B.attn_dec8_op, DEC8, dict(batch=1, n_q=1, n_kv=1, d=64, keys=1, cap=16, block=16, scale=1.0, splits=2)),
         (B.logprobs_op, LP, dict(rows=1, vocab=8, top=2, splits=2)),
         (B.logprobs_merge_op, LP, dict(rows=1, vocab=8, top=2, splits=2)),
         (B.logprobs_grad_op, GRAD, dict(rows=1, vocab=8))]


def make(call, types, rest, **other):
    return call(**{k: t(v) for k, v in {**types, **other}.items()}, **rest)


@pytest.mark.parametrize("call,types,rest", CALLS)
def test_tensors_of_the_operators_types_are_taken(call, types, rest):
    assert make(call, types, rest).kind > 0
    optional = {"zeros", "bias", "residual", "positions", "lens", "workspace", "tokens", "ids", "g_logprob", "g_entropy"}
    if call is not B.logprobs_merge_op:
        assert call(**{k: None if k in optional else t(v) for k, v in types.items()}, **rest).kind > 0


@pytest.mark.parametrize("call,types,rest,name", [(*c, n) for c in CALLS for n in c[1]])
@pytest.mark.parametrize("wrong", [I64, F16, torch.float64])
def test_tensors_of_other_types_are_refused(call, types, rest, name, wrong):
    with pytest.raises(ValueError, match=name):
        make(call, types, rest, **{name: wrong})


@pytest.mark.parametrize("call,types,rest,name,wrong", [
    (*CALLS[0], "codes", I32), (*CALLS[0], "scales", F32), (*CALLS[0], "zeros", F32), (*CALLS[0], "bias", BF), (*CALLS[0], "residual", BF),
    (*CALLS[1], "v", F32), (*CALLS[1], "kcodes", U8), (*CALLS[1], "vcodes", E4M3), (*CALLS[1], "scales", BF),
    (*CALLS[2], "kcodes", U8), (*CALLS[2], "vcodes", I8), (*CALLS[2], "workspace", BF), (*CALLS[3], "ids", F32), (*CALLS[5], "stats", BF)])
def test_types_that_other_arguments_have_are_refused(call, types, rest, name, wrong):
    with pytest.raises(ValueError):
        make(call, types, rest, **{name: wrong})
