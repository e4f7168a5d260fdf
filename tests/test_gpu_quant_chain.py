"""The decode step with 4-bit weights, an 8-bit cache and an answer: a run of its operators together, as the chain builds
them, against the same step in 64 bits on the codes that the chain holds."""
import math

import numpy as np
import pytest
import torch

from oracle import ops as O
from paper_2504_15465_amd import binding as B
from paper_2504_15465_amd import inputs, quant
from paper_2504_15465_amd.models import DecoderChain, run_ops
from gpu_util import bits_equal, ctx

pytestmark = pytest.mark.gpu

F64 = torch.float64
BATCH_SHAPES = [(1, 64), (3, 200), (16, 33), (20, 40)]
H, N_Q, N_KV, FFN, VOCAB, D = 1024, 8, 2, 1536, 3001, 128


def build(batch, pos, layers=2, **kw):
    params = inputs.decoder_params(layers, H, N_Q, N_KV, FFN, seed=30)
    ks, vs = inputs.decoder_kv_cache(layers, batch, pos, N_KV, D, seed=31)
    head = dict(rms=np.ones((H,), np.float32), w=inputs.normal_bits((H, VOCAB), 32, 0.05))
    chain = DecoderChain(params, ks, vs, batch, N_Q, N_KV, pos, head=head, top=5, **kw)
    chain.set_input(inputs.decoder_hidden(batch, H, seed=33))
    chain.tokens.copy_(torch.arange(batch, dtype=torch.int32) * 7)
    return chain, params, ks, vs, head


def dense(bits, group):
    """The [N, K] matrix that a chain's weight stands for."""
    w = inputs.bits_to_torch(np.ascontiguousarray(bits.T))
    if not group:
        return w.to(F64)
    q, s, z = quant.quantize_q4(w, group)
    wide = lambda t: t.to(F64).repeat_interleave(group, 1)[:, :w.shape[1]]  # noqa: E731
    return (q.to(F64) - wide(z)) * wide(s)


def rms(x):
    return x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-5)


def rope(x, pos):
    return torch.from_numpy(O.rope(x.numpy(), np.full((x.shape[0],), pos, dtype=np.int64)))


def plain_step(chain, params, head, group):
    """The step on the cache as the chain left it: its new keys and values are checked where they are made."""
    x = chain.x_in.cpu().to(F64)
    batch, pos = x.shape[0], chain.pos
    for li, L in enumerate(params):
        qkv = rms(x) @ dense(L["w_qkv"], group).t()
        q = rope(qkv[:, :N_Q * D].reshape(batch, N_Q, D), pos)
        k = rope(qkv[:, N_Q * D:(N_Q + N_KV) * D].reshape(batch, N_KV, D), pos)
        v = qkv[:, (N_Q + N_KV) * D:].reshape(batch, N_KV, D)
        cache = [c[li].cpu().to(torch.float32).to(F64) for c in (chain.kc, chain.vc)]
        if chain.kv8_block:
            s = chain.kv_scales[li].cpu().to(F64).repeat_interleave(chain.kv8_block, 2)[:, :, :chain.cap, :, None]
            for c, mine, si in zip(cache, (k, v), s):
                step = si[:, pos] * (1.0 if c.abs().max() <= 127 else 32.0)                # a code of int8; of e4m3 at most 32 apart
                c.mul_(si)
                assert bool(((c[:, pos] - mine).abs() <= step * 0.51).all())               # half a step, and the step before's fp32 error
        kk, vv = (c.repeat_interleave(N_Q // N_KV, 2).permute(0, 2, 1, 3) for c in cache)
        p = torch.softmax((kk @ q[..., None])[..., 0] / math.sqrt(D), 2)
        x = x + (p[:, :, None] @ vv)[:, :, 0].reshape(batch, -1) @ dense(L["w_o"], group).t()
        gu = rms(x) @ dense(L["w_gu"], group).t()
        g, u = gu[:, :FFN], gu[:, FFN:]
        x = x + (g * torch.sigmoid(g) * u) @ dense(L["w_d"], group).t()
    return x, rms(x) @ dense(head["w"], group).t()


def check(chain, params, head, group):
    x, logits = plain_step(chain, params, head, group)
    # a product of K = 1536 terms in fp32 is off by about sqrt(K) 2^-24 = 2.3e-6 of its norm; two layers of four products and
    # the norms and attention between them, then the head: 12 such steps, twice that for the residual stream's growth
    tol = 12 * 2.3e-6 * 2
    got = chain.logits.cpu().to(F64)
    assert float((chain.out.cpu().to(F64) - x).norm() / x.norm()) < tol
    assert float((got - logits).norm() / logits.norm()) < tol
    lp = torch.log_softmax(got, 1)                                  # the answer is that of the logits the chain made
    stats = chain.stats.cpu().to(F64)
    rows = torch.arange(chain.batch)
    assert float((stats[:, 0] - lp[rows, chain.tokens.cpu().long()]).abs().max()) < 1e-5
    assert float((stats[:, 1] + (lp.exp() * lp).sum(1)).abs().max()) < 1e-4
    top = torch.sort(got, dim=1, descending=True, stable=True)
    assert torch.equal(chain.ids.cpu().long(), top.indices[:, :5])
    assert float((stats[:, 3:] - lp.gather(1, top.indices[:, :5])).abs().max()) < 1e-5


@pytest.mark.parametrize("batch,pos", BATCH_SHAPES)
@pytest.mark.parametrize("kw", [dict(q4_group=64, kv8_block=32), dict(q4_group=128, kv8_block=64, kv8_e4m3=True),
                                dict(kv8_block=16), dict(q4_group=32), dict()])
def test_quantised_step(batch, pos, kw):
    chain, params, ks, vs, head = build(batch, pos, **kw)
    ops = chain.ops()
    run_ops(ctx(), ops)
    check(chain, params, head, kw.get("q4_group", 0))
    first = [t.clone() for t in (chain.out, chain.logits, chain.stats)]
    run_ops(ctx(), ops, None, atom_blocks=3)                        # again, in atoms: the cache slot is written anew
    for a, b in zip(first, (chain.out, chain.logits, chain.stats)):
        assert bits_equal(a, b)


def test_quantised_step_through_the_scheduler_and_split_launches():
    chain, params, ks, vs, head = build(2, 700, q4_group=64, kv8_block=32)
    chain.splits = 3
    chain.ws = torch.zeros(B.attn_workspace_floats(2, N_Q, D, 3), device="cuda")
    assert chain.head_splits == 1
    ops = chain.ops()
    c = B.lithos_init(0, B.Config.default(max_outstanding=1, max_outstanding_hp=64))
    part = B.lithos_create_partition(c, B.lithos_make_mask(c, 64))
    tenant = B.lithos_tenant_create(c, B.CLASS_HP, part)
    try:
        torch.cuda.synchronize()
        for _ in range(3):
            for op in ops:
                B.lithos_submit(tenant, op)
            B.lithos_sync(tenant)
            check(chain, params, head, 64)
    finally:
        B.lithos_tenant_destroy(tenant)
        B.lithos_destroy_partition(part)
        B.lithos_shutdown(c)


def test_quantised_weights_and_cache_stay_near_the_bf16_step():
    """4-bit weights of N(0, 0.02^2) in groups of 64 are off by 0.09 sigma each; what a random network makes of it is
    a relative error of the same order per layer."""
    exact, *_ = build(4, 100)
    run_ops(ctx(), exact.ops())
    for kw, most in ((dict(kv8_block=32), 0.02), (dict(q4_group=64, kv8_block=32), 0.5)):
        chain, *_ = build(4, 100, **kw)
        run_ops(ctx(), chain.ops())
        assert float((chain.logits - exact.logits).norm() / exact.logits.norm()) < most


def test_chain_refuses_what_does_not_go_together():
    with pytest.raises(ValueError):
        build(2, 10, q4_group=64, fused=True)


def test_graph_of_a_step_with_its_workspaces():
    """A captured step, replayed between eager work on another input and a second graph with workspaces of its own."""
    chains = [build(2, 600, q4_group=64, kv8_block=32)[0] for _ in range(2)]
    for c in chains:
        c.splits = 2
        c.ws = torch.zeros(B.attn_workspace_floats(2, N_Q, D, 2), device="cuda")
    chains[1].set_input(inputs.decoder_hidden(2, H, seed=77))
    lists = [c.ops() for c in chains]
    want = []
    for c, ops in zip(chains, lists):
        run_ops(ctx(), ops)
        want.append([t.clone() for t in (c.out, c.logits, c.stats)])
    stream = torch.cuda.Stream()
    graphs = []
    for c, ops in zip(chains, lists):
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            for op in ops:
                B.lithos_launch_atomized(ctx(), op, (0, 0, 0), 0, None, stream.cuda_stream)
        graphs.append(g)
    for i in (0, 1, 1, 0, 1, 0):
        for t in (chains[i].out, chains[i].logits, chains[i].stats):
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graphs[i].replay()
        torch.cuda.synchronize()
        for a, b in zip((chains[i].out, chains[i].logits, chains[i].stats), want[i]):
            assert bits_equal(a, b)
        run_ops(ctx(), lists[1 - i])                                # eager work of the other chain in between
