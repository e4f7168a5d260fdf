"""A decode step whose answer is split over many workgroups: in the chain, in atoms, through the scheduler and as a captured graph."""
import numpy as np
import pytest
import torch

from paper_2504_15465_amd import binding as B
from paper_2504_15465_amd import inputs
from paper_2504_15465_amd.models import DecoderChain, run_ops
from gpu_util import bits_equal, ctx
from test_gpu_quant_chain import D, FFN, H, N_KV, N_Q, check

pytestmark = pytest.mark.gpu

VOCAB = 70001
_made = {}


def build(batch=2, pos=75, seed=33):
    """One layer and a vocabulary whose rows are cut (the weights are made once)."""
    if not _made:
        ks, vs = inputs.decoder_kv_cache(1, batch, pos, N_KV, D, seed=31)
        _made.update(params=inputs.decoder_params(1, H, N_Q, N_KV, FFN, seed=30), ks=ks, vs=vs,
                     head=dict(rms=np.ones((H,), np.float32), w=inputs.normal_bits((H, VOCAB), 32, 0.05)))
    chain = DecoderChain(_made["params"], _made["ks"], _made["vs"], batch, N_Q, N_KV, pos, head=_made["head"], top=5, q4_group=64, kv8_block=32)
    chain.set_input(inputs.decoder_hidden(batch, H, seed=seed))
    chain.tokens.copy_(torch.arange(batch, dtype=torch.int32) * 30001)
    assert chain.head_splits > 1
    return chain


def answer(chain):
    return [t.clone() for t in (chain.logits, chain.stats)] + [chain.ids.clone()]


def same(a, b):
    return bits_equal(a[0], b[0]) and bits_equal(a[1], b[1]) and torch.equal(a[2], b[2])


def test_split_answer_whole_in_atoms_and_through_the_scheduler():
    chain = build()
    ops = chain.ops()
    assert ops[-1].kind == B.OP_LOGPROBS_MERGE and ops[-2].kind == B.OP_LOGPROBS
    run_ops(ctx(), ops)
    check(chain, _made["params"], _made["head"], 64)
    want = answer(chain)
    for t in (chain.logits, chain.stats, chain.head_ws):
        t.fill_(float("nan"))
    run_ops(ctx(), ops, None, atom_blocks=5)
    assert same(answer(chain), want)
    c = B.lithos_init(0, B.Config.default(max_outstanding=1, max_outstanding_hp=64))
    part = B.lithos_create_partition(c, B.lithos_make_mask(c, 64))
    tenant = B.lithos_tenant_create(c, B.CLASS_HP, part)
    try:
        for _ in range(3):
            for t in (chain.logits, chain.stats, chain.head_ws):
                t.fill_(float("nan"))
            torch.cuda.synchronize()
            for op in ops:
                B.lithos_submit(tenant, op)
            B.lithos_sync(tenant)
            assert same(answer(chain), want)
    finally:
        B.lithos_tenant_destroy(tenant)
        B.lithos_destroy_partition(part)
        B.lithos_shutdown(c)


def test_graphs_of_split_answers():
    """Two captured steps, each with its workspaces, replayed between eager work."""
    chains = [build(), build(seed=77)]
    lists = [c.ops() for c in chains]
    want = []
    for c, ops in zip(chains, lists):
        run_ops(ctx(), ops)
        want.append(answer(c))
    assert not same(*want)
    stream = torch.cuda.Stream()
    graphs = []
    for ops in lists:
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            for op in ops:
                B.lithos_launch_atomized(ctx(), op, (0, 0, 0), 0, None, stream.cuda_stream)
        graphs.append(g)
    for i in (0, 1, 1, 0, 1, 0):
        for t in (chains[i].logits, chains[i].stats, chains[i].head_ws):
            t.fill_(float("nan"))
        chains[i].ids.fill_(-1)
        torch.cuda.synchronize()
        graphs[i].replay()
        torch.cuda.synchronize()
        assert same(answer(chains[i]), want[i])
        run_ops(ctx(), lists[1 - i])                                # eager work of the other chain in between
