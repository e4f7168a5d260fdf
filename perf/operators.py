"""The operators of a quantised decode step and of the answer made from it, as timed cases.

Kinds

* ``q4``       product of a few rows with a weight matrix in 4 bits with a scale (and a zero point) per group
               of ``group`` consecutive k, with the epilogues of the weight-streaming GEMM or the gated SiLU.
* ``append``   new keys and values quantised into a cache of 8 bits with a scale per block of positions and head.
* ``attn``     one query token per sequence against such a cache, grouped-query, sequences of their own lengths.
* ``logprobs`` log probability of a given token per row of logits, the row's entropy and log-sum-exp and its
               most likely tokens.
* ``grad``     the gradient of log probability and entropy with respect to the logits.

A code ``c`` of 4 bits stands for ``scale * (c - zero)``.  Codes are kept as ``[N/16, K/128, 4, 16, 4, 4]`` bytes: of
16 weight rows (4th axis) and 128 k, the 32 k of step ``st`` (5th) and piece ``kg`` (3rd) are ``32 st + 8 kg + j`` and
``+ j + 4`` in the low and high half of byte ``j`` (6th).  Scales and zeros are bf16 ``[N/16, K/group, 16]``.

``own`` False: elementary torch operations; True: the library's operators through their descriptors.
"""
import math

import torch

own = False

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
E4M3 = torch.float8_e4m3fn


# ---- cases ---------------------------------------------------------------------------

def listed():
    return [
        # attention's output projection of one decode request, fp32 residual stream: launch latency counts
        dict(name="q4_b1", kind="q4", m=1, n=4096, k=4096, group=128, zeros=False, a32=True, out32=True, epilogue=1, glu=False),
        # gate and up matrix of a decode batch of 8, the largest of a layer
        dict(name="q4_b8_gate_up", kind="q4", m=8, n=14336, k=4096, group=64, zeros=True, a32=True, out32=True, epilogue=0, glu=True),
        # a projection whose sizes fill neither tiles nor groups, at the largest batch, bf16 in and out
        dict(name="q4_b27_odd", kind="q4", m=27, n=5003, k=2088, group=32, zeros=True, a32=False, out32=False, epilogue=2, glu=False),
        # one token of each of 16 sequences, each at a position of its own: the smallest call
        dict(name="append_step_b16", kind="append", batch=16, tokens=1, n_kv=8, d=128, pos=2049, cap=2304, block=32, ragged=True, e4m3=False, x32=True),
        # a whole prompt, written behind a shared prefix that ends inside a block
        dict(name="append_prompt_8192", kind="append", batch=1, tokens=8192, n_kv=8, d=128, pos=13, cap=8320, block=64, ragged=False, e4m3=True, x32=False),
        # a short conversation alone: latency
        dict(name="attn_b1_300", kind="attn", batch=1, n_kv=8, group=4, d=128, keys=300, cap=512, block=32, ragged=False, e4m3=False, q32=True),
        # a decode batch of unequal sequences, one of them not begun
        dict(name="attn_b16_2049", kind="attn", batch=16, n_kv=8, group=4, d=128, keys=2049, cap=2112, block=32, ragged=True, e4m3=True, q32=True),
        # long documents; heads of 64, seven query heads a key/value head
        dict(name="attn_b8_32768_d64", kind="attn", batch=8, n_kv=8, group=7, d=64, keys=32768, cap=32768, block=64, ragged=False, e4m3=False, q32=False),
        # the answers of a decode batch of 4: one row is split over many workgroups
        dict(name="logprobs_b4", kind="logprobs", rows=4, vocab=131072, pad=0, top=8, masked=False, x32=True, scale=0.7),
        # odd vocabulary, rows without alignment, three quarters of the tokens forbidden
        dict(name="logprobs_33_odd", kind="logprobs", rows=33, vocab=32003, pad=0, top=32, masked=True, x32=False, scale=1.0),
        # scoring a prompt: every row has a given token; the largest call
        dict(name="logprobs_2048", kind="logprobs", rows=2048, vocab=131072, pad=64, top=5, masked=False, x32=False, scale=1.0),
        # a training step on log probability and entropy
        dict(name="grad_1024", kind="grad", rows=1024, vocab=50001, pad=7, masked=False, x32=True, scale=1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["q4", "q4", "q4", "append", "attn", "attn", "attn", "logprobs", "logprobs", "grad"])
    if kind == "q4":
        m, n = _log(rng, 1, 32), _log(rng, 256, 28672)
        k = max(64, _log(rng, 256, min(14336, 28672 * 4096 // n)) // 8 * 8)
        glu = rng.random() < 0.25
        if glu:
            n = max(16, n // 32 * 16)
        return dict(kind=kind, m=m, n=n, k=k, group=rng.choice([32, 64, 128]), zeros=rng.random() < 0.5, a32=rng.random() < 0.6,
                    out32=rng.random() < 0.6, epilogue=0 if glu else rng.choice([0, 1, 2]), glu=glu)
    if kind == "append":
        batch, d, block = _log(rng, 1, 16), rng.choice([64, 128]), rng.choice([16, 32, 64, 128])
        tokens = rng.choice([1, 1, _log(rng, 2, max(2, 8192 // batch))])
        pos = rng.choice([0, _log(rng, 1, 4096)])
        return dict(kind=kind, batch=batch, tokens=tokens, n_kv=rng.choice([1, 2, 4, 8]), d=d, pos=pos,
                    cap=pos + tokens + _log(rng, 1, 300), block=block, ragged=rng.random() < 0.6, e4m3=rng.random() < 0.5, x32=rng.random() < 0.5)
    if kind == "attn":
        batch, n_kv, d = _log(rng, 1, 16), rng.choice([1, 2, 4, 8]), rng.choice([64, 128])
        keys = _log(rng, 1, 32768)
        keys = max(1, min(keys, (8 * 8 * 64 * 32768) // (batch * n_kv * d)))
        return dict(kind=kind, batch=batch, n_kv=n_kv, group=rng.choice([1, 2, 3, 4, 5, 7, 8, 16]), d=d, keys=keys, cap=keys + rng.randint(0, 100),
                    block=rng.choice([16, 32, 64, 128]), ragged=rng.random() < 0.5, e4m3=rng.random() < 0.5, q32=rng.random() < 0.5)
    rows, vocab = _log(rng, 1, 2048), _log(rng, 1000, 131072)
    x32 = rng.random() < 0.5
    rows = max(1, min(rows, (1024 * 50001 if kind == "grad" else 2048 * 65536) // vocab))
    c = dict(kind=kind, rows=rows, vocab=vocab, pad=rng.choice([0, 0, 1, 8]), masked=rng.random() < 0.3, x32=x32, scale=rng.choice([1.0, 0.7, 1.4]))
    if kind == "logprobs":
        c["top"] = rng.choice([0, 1, 5, 8, 20, 32])
    return c


# ---- what a user's program has before the call ------------------------------------------

class _Draws:
    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(1000003 * int(seed) + 29)

    def normal(self, shape, std=1.0, mean=0.0, dtype=F32):
        return torch.randn(shape, generator=self.gen, device="cuda", dtype=F32).mul_(std).add_(mean).to(dtype)

    def uniform(self, shape):
        return torch.rand(shape, generator=self.gen, device="cuda", dtype=F32)

    def ints(self, lo, hi, shape, dtype=torch.int32):
        return torch.randint(lo, hi, shape, generator=self.gen, device="cuda", dtype=dtype)


def _up(a, b):
    return -(-a // b)


def prepare(case, seed):
    d, kind = _Draws(seed), case["kind"]
    st = dict(case)
    if kind == "q4":
        m, n, k, g = case["m"], case["n"], case["k"], case["group"]
        rows = 2 * n if case["glu"] else n
        st["a"] = d.normal((m, k), dtype=F32 if case["a32"] else BF16)
        st["codes"] = d.ints(0, 256, (_up(rows, 16), _up(k, 128), 4, 16, 4, 4), torch.uint8)
        # scales of weights of N(0, 0.02^2) spread over 16 steps
        shape = (_up(rows, 16), _up(k, g), 16)
        st["scales"] = (0.004 + 0.004 * d.uniform(shape)).to(BF16)
        st["zeros"] = (7.5 + d.normal(shape)).to(BF16) if case["zeros"] else None
        st["bias"] = d.normal((n,)) if case["epilogue"] == 2 else None
        st["residual"] = d.normal((m, n)) if case["epilogue"] else None
        st["c"] = torch.zeros((m, n), dtype=F32 if case["out32"] else BF16, device="cuda")
        st["outs"] = [st["c"]]
    elif kind == "append":
        b, t, h, w, cap, blk = (case[x] for x in ("batch", "tokens", "n_kv", "d", "cap", "block"))
        dt = F32 if case["x32"] else BF16
        qmax = 448.0 if case["e4m3"] else 127.0
        # a packed row of projections, of which keys and values are the last parts; channels of unequal size
        chan = torch.exp(0.7 * d.normal((2 * h * w,)))
        st["x"] = (d.normal((b * t, 2 * h * w + 64)) * torch.cat([torch.ones(64, device="cuda"), chan])).to(dt)
        st["k"], st["v"] = st["x"][:, 64:64 + h * w], st["x"][:, 64 + h * w:]
        past = d.normal((2, b, cap, h, w)) * chan.view(2, 1, 1, h, w) * (0.3 * qmax / 4)
        past = past.clamp(-qmax, qmax)
        st["cache"] = past.to(E4M3) if case["e4m3"] else past.round().to(torch.int8)
        st["scales"] = (3.0 + d.uniform((2, b, _up(cap, blk), h))) / qmax
        span = case["pos"] + 1
        st["positions"] = d.ints(0, span, (b,)) if case["ragged"] else None
        st["outs"] = [st["cache"], st["scales"]]
    elif kind == "attn":
        b, h, g, w, keys, cap, blk = (case[x] for x in ("batch", "n_kv", "group", "d", "keys", "cap", "block"))
        qmax = 448.0 if case["e4m3"] else 127.0
        codes = torch.empty((2, b, cap, h, w), dtype=E4M3 if case["e4m3"] else torch.int8, device="cuda")
        for i in range(2):
            for j in range(b):
                x = d.normal((cap, h, w), qmax / 4).clamp_(-qmax, qmax)
                codes[i, j] = x.to(E4M3) if case["e4m3"] else x.round().to(torch.int8)
        st["cache"] = codes
        st["scales"] = (2.0 + 3.0 * d.uniform((2, b, _up(cap, blk), h))) / qmax
        st["q"] = d.normal((b, h * g * w), dtype=F32 if case["q32"] else BF16)
        st["scale"] = 1.0 / math.sqrt(w)
        st["lens"] = None
        if case["ragged"]:
            st["lens"] = d.ints(1, keys + 1, (b,))
            st["lens"][0] = keys
            if b > 1:
                st["lens"][1] = 0
        st["o"] = torch.zeros((b, h * g * w), dtype=F32 if case["q32"] else BF16, device="cuda")
        st["outs"] = [st["o"]]
    else:
        r, v = case["rows"], case["vocab"]
        dt = F32 if case["x32"] else BF16
        x = torch.empty((r, v + case["pad"]), dtype=dt, device="cuda")
        for i in range(0, r, 256):
            x[i:i + 256] = d.normal((min(256, r - i), v + case["pad"]), 3.0)
        if case["masked"]:
            x[d.uniform((r, v + case["pad"])) < 0.75] = -math.inf
        st["x"] = x
        st["targets"] = d.ints(0, v, (r,))
        if r >= 16:
            st["targets"][::16] = -1                    # padding: no given token
        if case["masked"]:                              # a given token is an allowed one
            x.scatter_(1, st["targets"].clamp(min=0).long().unsqueeze(1), torch.zeros((r, 1), dtype=dt, device="cuda"))
        if kind == "grad":
            z = x[:, :v].double() * case["scale"]
            lse = torch.logsumexp(z, 1)
            p = torch.exp(z - lse.unsqueeze(1))
            ent = lse - torch.where(p > 0, p * z, 0.0).sum(1)
            st["stats"] = torch.stack([torch.zeros_like(lse), ent, lse], 1).float()
            del z, p
            st["g_logprob"], st["g_entropy"] = d.normal((r,)), d.normal((r,), 0.01)
            st["dx"] = torch.zeros((r, v), dtype=dt, device="cuda")
            st["outs"] = [st["dx"]]
        else:
            st["stats"] = torch.zeros((r, 3 + case["top"]), dtype=F32, device="cuda")
            st["ids"] = torch.zeros((r, case["top"]), dtype=torch.int32, device="cuda")
            s = st["stats"]
            st["outs"] = [s[:, 0], s[:, 1], s[:, 2]] + ([s[:, 3:], st["ids"]] if case["top"] else [])
    if own:
        st["ops"] = _descriptors(st)
    torch.cuda.synchronize()        # the library's queues are not ordered behind torch's stream
    return st


# ---- the library's calls ------------------------------------------------------------------

_ctx = None


def _descriptors(st):
    """The operators of a pass, as a program keeps them, with the workspace that a split launch needs."""
    from paper_2504_15465_amd import binding as B
    global _ctx
    if _ctx is None:
        _ctx = B.lithos_init(0, None)
    kind = st["kind"]
    if kind == "q4":
        return [B.gemm_q4_op(st["a"], st["codes"], st["scales"], st["c"], st["m"], st["n"], st["k"], st["group"], zeros=st["zeros"],
                             bias=st["bias"], gelu=st["epilogue"] == 2, residual=st["residual"], glu=st["glu"])]
    if kind == "append":
        return [B.kv8_append_op(st["k"], st["v"], st["cache"][0], st["cache"][1], st["scales"], st["batch"], st["tokens"], st["n_kv"], st["d"],
                                st["pos"], st["cap"], st["block"], positions=st["positions"], ldx=st["x"].stride(0))]
    if kind == "attn":
        args = (st["q"], st["cache"][0], st["cache"][1], st["scales"], st["o"], st["batch"], st["n_kv"] * st["group"], st["n_kv"], st["d"],
                st["keys"], st["cap"], st["block"], st["scale"])
        splits = B.lithos_split_hint(B.attn_dec8_op(*args, lens=st["lens"]), 256)
        if splits == 1:
            return [B.attn_dec8_op(*args, lens=st["lens"])]
        n_q = st["n_kv"] * st["group"]
        ws = torch.empty(B.attn_workspace_floats(st["batch"], n_q, st["d"], splits), dtype=F32, device="cuda")
        return [B.attn_dec8_op(*args, lens=st["lens"], splits=splits, workspace=ws),
                B.attn_merge_op(ws, st["o"], st["batch"], n_q, st["n_kv"], st["d"], splits)]
    r, v, ld = st["rows"], st["vocab"], st["x"].stride(0)
    if kind == "grad":
        return [B.logprobs_grad_op(st["x"], st["targets"], st["stats"], st["g_logprob"], st["g_entropy"], st["dx"], r, v, scale=st["scale"], ldx=ld)]
    args = (st["x"], st["targets"], st["stats"], st["ids"], r, v, st["top"])
    splits = B.lithos_split_hint(B.logprobs_op(*args, scale=st["scale"], ldx=ld), 256)
    if splits == 1:
        return [B.logprobs_op(*args, scale=st["scale"], ldx=ld)]
    ws = torch.empty(B.logprobs_workspace_floats(r, st["top"], splits), dtype=F32, device="cuda")
    return [B.logprobs_op(*args, scale=st["scale"], ldx=ld, splits=splits, workspace=ws),
            B.logprobs_merge_op(ws, *args, splits, scale=st["scale"], ldx=ld)]


def _launch(st):
    from paper_2504_15465_amd import binding as B
    for op in st["ops"]:
        B.lithos_launch_atomized(_ctx, op)


# ---- the operators in elementary operations --------------------------------------------------

def _unpack(codes, rows, k):
    """[N/16, K/128, kg, row, st, j] bytes -> [rows, k] codes."""
    nt, kc = codes.shape[:2]
    both = torch.stack([codes & 15, codes >> 4], 5)                 # nt, kc, kg, row, st, half, j
    return both.permute(0, 3, 1, 4, 2, 5, 6).reshape(nt * 16, kc * 128)[:rows, :k]


def _q4(st):
    n, k, g = st["n"], st["k"], st["group"]
    rows = 2 * n if st["glu"] else n
    wide = lambda t: t.float().transpose(1, 2).reshape(-1, t.shape[1])[:rows].repeat_interleave(g, 1)[:, :k]  # noqa: E731
    w = _unpack(st["codes"], rows, k).float()
    w = (w - (wide(st["zeros"]) if st["zeros"] is not None else 8.0)) * wide(st["scales"])
    y = st["a"].float() @ w.t().contiguous()
    if st["glu"]:
        y = y[:, :n] / (1.0 + torch.exp(-y[:, :n])) * y[:, n:]
    if st["epilogue"] == 2:
        y = y + st["bias"]
        y = 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    if st["epilogue"]:
        y = y + st["residual"]
    st["c"].copy_(y)


def _append(st):
    b, t, h, w, cap, blk = (st[x] for x in ("batch", "tokens", "n_kv", "d", "cap", "block"))
    e4m3 = st["e4m3"]
    nb, dev = _up(cap, blk), st["x"].device
    x = torch.stack([st["k"], st["v"]]).float().reshape(2, b, t, h, w)
    p0 = st["positions"].long() if st["positions"] is not None else torch.full((b,), st["pos"], device=dev)
    at = p0[:, None] + torch.arange(t, device=dev)                                         # [b, t]
    block = (at // blk)[None, :, :, None].expand(2, b, t, h)
    qmax = torch.full((1,), 448.0 if e4m3 else 127.0, device=dev)                          # a number would be multiplied by its reciprocal
    fresh = torch.zeros((2, b, nb, h), device=dev).scatter_reduce_(2, block, x.abs().amax(4), "amax") / qmax
    first = torch.arange(nb, device=dev)[None, :] * blk                                    # [1, nb]
    touched = ((first < (p0 + t)[:, None]) & (first + blk > p0[:, None]))[None, :, :, None]
    begun = (first < p0[:, None])[None, :, :, None]                                        # holds earlier positions
    old = st["scales"]
    new = torch.where(touched, torch.where(begun, torch.maximum(old, fresh), fresh), old)
    grown = touched & begun & (new > old)
    code = lambda y: y.clamp(-448.0, 448.0).to(E4M3) if e4m3 else y.round().clamp(-127, 127).to(torch.int8)  # noqa: E731
    over = lambda y, s: torch.where(s > 0, y / s, 0.0)  # noqa: E731
    # the one block of a sequence that is written further: its codes at the new scale
    blk0 = (p0 // blk)
    pos = blk0[:, None] * blk + torch.arange(blk, device=dev)                              # [b, blk]
    mine = (pos < p0[:, None])
    pos = pos.clamp(max=cap - 1)
    rows = torch.arange(b, device=dev)[:, None]
    s0 = old.gather(2, blk0[None, :, None, None].expand(2, b, 1, h))[..., None]            # [2, b, 1, h, 1]
    s1 = new.gather(2, blk0[None, :, None, None].expand(2, b, 1, h))[..., None]
    g0 = grown.gather(2, blk0[None, :, None, None].expand(2, b, 1, h))[..., None]
    raw = st["cache"].view(torch.uint8)
    held = raw[:, rows, pos]                                                               # [2, b, blk, h, w]
    again = code(over(held.view(st["cache"].dtype).float() * s0, s1)).view(torch.uint8)
    raw[:, rows, pos] = torch.where(g0 & mine[None, :, :, None, None], again, held)
    raw[:, rows, at] = code(over(x, new.gather(2, block)[..., None])).view(torch.uint8)
    old.copy_(new)


def _attn(st):
    b, h, g, w, keys, blk = (st[x] for x in ("batch", "n_kv", "group", "d", "keys", "block"))
    wide = lambda i: st["scales"][i].repeat_interleave(blk, 1)[:, :keys, :, None]  # noqa: E731
    kv = lambda i: (st["cache"][i, :, :keys].float() * wide(i)).permute(0, 2, 1, 3).contiguous()  # noqa: E731
    q = st["q"].float().reshape(b, h, g, w)
    s = (kv(0) @ q.transpose(2, 3).contiguous()).transpose(2, 3).contiguous() * st["scale"]         # [b, h, g, keys]
    if st["lens"] is not None:
        dead = torch.arange(keys, device=s.device)[None, :] >= st["lens"][:, None]
        s = s.masked_fill(dead[:, None, None, :], -math.inf)
    top = s.amax(3, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    o = (p @ kv(1)) / p.sum(3, keepdim=True).clamp(min=1e-30)
    st["o"].copy_(o.reshape(b, h * g * w))


def _logprobs(st):
    v, top, x = st["vocab"], st["top"], st["x"][:, :st["vocab"]].float()
    z = x * st["scale"]
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    den = e.sum(1)
    lse = m[:, 0] + torch.log(den)
    s = st["stats"]
    t = st["targets"].long()
    s[:, 0] = torch.where(t >= 0, z.gather(1, t.clamp(min=0)[:, None])[:, 0] - lse, 0.0)
    s[:, 1] = torch.log(den) - torch.where(e > 0, e * (z - m), 0.0).sum(1) / den
    s[:, 2] = lse
    if top:
        # by value, then by the lower index: one whole number of both
        bits = (x + 0.0).view(torch.int32).long()                   # -0 is 0
        key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) * (1 << 32) + (v - torch.arange(v, device=x.device))
        ids = v - (key.topk(top, 1).values & 0xFFFFFFFF)
        st["ids"].copy_(ids)
        s[:, 3:] = z.gather(1, ids) - lse[:, None]


def _grad(st):
    z = st["x"][:, :st["vocab"]].float() * st["scale"]
    lp = z - st["stats"][:, 2:3]
    p = torch.exp(lp)
    t = st["targets"].long()
    g = torch.where(t >= 0, st["g_logprob"], 0.0)[:, None]
    dz = -g * p - st["g_entropy"][:, None] * torch.where(p > 0, p * (lp + st["stats"][:, 1:2]), 0.0)
    dz.scatter_add_(1, t.clamp(min=0)[:, None], g)
    st["dx"].copy_(dz * st["scale"])


_PLAIN = {"q4": _q4, "append": _append, "attn": _attn, "logprobs": _logprobs, "grad": _grad}


def run(st):
    if own:
        _launch(st)
    else:
        _PLAIN[st["kind"]](st)
    return st["outs"]


# ---- the definitions in 64 bits ------------------------------------------------------------------

def _exact_q4(st):
    a, n = st["a"].to(F64), st["n"]
    raw = st["codes"].to(torch.int64)
    nt, kc = raw.shape[:2]
    out = torch.empty((a.shape[0], nt * 16), dtype=F64, device="cuda")
    a = torch.nn.functional.pad(a, (0, kc * 128 - a.shape[1]))
    k = torch.arange(kc * 128, device="cuda")
    chunk, step, piece, byte, high = k // 128, k % 128 // 32, k % 32 // 8, k % 4, k % 8 // 4
    group = (k // st["group"]).clamp(max=st["scales"].shape[1] - 1)
    for t0 in range(0, nt, 64):                                    # 1024 weight rows at a time
        c = raw[t0:t0 + 64].permute(0, 3, 1, 4, 2, 5)[:, :, chunk, step, piece, byte]      # tile, row, k
        c = torch.bitwise_right_shift(c, 4 * high) % 16
        z = st["zeros"][t0:t0 + 64].to(F64).permute(0, 2, 1)[:, :, group] if st["zeros"] is not None else 8.0
        w = (c.to(F64) - z) * st["scales"][t0:t0 + 64].to(F64).permute(0, 2, 1)[:, :, group]
        out[:, 16 * t0:16 * t0 + 16 * c.shape[0]] = torch.einsum("mk,nk->mn", a, w.reshape(-1, kc * 128))
    y = out[:, :n]
    if st["glu"]:
        y = y * torch.sigmoid(y) * out[:, n:2 * n]
    if st["epilogue"] == 2:
        y = y + st["bias"].to(F64)
        y = y * torch.special.ndtr(y)
    if st["epilogue"]:
        y = y + st["residual"].to(F64)
    return [y]


def _round8(y, e4m3):
    """To the nearest code, ties to the even one; in 64 bits."""
    if not e4m3:
        return torch.round(y)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(y / step) * step).clamp(-448, 448)


def _exact_append(st):
    """Scale and code are defined with the quotients rounded to 32 bits, which rounding a 64-bit quotient gives exactly."""
    e4m3, blk, t = st["e4m3"], st["block"], st["tokens"]
    quot = lambda a, s: (a / s).to(F32).to(F64) if s > 0 else torch.zeros_like(a)  # noqa: E731
    cache, scales = st["cache"].to(F64), st["scales"].to(F64).cpu()
    starts = st["positions"].tolist() if st["positions"] is not None else [st["pos"]] * st["batch"]
    for i, x in enumerate((st["k"], st["v"])):
        x = x.to(F64).reshape(st["batch"], t, st["n_kv"], st["d"])
        for b, p0 in enumerate(starts):
            for j in range(p0 // blk, (p0 + t - 1) // blk + 1):
                lo, hi = max(p0, j * blk), min(p0 + t, (j + 1) * blk)
                part = x[b, lo - p0:hi - p0]
                peak = part.abs().amax((0, 2)).cpu()
                for h in range(st["n_kv"]):
                    s = float((peak[h] / (448.0 if e4m3 else 127.0)).to(F32))
                    was = float(scales[i, b, j, h])
                    if lo > j * blk:
                        if s > was:
                            held = (cache[i, b, j * blk:lo, h] * was).to(F32).to(F64)
                            cache[i, b, j * blk:lo, h] = _round8(quot(held, s), e4m3)
                        s = max(s, was)
                    scales[i, b, j, h] = s
                    cache[i, b, lo:hi, h] = _round8(quot(part[:, h], s), e4m3)
    return [cache if e4m3 else None, scales]


def _exact_attn(st):
    h, g, w, keys, blk = (st[x] for x in ("n_kv", "group", "d", "keys", "block"))
    o = torch.zeros((st["batch"], h, g, w), dtype=F64, device="cuda")
    blocks = torch.arange(keys, device="cuda") // blk
    for b in range(st["batch"]):
        n = keys if st["lens"] is None else int(st["lens"][b])
        if n == 0:
            continue
        k, v = (st["cache"][i, b, :n].to(F64) * st["scales"][i, b].to(F64)[blocks[:n]][:, :, None] for i in range(2))
        q = st["q"][b].to(F64).reshape(h, g, w)
        p = torch.softmax(torch.einsum("hgw,nhw->hgn", q, k) * st["scale"], 2)
        o[b] = torch.einsum("hgn,nhw->hgw", p, v)
    return [o.reshape(st["batch"], -1)]


def _exact_logprobs(st):
    logits = st["x"][:, :st["vocab"]]
    parts = []
    for i in range(0, st["rows"], 256):
        z = logits[i:i + 256].to(F64) * st["scale"]
        lp = torch.log_softmax(z, 1)
        t = st["targets"][i:i + 256].long()
        given = torch.where(t < 0, 0.0, lp[torch.arange(len(t), device="cuda"), t.clamp(min=0)])
        ent = -torch.where(lp == -math.inf, 0.0, torch.exp(lp) * lp).sum(1)
        part = [given, ent, torch.logsumexp(z, 1)]
        if st["top"]:
            part.append(torch.sort(lp, 1, descending=True).values[:, :st["top"]])
        parts.append(part)
    # the most likely tokens themselves are whole numbers: equal to the plain form's
    return [torch.cat(p) for p in zip(*parts)] + ([None] if st["top"] else [])


def _exact_grad(st):
    """Through automatic differentiation of the definition, for the rows that fit at a time."""
    out = []
    for i in range(0, st["rows"], 256):
        x = st["x"][i:i + 256, :st["vocab"]].to(F64).requires_grad_()
        lp = torch.log_softmax(x * st["scale"], 1)
        t = st["targets"][i:i + 256].long()
        given = torch.where(t < 0, 0.0, lp[torch.arange(len(t), device="cuda"), t.clamp(min=0)])
        lpf = torch.where(x == -math.inf, 0.0, lp)
        ent = -(torch.exp(lp) * lpf).sum(1)
        total = (given * st["g_logprob"][i:i + 256]).sum() + (ent * st["g_entropy"][i:i + 256]).sum()
        out.append(torch.autograd.grad(total, x)[0])
    return [torch.cat(out)]


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "append" and case["batch"] * (case["tokens"] / case["block"] + 2) * case["n_kv"] > 20000:
        return None
    return {"q4": _exact_q4, "append": _exact_append, "attn": _exact_attn, "logprobs": _exact_logprobs, "grad": _exact_grad}[kind](st)


# ---- what a pass cannot do without ----------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "q4":
        m, n, k = case["m"], case["n"], case["k"]
        rows = 2 * n if case["glu"] else n
        per = (2 + 2 * case["zeros"]) * _up(k, case["group"])
        io = (4 if case["a32"] else 2) * m * k + (4 if case["out32"] else 2) * m * n
        io += (4 * m * n if case["epilogue"] else 0) + (4 * n if case["epilogue"] == 2 else 0)
        return dict(bytes=rows * (0.5 * k + per) + io, flops=2.0 * m * rows * k)
    if kind == "append":
        n = 2.0 * case["batch"] * case["tokens"] * case["n_kv"] * case["d"]
        blocks = 2.0 * case["batch"] * case["n_kv"] * _up(case["tokens"], case["block"])
        return dict(bytes=n * ((4 if case["x32"] else 2) + 1) + 8 * blocks, flops=4.0 * n)
    if kind == "attn":
        b, h, g, w, keys = (case[x] for x in ("batch", "n_kv", "group", "d", "keys"))
        each = 0.5 if case["ragged"] else 1.0           # lengths are spread over 1 .. keys
        io = 2.0 * (4 if case["q32"] else 2) * b * h * g * w
        return dict(bytes=each * b * h * keys * (2.0 * w + 8.0 / case["block"]) + io, flops=each * 4.0 * b * h * g * w * keys)
    r, v, e = case["rows"], case["vocab"], 4.0 if case["x32"] else 2.0
    if kind == "grad":
        return dict(bytes=2 * e * r * v + 24.0 * r, flops=12.0 * r * v)
    return dict(bytes=e * r * v + r * (16.0 + 8.0 * case["top"]), flops=8.0 * r * v)
