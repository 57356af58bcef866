"""Measured cases of the layer-replay operators: attention forward and backward, 8-bit activation
checkpoints (pack and restore) and the weight gradient computed straight from such a checkpoint.

``run`` computes a case either in its plain form (elementary torch operations in 32 bits, rounded once at
the end) or, with ``own`` set, through ``paper_2608_11034_b200.replay``.  ``exact`` is the operators'
definition in 64 bits.
"""
import math

import torch

own = False

BLOCK = 32                      # features that share one exponent in an 8-bit checkpoint
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
# largest finite value's exponent: codes at this step stop at 63, so that a restored value stays finite
TOP_STEP = {"bf16": 122, "f32": 122, "f16": 10}


def _attention(name, op, dtype, batch, q_len, kv_len, q_heads, kv_heads, head_dim, causal, window=0, ragged=False):
    return dict(name=name, op=op, dtype=dtype, batch=batch, q_len=q_len, kv_len=kv_len, q_heads=q_heads, kv_heads=kv_heads,
                head_dim=head_dim, causal=causal, window=window, ragged=ragged)


def listed():
    return [
        # one new token per sequence against its keys so far, sequences of different lengths
        _attention("attend-token", "attend", "bf16", 8, 1, 4096, 32, 8, 128, True, ragged=True),
        # short sequences of odd length, every key visible
        _attention("attend-short", "attend", "f16", 4, 197, 197, 12, 12, 64, False),
        # one layer of a training step: 32 query heads share 8 key heads
        _attention("attend-layer", "attend", "bf16", 2, 2048, 2048, 32, 8, 128, True),
        # one long sequence whose length no tile divides
        _attention("attend-long", "attend", "bf16", 1, 8191, 8191, 32, 8, 128, True),
        # gradients of a padded batch of short sequences
        _attention("gradient-short", "gradient", "f16", 4, 333, 333, 12, 4, 64, True, ragged=True),
        # gradients of one layer of a training step
        _attention("gradient-layer", "gradient", "bf16", 2, 2048, 2048, 32, 8, 128, True),
        # gradients of a long sequence in which a token sees its last 1024 predecessors
        _attention("gradient-window", "gradient", "bf16", 1, 8192, 8192, 16, 4, 128, True, window=1024),
        # a small fp32 activation whose rows no block divides: saved, and restored for the backward pass
        dict(name="keep-small", op="keep", dtype="f32", rows=128, cols=1000),
        # a feed-forward layer's inner activations of one step
        dict(name="keep-layer", op="keep", dtype="bf16", rows=16384, cols=14336),
        # a small projection of odd sizes
        dict(name="weights-small", op="weights", dtype="f16", out="f16", rows=259, outs=1000, ins=520),
        # an attention projection, into the fp32 gradient that the optimizer reads
        dict(name="weights-attention", op="weights", dtype="bf16", out="f32", rows=4096, outs=4096, ins=4096),
        # a feed-forward projection, into a bf16 gradient bucket
        dict(name="weights-feed", op="weights", dtype="bf16", out="bf16", rows=8192, outs=14336, ins=4096),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attend", "gradient", "keep", "weights"])
    if op in ("attend", "gradient"):
        kv_heads = rng.choice([1, 2, 4, 8])
        q_heads = kv_heads * rng.choice([1, 2, 3, 4])
        batch = rng.randint(1, 8)
        kv_len = _log_int(rng, 16, 8192)
        q_len = kv_len
        if op == "attend" and rng.random() < 0.4:
            q_len = min(kv_len, rng.choice([1, 1, rng.randint(2, 64)]))
        while batch * q_heads * q_len * kv_len > 2 ** 30:      # the plain form's score matrix: at most 4 GiB
            batch, q_len, kv_len = max(1, batch // 2), max(1, q_len * 2 // 3), max(1, kv_len * 2 // 3)
        causal = rng.random() < 0.7
        window = _log_int(rng, 8, 2048) if causal and rng.random() < 0.25 else 0
        c = _attention("", op, rng.choice(["bf16", "bf16", "f16"]), batch, q_len, kv_len, q_heads, kv_heads,
                       rng.choice([64, 128, 128, 8 * rng.randint(2, 16)]), causal, window, rng.random() < 0.3)
    elif op == "keep":
        c = dict(op=op, dtype=rng.choice(["bf16", "f16", "f32"]), rows=_log_int(rng, 1, 16384), cols=_log_int(rng, 8, 14336))
    else:
        dtype = rng.choice(["bf16", "bf16", "f16"])
        c = dict(op=op, dtype=dtype, out=rng.choice(["f32", dtype]), rows=_log_int(rng, 16, 8192),
                 outs=8 * _log_int(rng, 8, 1792), ins=8 * _log_int(rng, 8, 512))
    c.pop("name", None)
    return c


# ---- inputs ------------------------------------------------------------------------------------------

def _lengths(case, gen):
    """Tokens in use of every sequence of a padded batch; the padding itself holds whatever was there."""
    if not case["ragged"]:
        return None, None
    b, tq, tk = case["batch"], case["q_len"], case["kv_len"]
    if tq == tk:
        n = torch.randint((tk + 1) // 2, tk + 1, (b,), generator=gen, device="cuda", dtype=torch.int32)
        return n, n
    kv = torch.randint(max(tq, (tk + 1) // 2), tk + 1, (b,), generator=gen, device="cuda", dtype=torch.int32)
    return None, kv


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype, scale=1.0):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32).mul_(scale).to(TYPES[dtype])

    if case["op"] in ("attend", "gradient"):
        b, tq, tk, d, t = case["batch"], case["q_len"], case["kv_len"], case["head_dim"], case["dtype"]
        s = dict(case=case, q=normal(b, tq, case["q_heads"], d, dtype=t), k=normal(b, tk, case["kv_heads"], d, dtype=t),
                 v=normal(b, tk, case["kv_heads"], d, dtype=t))
        s["q_lens"], s["kv_lens"] = _lengths(case, gen)
        if case["op"] == "gradient":
            # fp16 training scales its loss so that gradients stay in range; bf16 needs no such scale
            s["do"] = normal(b, tq, case["q_heads"], d, dtype=t, scale=1.0 if t == "f16" else 1e-3)
            s["o"], s["lse"] = _plain_attend(s)     # kept by the forward pass
        return s
    if case["op"] == "keep":
        return dict(case=case, x=_activation(case["rows"], case["cols"], gen).to(TYPES[case["dtype"]]))
    x = _activation(case["rows"], case["ins"], gen).to(TYPES[case["dtype"]])
    codes, exps = _plain_pack(x, case["dtype"])
    return dict(case=case, codes=codes, exps=exps,
                dy=normal(case["rows"], case["outs"], dtype=case["dtype"], scale=1.0 if case["dtype"] == "f16" else 1e-3))


def _activation(rows, cols, gen):
    """Hidden activations: normal, with a few feature columns an order of magnitude larger."""
    x = torch.randn(rows, cols, generator=gen, device="cuda", dtype=torch.float32)
    gain = torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.01, 12.0, 1.0)
    return x.mul_(gain)


# ---- plain forms: elementary operations in 32 bits -----------------------------------------------------

def _visible(case, q_lens, kv_lens):
    """[b or 1, q_len, kv_len] truth values: which key a query sees."""
    tq, tk = case["q_len"], case["kv_len"]
    dev = "cuda"
    nq = torch.full((1,), tq, device=dev) if q_lens is None else q_lens.long()
    nk = torch.full((1,), tk, device=dev) if kv_lens is None else kv_lens.long()
    n = max(len(nq), len(nk))
    nq, nk = nq.expand(n)[:, None, None], nk.expand(n)[:, None, None]
    i = torch.arange(tq, device=dev)[None, :, None]
    j = torch.arange(tk, device=dev)[None, None, :]
    ok = (i < nq) & (j < nk)
    if case["causal"]:
        at = i + nk - nq
        ok = ok & (j <= at)
        if case["window"]:
            ok = ok & (j > at - case["window"])
    return ok


def _heads(case, x):
    """[b, t, heads, d] -> fp32 [b, kv heads, heads per kv head, t, d]"""
    b, t, h, d = x.shape
    return x.float().reshape(b, t, case["kv_heads"], h // case["kv_heads"], d).permute(0, 2, 3, 1, 4)


def _plain_attend(s):
    case = s["case"]
    q, k, v = _heads(case, s["q"]), _heads(case, s["k"]), _heads(case, s["v"])
    hide = ~_visible(case, s["q_lens"], s["kv_lens"])[:, None, None]
    score = torch.matmul(q, k.transpose(-1, -2)).mul_(1.0 / math.sqrt(case["head_dim"]))
    score.masked_fill_(hide, -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), 0.0, top)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total == 0, 1.0, total)
    lse = (top + total.log()).squeeze(-1)
    b, g, r, t, d = o.shape
    return o.permute(0, 3, 1, 2, 4).reshape(b, t, g * r, d).to(TYPES[case["dtype"]]), lse.reshape(b, g * r, t)


def _plain_gradient(s):
    case = s["case"]
    scale = 1.0 / math.sqrt(case["head_dim"])
    q, k, v, o, do = (_heads(case, s[n]) for n in ("q", "k", "v", "o", "do"))
    hide = ~_visible(case, s["q_lens"], s["kv_lens"])[:, None, None]
    lse = s["lse"].reshape(q.shape[:-1]).unsqueeze(-1)
    p = torch.matmul(q, k.transpose(-1, -2)).mul_(scale).sub_(lse).exp_().masked_fill_(hide, 0.0)
    dv = torch.matmul(p.transpose(-1, -2), do).sum(2, keepdim=True)
    delta = (do * o).sum(-1, keepdim=True)
    ds = torch.matmul(do, v.transpose(-1, -2)).sub_(delta).mul_(p).mul_(scale)
    del p
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(-1, -2), q).sum(2, keepdim=True)

    def back(x):
        b, g, r, t, d = x.shape
        return x.permute(0, 3, 1, 2, 4).reshape(b, t, g * r, d).to(TYPES[case["dtype"]])

    return back(dq), back(dk), back(dv)


def _plain_pack(x, dtype):
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    xf = torch.nn.functional.pad(x.float(), (0, nb * BLOCK - cols)).view(rows, nb, BLOCK)
    fine = torch.isfinite(xf)
    amax = torch.where(fine, xf.abs(), 0.0).amax(-1)
    m, e = torch.frexp(amax)                           # amax = m * 2^e, m in [0.5, 1)
    e = torch.where(m <= 127.0 / 128.0, e - 7, e - 6).clamp(min=-126)
    e = torch.where(amax == 0, -126, e)
    # x * 2^-e in two exact steps: 2^126 is the largest power of two needed and both factors are finite
    half = torch.div(e, 2, rounding_mode="floor")
    one = torch.ones((), device=x.device)
    code = (xf * torch.ldexp(one, -half)[..., None] * torch.ldexp(one, half - e)[..., None]).round()
    top = torch.where(e == TOP_STEP[dtype], 63.0, 127.0)[..., None]
    code = torch.where(fine, torch.minimum(torch.maximum(code, -top), top), -128.0)
    return code.to(torch.int8).view(rows, nb * BLOCK)[:, :cols].contiguous(), e.to(torch.int8)


def _plain_restore(codes, exps):
    rows, cols = codes.shape
    step = torch.ldexp(torch.ones((), device=codes.device), exps.int()).repeat_interleave(BLOCK, dim=1)[:, :cols]
    c = codes.float()
    return torch.where(codes == -128, math.nan, c * step)


def run(state):
    case = state["case"]
    if own:
        from paper_2608_11034_b200 import replay
    if case["op"] == "attend":
        if own:
            return replay.attention_forward(state["q"], state["k"], state["v"], causal=case["causal"], window=case["window"],
                                            q_lens=state["q_lens"], kv_lens=state["kv_lens"])
        return _plain_attend(state)
    if case["op"] == "gradient":
        if own:
            return replay.attention_backward(state["q"], state["k"], state["v"], state["o"], state["lse"], state["do"],
                                             causal=case["causal"], window=case["window"], q_lens=state["q_lens"],
                                             kv_lens=state["kv_lens"])
        return _plain_gradient(state)
    if case["op"] == "keep":
        if own:
            codes, exps = replay.checkpoint_pack(state["x"])
            return replay.checkpoint_unpack(codes, exps, state["x"].dtype), exps
        codes, exps = _plain_pack(state["x"], case["dtype"])
        return _plain_restore(codes, exps).to(state["x"].dtype), exps
    if own:
        return replay.checkpoint_wgrad(state["dy"], state["codes"], state["exps"], out_dtype=TYPES[case["out"]])
    return torch.matmul(state["dy"].float().t(), _plain_restore(state["codes"], state["exps"])).to(TYPES[case["out"]])


# ---- what a pass cannot do without ---------------------------------------------------------------------

def _pairs(case):
    """Visible (query, key) pairs of one head; padded batches hold on average three quarters of their tokens."""
    b, tq, tk = case["batch"], case["q_len"], case["kv_len"]
    if case["ragged"]:
        tk = max(1, tk * 3 // 4)
        tq = tk if case["q_len"] == case["kv_len"] else tq
    if not case["causal"]:
        return b * tq * tk
    w = case["window"] or tk
    first = max(0, tk - tq)                # query i stands at position first + i
    return b * sum(min(first + i + 1, w) for i in range(tq))


def work(case):
    if case["op"] in ("attend", "gradient"):
        d, hq, hk, b = case["head_dim"], case["q_heads"], case["kv_heads"], case["batch"]
        share = 0.75 if case["ragged"] else 1.0
        nq = b * case["q_len"] * (share if case["q_len"] == case["kv_len"] else 1.0)
        nk = b * case["kv_len"] * share
        pairs = _pairs(case) * hq
        if case["op"] == "attend":
            return {"bytes": 2 * d * (2 * nq * hq + 2 * nk * hk) + 4 * nq * hq, "flops": 4 * d * pairs}
        return {"bytes": 2 * d * (4 * nq * hq + 4 * nk * hk) + 4 * nq * hq, "flops": 10 * d * pairs}
    if case["op"] == "keep":
        n = case["rows"] * case["cols"]
        size = 4 if case["dtype"] == "f32" else 2
        # saved and restored: the activation read and written, its codes and exponents written and read
        return {"bytes": 2 * size * n + 2 * n + 2 * n / BLOCK, "flops": 4 * n}
    t, o, i = case["rows"], case["outs"], case["ins"]
    return {"bytes": 2 * t * o + t * i + t * i / BLOCK + o * i * (4 if case["out"] == "f32" else 2), "flops": 2 * t * o * i}


# ---- the definition in 64 bits -------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("attend", "gradient"):
        return _exact_attention(case, s)
    if case["op"] == "keep":
        x = s["x"].double()
        rows, cols = x.shape
        back = torch.empty_like(x)
        exps = []
        for c0 in range(0, cols, BLOCK):
            part = x[:, c0:c0 + BLOCK]
            amax = part.abs().amax(1)
            e = torch.ceil(torch.log2(amax / 127.0)).clamp(min=-126.0)
            e = torch.where(amax > 127.0 * torch.exp2(e), e + 1, e)
            e = torch.where((amax <= 127.0 * torch.exp2(e - 1)) & (e > -126), e - 1, e)
            top = torch.where(e == TOP_STEP[case["dtype"]], 63.0, 127.0)[:, None]
            code = torch.round(part / torch.exp2(e)[:, None])
            back[:, c0:c0 + BLOCK] = torch.minimum(torch.maximum(code, -top), top) * torch.exp2(e)[:, None]
            exps.append(e)
        return back, None
    step = torch.exp2(s["exps"].double())
    x = s["codes"].double()
    for n in range(step.shape[1]):
        x[:, n * BLOCK:(n + 1) * BLOCK] *= step[:, n:n + 1]
    return s["dy"].double().t() @ x


def _exact_attention(case, s):
    """One sequence and one query head after the other, straight from the definition."""
    b, tq, tk, hq, d = case["batch"], case["q_len"], case["kv_len"], case["q_heads"], case["head_dim"]
    group = hq // case["kv_heads"]
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    o, lse = torch.zeros_like(q), torch.full((b, hq, tq), -math.inf, dtype=torch.float64, device="cuda")
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for n in range(b):
        nq = tq if s["q_lens"] is None else int(s["q_lens"][n])
        nk = tk if s["kv_lens"] is None else int(s["kv_lens"][n])
        at = torch.arange(nq, device="cuda")[:, None] + (nk - nq)
        key = torch.arange(nk, device="cuda")[None, :]
        seen = torch.ones(nq, nk, dtype=torch.bool, device="cuda")
        if case["causal"]:
            seen = key <= at
            if case["window"]:
                seen &= at - key < case["window"]
        any_seen = seen.any(1)
        for h in range(hq):
            g = h // group
            score = (q[n, :nq, h] @ k[n, :nk, g].t()) / math.sqrt(d)
            score = torch.where(seen, score, -math.inf)
            total = torch.logsumexp(score, 1)
            lse[n, h, :nq] = total
            p = torch.exp(score - torch.where(any_seen, total, 0.0)[:, None])
            out = p @ v[n, :nk, g]
            o[n, :nq, h] = out
            if case["op"] == "gradient":
                grad = s["do"][n, :nq, h].double()
                dp = grad @ v[n, :nk, g].t()
                ds = p * (dp - (p * dp).sum(1, keepdim=True)) / math.sqrt(d)
                dv[n, :nk, g] += p.t() @ grad
                dq[n, :nq, h] = ds @ k[n, :nk, g]
                dk[n, :nk, g] += ds.t() @ q[n, :nq, h]
    return (dq, dk, dv) if case["op"] == "gradient" else (o, lse)
