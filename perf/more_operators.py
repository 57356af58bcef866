"""Measured cases of the step operators, which lie around the layers of a replayed training step: token embedding and
its gradient, dropout from a counter, the join of a block with the residual stream (norms before and after the block, gate,
dropout, residual scale) and its gradient, and the softmax cross entropy over a vocabulary with its gradients.

``run`` computes a case either in its plain form (elementary torch operations in 32 bits, rounded once at the end)
or, with ``own`` set, through ``paper_2608_11034_b200.step``.  ``exact`` is the operators' definition in 64 bits.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-6
STEP_OF_TRAINING = (1 << 33) + 7      # the counter's offset: a step's number times what a step uses of it


def _join(name, op, dtype, stream, weights, rows, dim, groups, p):
    return dict(name=name, op=op, dtype=dtype, stream=stream, weights=weights, rows=rows, dim=dim, groups=groups, p=p)


def listed():
    return [
        # the tokens of a long training batch looked up in a large table, scaled by the root of the width
        dict(name="lookup-step", op="lookup", dtype="bf16", out="bf16", rows=16384, dim=4096, vocab=128000, padding=0.0),
        # a short padded batch: gradient of a small fp16 table of odd width
        dict(name="table-gradient-short", op="table", dtype="f16", out="f16", rows=1003, dim=1000, vocab=50257, padding=0.2),
        # the same for a long batch, into the fp32 gradient that the optimizer reads
        dict(name="table-gradient-step", op="table", dtype="bf16", out="f32", rows=16384, dim=4096, vocab=32000, padding=0.0),
        # dropout of a small fp32 activation, of few columns no vector divides
        dict(name="dropout-small", op="dropout", dtype="f32", rows=128, dim=1001, p=0.25),
        # a feed-forward layer's inner activations
        dict(name="dropout-step", op="dropout", dtype="bf16", rows=16384, dim=14336, p=0.1),
        # one token of each of 8 sequences passes from one block to the next
        _join("join-token", "join", "bf16", "bf16", "bf16", 8, 4096, 1, 0.0),
        # the tokens of a training step, residual stream kept in fp32, a gate for each of 8 sequences
        _join("join-step", "join", "bf16", "f32", "f32", 16384, 4096, 8, 0.1),
        # gradients for a few tokens of odd width
        _join("join-gradient-short", "join-gradient", "f16", "f16", "f16", 777, 1001, 7, 0.1),
        # gradients of a training step
        _join("join-gradient-step", "join-gradient", "bf16", "bf16", "bf16", 16384, 4096, 1, 0.1),
        # held-out text scored by a narrow model: forward pass alone, odd vocabulary
        dict(name="loss-score", op="score", dtype="bf16", rows=2048, dim=1024, vocab=50257, padding=0.0),
        # a short fp16 batch, forward and gradients
        dict(name="loss-short", op="loss", dtype="f16", rows=259, dim=520, vocab=5003, padding=0.3),
        # a training step's tokens over a large vocabulary, forward and gradients; padding does not count
        dict(name="loss-step", op="loss", dtype="bf16", rows=8192, dim=4096, vocab=128000, padding=0.1),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["lookup", "table", "dropout", "join", "join-gradient", "score", "loss", "loss"])
    if op in ("lookup", "table"):
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        return dict(op=op, dtype=dtype, out=rng.choice([dtype, "f32"]), rows=_log_int(rng, 1, 16384),
                    dim=rng.choice([8 * _log_int(rng, 8, 512), _log_int(rng, 64, 4096)]), vocab=_log_int(rng, 1000, 128000),
                    padding=rng.choice([0.0, 0.0, 0.3]))
    if op == "dropout":
        return dict(op=op, dtype=rng.choice(["bf16", "f16", "f32"]), rows=_log_int(rng, 1, 16384), dim=_log_int(rng, 64, 14336),
                    p=rng.choice([0.1, 0.5, round(rng.uniform(0.01, 0.9), 3)]))
    if op in ("join", "join-gradient"):
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        groups = rng.choice([1, 1, rng.randint(2, 16)])
        c = _join("", op, dtype, rng.choice([dtype, "f32"]), rng.choice([dtype, "f32"]), groups * _log_int(rng, 1, 16384 // groups),
                  rng.choice([8 * _log_int(rng, 8, 512), _log_int(rng, 64, 4096)]), groups, rng.choice([0.0, 0.1]))
        c.pop("name")
        return c
    return dict(op=op, dtype=rng.choice(["bf16", "bf16", "f16"]), rows=_log_int(rng, 1, 8192), dim=8 * _log_int(rng, 8, 512),
                vocab=_log_int(rng, 1000, 128000), padding=rng.choice([0.0, 0.2]))


# ---- inputs ------------------------------------------------------------------------------------------

def _tokens(case, gen):
    """Token ids by Zipf's law, in an order of the vocabulary that has nothing to do with how frequent they are; -1 for padding."""
    rows, vocab = case["rows"], case["vocab"]
    u = torch.rand(rows, generator=gen, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(vocab)).long() - 1).clamp_(0, vocab - 1)
    ids = torch.randperm(vocab, generator=gen, device="cuda")[rank]
    if case["padding"]:
        ids = torch.where(torch.rand(rows, generator=gen, device="cuda") < case["padding"], -1, ids)
    return ids


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[case["dtype"]]

    def normal(*shape, dtype=t, scale=1.0, mean=0.0):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32).mul_(scale).add_(mean).to(dtype)

    op = case["op"]
    # fp16 training scales its loss so that gradients stay in range; bf16 and fp32 need no such scale
    small = 1.0 if case["dtype"] == "f16" else 1e-3
    if op == "lookup":
        return dict(case=case, ids=_tokens(case, gen), table=normal(case["vocab"], case["dim"], scale=0.02))
    if op == "table":
        return dict(case=case, ids=_tokens(case, gen), dy=normal(case["rows"], case["dim"], scale=small))
    if op == "dropout":
        return dict(case=case, x=normal(case["rows"], case["dim"]), seed=seed)
    if op in ("join", "join-gradient"):
        rows, dim, tw, ts = case["rows"], case["dim"], TYPES[case["weights"]], TYPES[case["stream"]]
        s = dict(case=case, seed=seed, x=normal(rows, dim, dtype=ts), block=normal(rows, dim, scale=0.5),
                 gate=normal(case["groups"], dim, dtype=tw, scale=0.2, mean=0.7),
                 post=normal(dim, dtype=tw, scale=0.1, mean=1.0), norm=normal(dim, dtype=tw, scale=0.1, mean=1.0))
        if op == "join-gradient":
            s["y"], _, s["stats"] = _plain_join(s)      # kept by the forward pass
            s["dy"], s["dn"] = normal(rows, dim, dtype=ts, scale=small), normal(rows, dim, scale=small)
        return s
    rows, dim, vocab = case["rows"], case["dim"], case["vocab"]
    w, targets = normal(vocab, dim, scale=dim ** -0.5), _tokens(case, gen)
    # hidden states of a model that has learned something: each leans towards its target's row, by 4 to 14
    lean = torch.rand(rows, 1, generator=gen, device="cuda") * 10 + 4
    x = (torch.randn(rows, dim, generator=gen, device="cuda") + lean * w[targets.clamp(min=0)].float()).to(t)
    # every token that counts weighs the same in the mean over the batch
    dloss = (1.0 if case["dtype"] == "bf16" else 1024.0) / (targets >= 0).sum().clamp(min=1).float()
    return dict(case=case, x=x, w=w, targets=targets, dloss=dloss.expand(rows))


# ---- plain forms: elementary operations in 32 bits -----------------------------------------------------

def _plain_lookup(s, scale):
    ids = s["ids"]
    y = s["table"][ids.clamp(min=0)].float().mul_(scale).masked_fill_((ids < 0)[:, None], 0.0)
    return y.to(TYPES[s["case"]["out"]])


def _plain_table(s, scale):
    case, ids = s["case"], s["ids"]
    total = torch.zeros(case["vocab"] + 1, case["dim"], device="cuda")          # the last row takes what has no id
    total.index_add_(0, torch.where(ids < 0, case["vocab"], ids), s["dy"].float())
    return total[:-1].mul_(scale).to(TYPES[case["out"]])


def _bits(rows, dim, seed, offset):
    """16 random bits for each place, as whole numbers: Philox 4x32 with ten rounds (Salmon, Moraes, Dror, Shaw: "Parallel random
    numbers: as easy as 1, 2, 3", 2011), counter (column / 8, row, offset), key the seed; eight places share a counter."""
    low = 0xFFFFFFFF
    shape = (rows, -(-dim // 8))
    c0 = torch.arange(shape[1], device="cuda").expand(shape)
    c1 = torch.arange(rows, device="cuda")[:, None].expand(shape)
    c2, c3 = torch.full(shape, offset & low, device="cuda"), torch.full(shape, (offset >> 32) & low, device="cuda")
    k0, k1 = seed & low, (seed >> 32) & low
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0, c0 >> 16, c1, c1 >> 16, c2, c2 >> 16, c3, c3 >> 16], -1) & 0xFFFF
    return words.view(rows, -1)[:, :dim]


def _kept(rows, dim, p, seed, offset):
    """Which places dropout keeps, and the factor of those."""
    cut = min(65535, math.floor(p * 65536 + 0.5))
    return _bits(rows, dim, seed, offset) >= cut, 65536 / (65536 - cut)


def _plain_dropout(s):
    case = s["case"]
    keep, factor = _kept(case["rows"], case["dim"], case["p"], s["seed"], STEP_OF_TRAINING)
    return torch.where(keep, s["x"].float() * factor, 0.0).to(s["x"].dtype)


def _by_row(case, gate):
    return gate.float().repeat_interleave(case["rows"] // case["groups"], 0)


def _plain_join(s):
    case, b = s["case"], s["block"].float()
    rb = torch.rsqrt(b.square().mean(1, keepdim=True) + EPS)
    u = b * rb * s["post"].float()
    if case["p"]:
        keep, factor = _kept(case["rows"], case["dim"], case["p"], s["seed"], STEP_OF_TRAINING)
        u = torch.where(keep, u * factor, 0.0)
    y = s["x"].float() + _scale(case) * _by_row(case, s["gate"]) * u
    ry = torch.rsqrt(y.square().mean(1, keepdim=True) + EPS)
    n = y * ry * s["norm"].float()
    return y.to(s["x"].dtype), n.to(s["block"].dtype), torch.stack([rb[:, 0], ry[:, 0]])


def _plain_join_gradient(s):
    case, b, y, dn = s["case"], s["block"].float(), s["y"].float(), s["dn"].float()
    rb, ry = s["stats"][0][:, None], s["stats"][1][:, None]
    y_hat, b_hat = y * ry, b * rb
    t = dn * s["norm"].float()
    g = s["dy"].float() + ry * (t - y_hat * (t * y_hat).mean(1, keepdim=True))
    u, h = b_hat * s["post"].float(), _scale(case) * g
    du = h * _by_row(case, s["gate"])
    if case["p"]:
        keep, factor = _kept(case["rows"], case["dim"], case["p"], s["seed"], STEP_OF_TRAINING)
        u, du = torch.where(keep, u * factor, 0.0), torch.where(keep, du * factor, 0.0)
    dgate = (h * u).view(case["groups"], -1, case["dim"]).sum(1)
    dpost, dnorm = (du * b_hat).sum(0), (dn * y_hat).sum(0)
    t = du * s["post"].float()
    db = rb * (t - b_hat * (t * b_hat).mean(1, keepdim=True))
    tw = s["gate"].dtype
    return g.to(s["x"].dtype), db.to(s["block"].dtype), dgate.to(tw), dpost.to(tw), dnorm.to(tw)


def _plain_loss(s):
    case, targets = s["case"], s["targets"]
    x, w = s["x"].float(), s["w"].float()
    counts = (targets >= 0)[:, None]
    at = targets.clamp(min=0)[:, None]
    score = torch.matmul(x, w.t())
    top = score.amax(1, keepdim=True)
    lse = top + (score - top).exp_().sum(1, keepdim=True).log_()
    loss = torch.where(counts, lse - score.gather(1, at), 0.0)[:, 0]
    if case["op"] == "score":
        return loss, lse[:, 0].where(counts[:, 0], torch.zeros((), device="cuda"))
    g = score.sub_(lse).exp_()
    g.scatter_add_(1, at, torch.full_like(lse, -1.0))
    g.mul_(torch.where(counts, s["dloss"][:, None], 0.0))
    dx, dw = torch.matmul(g, w), torch.matmul(g.t(), x)
    return loss, dx.to(s["x"].dtype), dw.to(s["w"].dtype)


def _scale(case):
    """The residual scale of a deep model; a power of two it is not."""
    return 0.7


def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        from paper_2608_11034_b200 import step
    if op == "lookup":
        scale = math.sqrt(case["dim"])
        if own:
            return step.embedding_forward(state["ids"], state["table"], scale=scale, out_dtype=TYPES[case["out"]])
        return _plain_lookup(state, scale)
    if op == "table":
        scale = math.sqrt(case["dim"])
        if own:
            return step.embedding_backward(state["dy"], state["ids"], case["vocab"], scale=scale, out_dtype=TYPES[case["out"]])
        return _plain_table(state, scale)
    if op == "dropout":
        if own:
            return step.dropout(state["x"], case["p"], seed=state["seed"], offset=STEP_OF_TRAINING)
        return _plain_dropout(state)
    if op in ("join", "join-gradient"):
        if own:
            how = dict(gate=state["gate"], post_weight=state["post"], norm_weight=state["norm"], scale=_scale(case), p=case["p"],
                       seed=state["seed"], offset=STEP_OF_TRAINING)
            if op == "join":
                return step.join_forward(state["x"], state["block"], eps=EPS, **how)
            return step.join_backward(state["dy"], state["dn"], state["block"], state["y"], state["stats"], **how)
        return _plain_join(state) if op == "join" else _plain_join_gradient(state)
    if own:
        loss, lse = step.loss_forward(state["x"], state["w"], state["targets"])
        if op == "score":
            return loss, lse
        dx, dw = step.loss_backward(state["x"], state["w"], state["targets"], lse, state["dloss"], out_dtype=state["w"].dtype)
        return loss, dx, dw
    return _plain_loss(state)


# ---- what a pass cannot do without ---------------------------------------------------------------------

def work(case):
    size = {"bf16": 2, "f16": 2, "f32": 4}
    op, e = case["op"], size[case["dtype"]]
    n = case["rows"] * case["dim"]
    if op == "lookup":
        # tokens drawn by Zipf's law come again: every distinct row of the table is read once
        return {"bytes": 8 * case["rows"] + e * _distinct(case) * case["dim"] + size[case["out"]] * n, "flops": n}
    if op == "table":
        live = n * (1 - case["padding"])
        return {"bytes": 8 * case["rows"] + e * live + size[case["out"]] * case["vocab"] * case["dim"], "flops": live}
    if op == "dropout":
        return {"bytes": 2 * e * n, "flops": n}
    if op == "join":
        st, wt = size[case["stream"]], size[case["weights"]]
        return {"bytes": (2 * st + 2 * e) * n + wt * (2 + case["groups"]) * case["dim"] + 8 * case["rows"], "flops": 12 * n}
    if op == "join-gradient":
        st, wt = size[case["stream"]], size[case["weights"]]
        # dy, y and dx are of the stream's type, dn, block and its gradient of the block's
        return {"bytes": (3 * st + 3 * e) * n + 2 * wt * (2 + case["groups"]) * case["dim"] + 8 * case["rows"], "flops": 30 * n}
    live, table = case["rows"] * (1 - case["padding"]), case["vocab"] * case["dim"]
    once = 2 * live * table
    if op == "score":
        return {"bytes": e * (live * case["dim"] + table) + 16 * case["rows"], "flops": once}
    # the scores and the two products of the gradients; dx is written for padding too
    return {"bytes": e * (live * case["dim"] + n + 2 * table) + 16 * case["rows"], "flops": 3 * once}


def _distinct(case):
    """Expected number of different tokens among those of a batch: rank r is drawn with probability ln((r + 1) / r) / ln(vocab)."""
    rank = torch.arange(1, case["vocab"], dtype=torch.float64)
    live = case["rows"] * (1 - case["padding"])
    return float((1 - (1 - torch.log1p(1 / rank) / math.log(case["vocab"])) ** live).sum())


# ---- the definition in 64 bits -------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "lookup":
        hot = s["ids"] >= 0
        y = torch.zeros(case["rows"], case["dim"], dtype=torch.float64, device="cuda")
        y[hot] = s["table"][s["ids"][hot]].double() * case["dim"] ** 0.5
        return y
    if op == "table":
        hot = s["ids"] >= 0
        total = torch.zeros(case["vocab"], case["dim"], dtype=torch.float64, device="cuda")
        total.index_put_((s["ids"][hot],), s["dy"][hot].double() * case["dim"] ** 0.5, accumulate=True)
        return total
    if op == "dropout":
        return s["x"].double() * _exact_mask(case, s["seed"])
    if op in ("join", "join-gradient"):
        return _exact_join(case, s)
    return _exact_loss(case, s)


def _exact_mask(case, seed):
    """Zero or the factor of a place that is kept, in 64 bits.  The generator is written out on the CPU, in numpy's unsigned words."""
    import numpy as np
    rows, dim = case["rows"], case["dim"]
    cut = min(65535, math.floor(case["p"] * 65536 + 0.5))
    mask32, shift = np.uint64(0xFFFFFFFF), np.uint64(32)
    out = torch.empty(rows, dim, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 22) // max(1, dim))
    for r0 in range(0, rows, step):
        r1 = min(rows, r0 + step)
        col, row = np.meshgrid(np.arange(-(-dim // 8), dtype=np.uint64), np.arange(r0, r1, dtype=np.uint64))
        ctr = [col, row, np.full_like(col, STEP_OF_TRAINING & 0xFFFFFFFF), np.full_like(col, STEP_OF_TRAINING >> 32)]
        key = [np.uint64(seed & 0xFFFFFFFF), np.uint64(seed >> 32)]
        for _ in range(10):
            p0, p1 = np.uint64(0xD2511F53) * ctr[0], np.uint64(0xCD9E8D57) * ctr[2]
            ctr = [(p1 >> shift) ^ ctr[1] ^ key[0], p1 & mask32, (p0 >> shift) ^ ctr[3] ^ key[1], p0 & mask32]
            key = [(key[0] + np.uint64(0x9E3779B9)) & mask32, (key[1] + np.uint64(0xBB67AE85)) & mask32]
        words = np.stack(ctr, -1).astype("<u4").view("<u2").reshape(r1 - r0, -1)[:, :dim]
        out[r0:r1] = torch.from_numpy(np.where(words >= cut, 65536 / (65536 - cut), 0.0)).cuda()
    return out


def _exact_join(case, s):
    rows, dim = case["rows"], case["dim"]
    group = torch.arange(rows, device="cuda") // (rows // case["groups"])
    b, post, norm = s["block"].double(), s["post"].double(), s["norm"].double()
    factor = s["gate"].double()[group] * 0.7
    if case["p"]:
        factor *= _exact_mask(case, s["seed"])          # what u is multiplied by
    if case["op"] == "join":
        rb = 1 / torch.sqrt((b * b).sum(1) / dim + EPS)
        y = s["x"].double() + factor * (b * rb[:, None] * post)
        ry = 1 / torch.sqrt((y * y).sum(1) / dim + EPS)
        return y, y * ry[:, None] * norm, torch.stack([rb, ry])
    rb, ry = s["stats"].double()
    yh = s["y"].double() * ry[:, None]
    dn = s["dn"].double()
    dnorm = (dn * yh).sum(0)
    dn = dn * norm
    g = s["dy"].double() + ry[:, None] * (dn - yh * ((dn * yh).sum(1) / dim)[:, None])
    bh = b * rb[:, None]
    dgate = torch.zeros(case["groups"], dim, dtype=torch.float64, device="cuda")
    gate = s["gate"].double()[group]
    mask = factor / 0.7 / torch.where(gate == 0, 1.0, gate)
    dgate.index_add_(0, group, g * 0.7 * mask * bh * post)
    du = g * factor
    dpost = (du * bh).sum(0)
    du = du * post
    db = rb[:, None] * (du - bh * ((du * bh).sum(1) / dim)[:, None])
    return g, db, dgate, dpost, dnorm


def _exact_loss(case, s):
    """Some rows after the others, those that count alone."""
    rows = torch.nonzero(s["targets"] >= 0)[:, 0]
    w = s["w"].double()
    loss = torch.zeros(case["rows"], dtype=torch.float64, device="cuda")
    lse, dx, dw = torch.zeros_like(loss), torch.zeros(s["x"].shape, dtype=torch.float64, device="cuda"), torch.zeros_like(w)
    for part in rows.split(1024):
        x, at = s["x"][part].double(), s["targets"][part]
        score = x @ w.t()
        total = torch.logsumexp(score, 1)
        lse[part] = total
        loss[part] = total - score[torch.arange(len(part), device="cuda"), at]
        if case["op"] == "loss":
            p = torch.softmax(score, 1)
            p[torch.arange(len(part), device="cuda"), at] -= 1
            p *= s["dloss"][part].double()[:, None]
            dx[part] = p @ w
            dw += p.t() @ x
    return (loss, lse) if case["op"] == "score" else (loss, dx, dw)
