"""Replay of a training step, from its tokens to its gradients, on R replicas, and consensus over what it leaves.

    python -m paper_2608_11034_b200.step_replay [--tokens 2048] [--layers 2] [--replicas 3]

What ``layer_replay`` does for one layer, for all that lies between a step's tokens and the gradient of its embedding
(Sec. 6): lookup, dropout, attention blocks that join the residual stream (norm, dropout, gate, scale, the next
block's norm), cross entropy over the vocabulary, and back.  Dropout draws from the step's counter, so every
replica drops the same places; sums have fixed orders, so healthy replicas leave the same bits.  The surfaces (loss,
hidden states, gradients) are signed and voted on: a single flipped bit of one replica's table names that replica.
The projections are plain library products; everything between them is this package's.
"""
from __future__ import annotations

import argparse
import math
from types import SimpleNamespace

import torch

from . import binding, replay, step
from .layer_replay import compare


def make_step(tokens: int, hidden: int, q_heads: int, kv_heads: int, head_dim: int, vocab: int, layers: int = 2, dtype=torch.bfloat16,
              p: float = 0.1, seed: int = 0):
    """Random weights, tokens and targets (every eighth token is padding, which counts for nothing)."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*s, scale, mean=0.0):
        return (torch.randn(*s, generator=g, device="cuda") * scale + mean).to(dtype)

    width = {"q": q_heads * head_dim, "k": kv_heads * head_dim, "v": kv_heads * head_dim}
    blocks = [SimpleNamespace(w={n: normal(k, hidden, scale=hidden ** -0.5) for n, k in width.items()},
                              out=normal(hidden, width["q"], scale=width["q"] ** -0.5), gate=normal(hidden, scale=0.1, mean=0.5),
                              post=normal(hidden, scale=0.1, mean=1.0), norm=normal(hidden, scale=0.1, mean=1.0)) for _ in range(layers)]
    ids = torch.randint(0, vocab, (tokens + 1,), generator=g, device="cuda")
    targets = ids[1:].clone()
    ids = ids[:-1].contiguous()
    targets[::8] = -1
    dloss = (1024.0 if dtype == torch.float16 else 1.0) / (targets >= 0).sum().float()      # of the mean; fp16 is loss-scaled
    return SimpleNamespace(table=normal(vocab, hidden, scale=0.02), head=normal(vocab, hidden, scale=hidden ** -0.5), blocks=blocks,
                           first_norm=normal(hidden, scale=0.1, mean=1.0), ids=ids, targets=targets, dloss=dloss.expand(tokens), dtype=dtype,
                           heads=dict(q=q_heads, k=kv_heads, v=kv_heads), head_dim=head_dim, p=p, seed=seed, scale=1 / math.sqrt(layers))


def replay_step(s, table: torch.Tensor, number: int = 0):
    """One replay of step `number` with the embedding `table`: the surfaces that peers compare.  Raises replay.WaitGaveUp where they
    are not valid."""
    t, vocab = len(s.ids), len(table)
    places = len(s.blocks) + 1                                     # that drop something, each with a counter of its own
    drop = [dict(p=s.p, seed=s.seed, offset=number * places + i) for i in range(places)]
    root = math.sqrt(table.shape[1])
    with replay.waits_checked(table.device), torch.no_grad():
        e = step.embedding_forward(s.ids, table, scale=root)
        y, n, stats = step.join_forward(None, e, norm_weight=s.first_norm, **drop[0])
        kept = [(None, None, None, None, None, e, y, stats)]
        for b, d in zip(s.blocks, drop[1:]):
            q, k, v = ((n @ b.w[c].t()).view(1, t, s.heads[c], s.head_dim) for c in "qkv")
            o, lse = replay.attention_forward(q, k, v, causal=True)
            block = o.view(t, -1) @ b.out.t()
            before = n
            y, n, stats = step.join_forward(y, block, gate=b.gate, post_weight=b.post, norm_weight=b.norm, scale=s.scale, **d)
            kept.append((before, q, k, v, (o, lse), block, y, stats))
        loss, lse = step.loss_forward(n, s.head, s.targets)
        dn, dhead = step.loss_backward(n, s.head, s.targets, lse, s.dloss, out_dtype=s.dtype)
        surfaces = dict(loss=loss, hidden=y, dhead=dhead)
        dy = None
        for i in range(len(s.blocks), 0, -1):
            b = s.blocks[i - 1]
            before, q, k, v, (o, olse), block, y, stats = kept[i]
            dy, dblock, dgate, dpost, dnorm = step.join_backward(dy, dn, block, y, stats, gate=b.gate, post_weight=b.post, norm_weight=b.norm,
                                                                 scale=s.scale, **drop[i])
            grads = replay.attention_backward(q, k, v, o, olse, (dblock @ b.out).view(o.shape), causal=True)
            surfaces.update({f"dgate{i}": dgate, f"dpost{i}": dpost, f"dnorm{i}": dnorm, f"dout{i}": dblock.t() @ o.view(t, -1)})
            dn = 0
            for c, g in zip("qkv", grads):
                g = g.view(t, -1)
                surfaces[f"d{c}{i}"] = g.t() @ before
                dn = g @ b.w[c] + dn
        _, de, _, _, surfaces["dnorm0"] = step.join_backward(dy, dn, e, kept[0][6], kept[0][7], norm_weight=s.first_norm, **drop[0])
        surfaces["dtable"] = step.embedding_backward(de, s.ids, vocab, scale=root)
    return surfaces


def flip_bit(table: torch.Tensor, row: int, column: int, bit: int) -> torch.Tensor:
    """A copy of a 16-bit table with one bit flipped."""
    bad = table.clone()
    bad.view(torch.int16)[row, column] ^= (1 << bit) if bit < 15 else -32768
    return bad


def main(argv=None) -> int:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--vocab", type=int, default=32000)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--replicas", type=int, default=3)
    a = ap.parse_args(argv)
    s = make_step(a.tokens, a.hidden, max(2, a.hidden // 128), max(1, a.hidden // 256), 128, a.vocab, a.layers)
    verdicts = {binding.CERTIFIED: "certified", binding.VERDICT_ATTRIBUTED: "attributed", binding.UNDECIDED: "undecided"}

    def run(title, table_of):
        result, where = compare([replay_step(s, table_of(r), number=7) for r in range(a.replicas)])
        rep = result["report"]
        names = sorted({n for n, _ in where})
        print("%-28s %s: %d of %d chunks disagree%s" % (title, verdicts[rep["verdict"]], rep["n_attributed"] + rep["n_inconclusive"], rep["n_chunks"],
              "; replica %s in %s" % (", ".join(map(str, sorted({r for _, r in where}))), ", ".join(names)) if where else ""))

    run("healthy replicas:", lambda r: s.table)
    # a place that the step's dropout keeps: what it drops reaches nothing
    at = a.tokens // 3
    keeps = step.dropout(torch.ones(a.tokens, a.hidden, device="cuda"), s.p, seed=s.seed, offset=7 * (a.layers + 1))[at]
    bad = flip_bit(s.table, int(s.ids[at]), int(keeps.nonzero()[0]), 14)
    run("one bit flipped in replica 1:", lambda r: bad if r == 1 else s.table)
    return 0


if __name__ == "__main__":
    raise SystemExit(main())
