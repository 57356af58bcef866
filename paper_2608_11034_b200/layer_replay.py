"""Replay of an attention layer on R replicas, and consensus over what it leaves.

    python -m paper_2608_11034_b200.layer_replay [--tokens 2048] [--replicas 3]

The dense recipe of Sec. 6 for one layer: the input x that the layer captured is kept
in 8 bits (``replay.checkpoint_pack``); a replay restores it, runs the projections and
attention forward, attention backward, and takes the weight gradients of the query,
key and value projections straight from the checkpoint.  Output, row statistics and
all gradients of every replica are then signed and voted on (``binding.Plan``): a
healthy group certifies, and a single flipped bit in one replica's checkpoint names
that replica.  The projections themselves are plain library products; everything
between them is this package's.
"""
from __future__ import annotations

import argparse
from types import SimpleNamespace

import torch

from . import binding, replay

_NAMES = {torch.bfloat16: "bf16", torch.float16: "f16", torch.float32: "f32"}


def make_layer(tokens: int, hidden: int, q_heads: int, kv_heads: int, head_dim: int, dtype=torch.bfloat16, seed: int = 0):
    """Random weights, a captured input and the gradient that arrives at the layer's attention output."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s, scale: (torch.randn(*s, generator=g, device="cuda") * scale).to(dtype)     # noqa: E731
    w = {n: normal(h * head_dim, hidden, scale=hidden ** -0.5) for n, h in (("q", q_heads), ("k", kv_heads), ("v", kv_heads))}
    codes, exps = replay.checkpoint_pack(normal(tokens, hidden, scale=1.0))
    return SimpleNamespace(w=w, codes=codes, exps=exps, dtype=dtype, heads=dict(q=q_heads, k=kv_heads, v=kv_heads),
                           head_dim=head_dim, grad=normal(1, tokens, q_heads, head_dim, scale=1e-3))


def replay_layer(layer, codes: torch.Tensor, exps: torch.Tensor):
    """One replay from the checkpoint (codes, exps) of the layer's input: the surfaces that peers compare.  Raises
    replay.WaitGaveUp where they are not valid: a replica that has not computed them does not take part in the vote."""
    with replay.waits_checked(codes.device):
        x = replay.checkpoint_unpack(codes, exps, layer.dtype)
        t = x.shape[0]
        q, k, v = ((x @ layer.w[n].t()).view(1, t, layer.heads[n], layer.head_dim) for n in "qkv")
        o, lse = replay.attention_forward(q, k, v, causal=True)
        grads = replay.attention_backward(q, k, v, o, lse, layer.grad, causal=True)
        surfaces = dict(o=o, lse=lse)
        for n, g in zip("qkv", grads):
            surfaces["d" + n] = g
            surfaces["dw" + n] = replay.checkpoint_wgrad(g.view(t, -1), codes, exps)
    return surfaces


def compare(replicas, chunk_bytes: int = 1 << 16):
    """Certify the surfaces of all replicas.  -> (report of Plan.certify, names of the surfaces it speaks of, per outlier)"""
    names = list(replicas[0])
    specs = [SimpleNamespace(nbytes=x.numel() * x.element_size(), dtype=_NAMES[x.dtype], shape=tuple(x.shape))
             for x in replicas[0].values()]
    plan = binding.Plan(len(replicas), binding.make_tensor_table(specs), chunk_bytes)
    plan.bind([[r[n] for n in names] for r in replicas])
    result = plan.certify()
    where = sorted({(names[binding.scout_plan_chunk_info(plan.handle, c)[0]], r) for c, r in result["outliers"]})
    plan.close()
    return result, where


def flip_bit(codes: torch.Tensor, index: int, bit: int) -> torch.Tensor:
    """A copy of a checkpoint's codes with one bit flipped, made on the host side of the tensor."""
    bad = codes.clone()
    bad.view(-1)[index] ^= (1 << bit) if bit < 7 else -128
    return bad


def main(argv=None) -> int:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--replicas", type=int, default=3)
    a = ap.parse_args(argv)
    layer = make_layer(a.tokens, a.hidden, 32, 8, 128)
    verdicts = {binding.CERTIFIED: "certified", binding.VERDICT_ATTRIBUTED: "attributed", binding.UNDECIDED: "undecided"}

    def run(title, codes_of):
        replicas = [replay_layer(layer, codes_of(r), layer.exps) for r in range(a.replicas)]
        result, where = compare(replicas)
        rep = result["report"]
        print("%-28s %s: %d of %d chunks disagree%s" % (title, verdicts[rep["verdict"]], rep["n_attributed"] + rep["n_inconclusive"],
              rep["n_chunks"], "; " + ", ".join("%s of replica %d" % w for w in where) if where else ""))

    run("healthy replicas:", lambda r: layer.codes)
    bad = flip_bit(layer.codes, (a.tokens // 3) * a.hidden + 17, 6)
    run("one bit flipped in replica 1:", lambda r: bad if r == 1 else layer.codes)
    return 0


if __name__ == "__main__":
    raise SystemExit(main())
