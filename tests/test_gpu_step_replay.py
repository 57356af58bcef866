"""The step operators together with attention, as a replay of a training step uses them: the gradients are those of the model
written out in 64 bits, healthy replicas certify bit by bit, and a flipped bit of one replica's table is attributed to it."""
import math

import pytest
import torch

import step_defn as defn

pytestmark = pytest.mark.gpu


def definition(s, number):
    """The same step by autograd in 64 bits, masks from the definition -> loss and gradients by the surfaces' names."""
    leaf = lambda x: x.double().requires_grad_()                                   # noqa: E731
    table, head, first = leaf(s.table), leaf(s.head), leaf(s.first_norm)
    blocks = [{**{n: leaf(w) for n, w in b.w.items()}, **{n: leaf(getattr(b, n)) for n in ("out", "gate", "post", "norm")}} for b in s.blocks]
    t, hidden = len(s.ids), s.table.shape[1]
    places = len(blocks) + 1
    mask = [defn.mask(t, hidden, s.p, s.seed, number * places + i).cuda() for i in range(places)]
    rms = lambda z, w: z * (z.square().mean(1, keepdim=True) + 1e-6).rsqrt() * w   # noqa: E731
    y = table[s.ids] * math.sqrt(hidden) * mask[0]
    n = rms(y, first)
    group = s.heads["q"] // s.heads["k"]
    see = torch.ones(t, t, dtype=torch.bool, device="cuda").tril()
    for b, m in zip(blocks, mask[1:]):
        q, k, v = ((n @ b[c].t()).view(t, s.heads[c], s.head_dim).transpose(0, 1) for c in "qkv")
        k, v = (x.repeat_interleave(group, 0) for x in (k, v))
        pr = torch.softmax((q @ k.transpose(1, 2) / math.sqrt(s.head_dim)).masked_fill(~see, -math.inf), -1)
        block = (pr @ v).transpose(0, 1).reshape(t, -1) @ b["out"].t()
        y = y + s.scale * b["gate"] * (rms(block, b["post"]) * m)
        n = rms(y, b["norm"])
    live = s.targets >= 0
    score = n @ head.t()
    loss = torch.where(live, torch.logsumexp(score, 1) - score.gather(1, s.targets.clamp(min=0)[:, None])[:, 0], 0.0)
    (loss * s.dloss.double()).sum().backward()
    want = dict(loss=loss.detach(), hidden=y.detach(), dhead=head.grad, dtable=table.grad, dnorm0=first.grad)
    for i, b in enumerate(blocks, 1):
        want.update({f"d{n}{i}": x.grad for n, x in b.items()})
    return want


@pytest.mark.parametrize("tokens,hidden,heads,vocab,layers", [(200, 256, (4, 2, 64), 1000, 2), (67, 136, (2, 1, 64), 333, 1)])
def test_gradients_of_a_step(tokens, hidden, heads, vocab, layers):
    """In float16.  A gradient passes some 16 stored values a layer, in the forward pass and back, each off by 2^-11 of itself at most and
    independently of the others; a norm's or a softmax's gradient may double what enters it.  64 values of twice 2^-11 are 2^-4."""
    from paper_2608_11034_b200 import step_replay
    s = step_replay.make_step(tokens, hidden, *heads, vocab, layers, dtype=torch.float16, p=0.2, seed=3)
    got, want = step_replay.replay_step(s, s.table, number=5), definition(s, 5)
    assert set(got) == set(want)
    for n, w in want.items():
        off = float((got[n].double() - w).norm() / w.norm())
        assert off <= 2.0 ** -4, (n, off)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_replicas_certify_and_a_flipped_bit_is_attributed(dtype):
    from paper_2608_11034_b200 import binding, step_replay
    from paper_2608_11034_b200.layer_replay import compare
    s = step_replay.make_step(300, 256, 4, 2, 64, 2000, dtype=dtype)
    healthy = [step_replay.replay_step(s, s.table, 1) for _ in range(3)]
    result, where = compare(healthy, 4096)
    assert result["report"]["verdict"] == binding.CERTIFIED and not where
    # the only token of its kind, so that one place decides: what dropout keeps there reaches the loss, what it drops reaches nothing
    at = 100
    assert int((s.ids == s.ids[at]).sum()) == 1
    kept = defn.mask(300, 256, s.p, s.seed, 1 * 3)[at] > 0
    dropped = step_replay.replay_step(s, step_replay.flip_bit(s.table, int(s.ids[at]), int((~kept).nonzero()[0]), 14), 1)
    assert compare([healthy[0], dropped, healthy[2]], 4096)[0]["report"]["verdict"] == binding.CERTIFIED
    struck = step_replay.replay_step(s, step_replay.flip_bit(s.table, int(s.ids[at]), int(kept.nonzero()[0]), 14), 1)
    result, where = compare([healthy[0], struck, healthy[2]], 4096)
    assert result["report"]["verdict"] == binding.VERDICT_ATTRIBUTED
    assert {r for _, r in where} == {1} and {"loss", "hidden", "dhead", "dtable", "dgate1", "dnorm0"} <= {n for n, _ in where}
    first = int((s.ids == s.ids[at]).nonzero()[0])
    assert torch.equal(struck["loss"][:first], healthy[0]["loss"][:first])        # tokens before it do not see it
    # another step drops other places
    assert not torch.equal(step_replay.replay_step(s, s.table, 2)["loss"], healthy[0]["loss"])


def test_a_captured_step():
    from paper_2608_11034_b200 import replay, step_replay
    s = step_replay.make_step(130, 128, 2, 1, 64, 500)
    want = step_replay.replay_step(s, s.table)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step_replay.replay_step(s, s.table)
    for _ in range(2):
        with replay.waits_checked(torch.device("cuda")):
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], want[n]) for n in want)


def test_command(capsys):
    from paper_2608_11034_b200 import step_replay
    assert step_replay.main(["--tokens", "256", "--hidden", "256", "--vocab", "1000"]) == 0
    out = capsys.readouterr().out
    assert "certified: 0 of" in out and "attributed" in out and "replica 1 in" in out
