"""The operators together, as a replay uses them: healthy replicas certify bit by bit, a flipped bit of one replica's
checkpoint is attributed to it, in the surfaces that depend on that bit and in no others."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tokens,hidden,heads", [(300, 512, (4, 2, 128)), (130, 264, (3, 1, 64))])
def test_replay_certifies_and_attributes(tokens, hidden, heads, dtype):
    from paper_2608_11034_b200 import binding, layer_replay
    layer = layer_replay.make_layer(tokens, hidden, *heads, dtype=dtype)
    healthy = [layer_replay.replay_layer(layer, layer.codes, layer.exps) for _ in range(3)]
    result, where = layer_replay.compare(healthy, 4096)
    assert result["report"]["verdict"] == binding.CERTIFIED and not where
    at = tokens // 3
    bad = layer_replay.flip_bit(layer.codes, at * hidden + 17, 6)
    assert int((bad != layer.codes).sum()) == 1
    struck = layer_replay.replay_layer(layer, bad, layer.exps)
    result, where = layer_replay.compare([healthy[0], struck, healthy[2]], 4096)
    assert result["report"]["verdict"] == binding.VERDICT_ATTRIBUTED
    assert {r for _, r in where} == {1} and {"o", "dq", "dk", "dv", "dwq", "dwk", "dwv"} <= {n for n, _ in where}
    # rows before the struck token do not see it: their outputs are the same bits
    assert torch.equal(struck["o"][:, :at], healthy[0]["o"][:, :at])
    assert torch.equal(struck["lse"][..., :at], healthy[0]["lse"][..., :at])
    # two against two of four: no side is chosen
    result, _ = layer_replay.compare([healthy[0], struck, healthy[2], layer_replay.replay_layer(layer, bad, layer.exps)], 4096)
    assert result["report"]["verdict"] == binding.UNDECIDED


def test_command(capsys):
    from paper_2608_11034_b200 import layer_replay
    assert layer_replay.main(["--tokens", "256", "--hidden", "512"]) == 0
    out = capsys.readouterr().out
    assert "certified: 0 of" in out and "attributed" in out and "of replica 1" in out
