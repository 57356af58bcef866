"""A replay in which a wait gave up is refused on the host, before its surfaces can be signed or voted on."""
from types import SimpleNamespace

import pytest
import torch

from paper_2608_11034_b200 import binding, build, layer_replay, replay


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()


class NoDevice:
    def __init__(self, device):
        pass

    def __enter__(self):
        return self

    def __exit__(self, *a):
        return False


def with_readings(monkeypatch, *readings):
    left = list(readings)
    monkeypatch.setattr(torch.cuda, "device", NoDevice)
    monkeypatch.setattr(binding, "scout_replay_waits", lambda: left.pop(0))
    return left


@pytest.mark.parametrize("before,after,raises", [(0, 0, False), (7, 7, False), (0, 1, True), (7, 9, True), (2 ** 32 - 1, 0, True)])
def test_two_readings_that_differ(monkeypatch, before, after, raises):
    left = with_readings(monkeypatch, before, after)
    if raises:
        with pytest.raises(replay.WaitGaveUp):
            with replay.waits_checked("cuda"):
                pass
    else:
        with replay.waits_checked("cuda"):
            pass
    assert not left


def test_an_error_of_the_calls_is_not_replaced(monkeypatch):
    with_readings(monkeypatch, 0, 1)
    with pytest.raises(KeyError):
        with replay.waits_checked("cuda"):
            raise KeyError


def test_a_replay_is_refused(monkeypatch):
    """replay_layer with the operators taken by stand-ins on the CPU."""
    heads, d, t = dict(q=2, k=1, v=1), 8, 5
    layer = SimpleNamespace(w={n: torch.zeros(h * d, 16) for n, h in heads.items()}, dtype=torch.float32, heads=heads, head_dim=d,
                            grad=torch.zeros(1, t, 2, d))
    monkeypatch.setattr(replay, "checkpoint_unpack", lambda c, e, dt: c.to(dt))
    monkeypatch.setattr(replay, "attention_forward", lambda q, k, v, causal: (q, q[..., 0].transpose(1, 2)))
    monkeypatch.setattr(replay, "attention_backward", lambda q, k, v, o, lse, do, causal: (q, k, v))
    monkeypatch.setattr(replay, "checkpoint_wgrad", lambda dy, c, e: dy.t() @ c.float())
    codes = torch.zeros(t, 16, dtype=torch.int8)
    with_readings(monkeypatch, 3, 3)
    assert set(layer_replay.replay_layer(layer, codes, None)) == {"o", "lse", "dq", "dk", "dv", "dwq", "dwk", "dwv"}
    with_readings(monkeypatch, 3, 4)
    with pytest.raises(replay.WaitGaveUp):
        layer_replay.replay_layer(layer, codes, None)


def test_refusals():
    assert binding.lib().scout_replay_waits(None) == binding.lib().scout_replay_error(None) == binding.ERR_INVALID
