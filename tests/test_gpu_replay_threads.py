"""A call from a host thread that has not used the GPU before (autograd runs the backward pass in one) gives the same bits as any other."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


def in_a_new_thread(f):
    got = []

    def run():
        try:
            got.append(f())
        except Exception as e:      # noqa: BLE001 - handed to the thread that waits
            got.append(e)

    t = threading.Thread(target=run)
    t.start()
    t.join()
    if isinstance(got[0], Exception):
        raise got[0]
    return got[0]


def operators():
    from paper_2608_11034_b200 import replay
    g = torch.Generator(device="cuda").manual_seed(2)
    q, k, v, do = (torch.randn(2, 300, 4, 64, generator=g, device="cuda").bfloat16() for _ in range(4))
    o, lse = replay.attention_forward(q, k, v, causal=True)
    x, dy = torch.randn(700, 200, generator=g, device="cuda"), torch.randn(700, 136, generator=g, device="cuda").bfloat16()
    codes, exps = replay.checkpoint_pack(x)
    return {"forward": lambda: replay.attention_forward(q, k, v, causal=True),
            "backward": lambda: replay.attention_backward(q, k, v, o, lse, do, causal=True),
            "wgrad": lambda: (replay.checkpoint_wgrad(dy, codes, exps),),
            "pack": lambda: replay.checkpoint_pack(x),
            "unpack": lambda: (replay.checkpoint_unpack(codes, exps),)}


@pytest.mark.parametrize("name", ["forward", "backward", "wgrad", "pack", "unpack"])
def test_first_call_of_a_thread(name):
    f = operators()[name]
    want = f()
    torch.cuda.synchronize()
    for _ in range(3):
        got = in_a_new_thread(f)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
