"""The weight gradient where it is cut: many output tiles, many tokens, rows of dy on any boundary.  Sums of small integers
are exact in fp32, so that a lost or doubled token shows; sums of one sign over many tokens show how chains round."""
import pytest
import torch

import replay_defn as defn

pytestmark = pytest.mark.gpu
BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(autouse=True)
def no_wait_gives_up():
    yield
    from paper_2608_11034_b200 import binding
    assert binding.scout_replay_error() == 0


def integers(seed, rows, cols, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-3, 4, (rows, cols), generator=g, device="cuda").to(dtype)


def off_boundary(x, by):
    """the same matrix as a view whose rows start `by` elements past those of a larger one, of odd width"""
    room = torch.full((x.shape[0], x.shape[1] + by + (x.shape[1] + by + 1) % 2), float("nan"), dtype=x.dtype, device=x.device)
    room[:, by:by + x.shape[1]] = x
    return room[:, by:by + x.shape[1]]


SIZES = [  # rows, outs, ins
    (1, 1, 1), (1, 8, 8), (31, 40, 33), (33, 63, 129), (64, 128, 256), (255, 64, 64), (256, 64, 64), (257, 72, 67), (259, 1000, 520), (1025, 130, 257),
    (4100, 20, 40), (70000, 9, 17), (67528, 9, 17),   # few outputs: parts of 1120 and of 1056 tokens, the last of 1000
    (2100, 1700, 2900), (3001, 2050, 2570),  # more than 148 tiles: several to a block, three chains each
    (700, 1281, 5121), (2049, 60, 19000),    # the same with few outputs a token
    (8, 1031, 1024),
]


@pytest.mark.parametrize("dtype,out", [(BF, F32), (BF, BF), (HF, F32), (HF, HF)])
@pytest.mark.parametrize("rows,outs,ins", SIZES)
def test_every_token_once(dtype, out, rows, outs, ins):
    from paper_2608_11034_b200 import replay
    x, dy = integers(rows, rows, ins, dtype), integers(rows + 1, rows, outs, dtype)
    codes, exps = replay.checkpoint_pack(x)
    assert torch.equal(defn.restore(codes[:64], exps[:64]), x[:64].double())
    want = (dy.double().t() @ x.double())
    assert rows * 9 < 1 << 24
    got = replay.checkpoint_wgrad(dy, codes, exps, out_dtype=out)
    assert torch.equal(got, want.to(out))
    room = integers(7, outs, ins + 3, out)
    before = room.clone()
    grad = room[:, 1:1 + ins]
    replay.checkpoint_wgrad(dy, codes, exps, grad=grad)
    assert torch.equal(grad, (want + before[:, 1:1 + ins].double()).to(out))
    assert torch.equal(room[:, :1], before[:, :1]) and torch.equal(room[:, 1 + ins:], before[:, 1 + ins:])


@pytest.mark.parametrize("dtype,out", [(BF, F32), (BF, BF), (HF, F32)])
@pytest.mark.parametrize("rows,outs,ins", [(300, 64, 64), (2500, 128, 300), (4096, 256, 512), (3000, 131, 259), (2100, 1700, 2900), (5000, 40, 72)])
def test_the_bits_do_not_depend_on_where_dy_lies(dtype, out, rows, outs, ins):
    """What consensus rests on: equal values give equal bits, whatever the boundary and stride of their rows."""
    from paper_2608_11034_b200 import replay
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(rows, ins, generator=g, device="cuda").to(dtype)
    dy = torch.randn(rows, outs, generator=g, device="cuda").to(dtype)
    codes, exps = replay.checkpoint_pack(x)
    want = replay.checkpoint_wgrad(dy, codes, exps, out_dtype=out)
    croom = torch.full((rows, ins + 5), -128, dtype=torch.int8, device="cuda")
    croom[:, 3:3 + ins] = codes
    for by in (1, 2, 4, 7, 8):
        assert torch.equal(replay.checkpoint_wgrad(off_boundary(dy, by), codes, exps, out_dtype=out), want), by
    assert torch.equal(replay.checkpoint_wgrad(off_boundary(dy, 3), croom[:, 3:3 + ins], exps, out_dtype=out), want)
    # and the gradient that it is added to
    grad, room = torch.full((outs, ins), 0.5, dtype=out, device="cuda"), torch.full((outs, ins + 1), 0.5, dtype=out, device="cuda")
    replay.checkpoint_wgrad(dy, codes, exps, grad=grad)
    replay.checkpoint_wgrad(off_boundary(dy, 5), codes, exps, grad=room[:, 1:])
    assert torch.equal(grad, room[:, 1:])


@pytest.mark.parametrize("rows,outs,ins", [(16384, 1700, 2900), (16384, 40, 19000), (16384, 1701, 2900), (131072, 60, 129)])
def test_chains_are_cut(rows, outs, ins):
    """Tokens of one sign and similar size.  A matrix instruction of 16 tokens drops, on average, at most half a unit in the last place
    (2^-24) of the sum that it adds to; over a chain of 1024 tokens that sum is on average half of the chain's, and additions in
    fp32 round to nearest: no bias beyond 64 * 2^-24 / 2.  One chain over all tokens would have rows / 1024 times that."""
    from paper_2608_11034_b200 import replay
    g = torch.Generator(device="cuda").manual_seed(9)
    x = (1.0 + torch.rand(rows, ins, generator=g, device="cuda")).to(BF)
    dy = (1.0 + torch.rand(rows, outs, generator=g, device="cuda")).to(BF)
    if outs % 2:
        dy = off_boundary(dy, 1)
    codes, exps = replay.checkpoint_pack(x)
    xd = defn.restore(codes, exps)
    want = dy.double().t() @ xd
    got = replay.checkpoint_wgrad(dy, codes, exps).double()
    off = (got - want) / want
    assert off.mean().abs() <= 64 * 2.0 ** -24 / 2
    assert off.abs().max() <= 64 * 2.0 ** -23 + (rows // 1024) * 2.0 ** -24
