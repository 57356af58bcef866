"""What the torch front end of the replay operators refuses rather than doing something other than was asked for."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def test_a_type_for_the_result_that_is_not_the_accumulated_gradients():
    from paper_2608_11034_b200 import replay
    x, dy = torch.randn(40, 64, device="cuda").to(BF), torch.randn(40, 16, device="cuda").to(BF)
    codes, exps = replay.checkpoint_pack(x)
    assert replay.checkpoint_wgrad(dy, codes, exps).dtype == F32
    for have, asked in ((F32, BF), (BF, F32)):
        grad = torch.zeros(16, 64, dtype=have, device="cuda")
        with pytest.raises(ValueError):
            replay.checkpoint_wgrad(dy, codes, exps, grad=grad, out_dtype=asked)
        assert (grad == 0).all()
        assert replay.checkpoint_wgrad(dy, codes, exps, grad=grad, out_dtype=have) is grad
        assert torch.equal(grad, replay.checkpoint_wgrad(dy, codes, exps, out_dtype=have))


def test_a_gradient_is_not_dropped_without_a_word():
    """Grad mode on and an input that requires a gradient: an error.  Off, or inside an autograd.Function, the calls run, and the
    function's gradients are the formula's."""
    from paper_2608_11034_b200 import replay

    class Attention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v):
            o, lse = replay.attention_forward(q, k, v, causal=True)
            ctx.save_for_backward(q, k, v, o, lse)
            return o

        @staticmethod
        def backward(ctx, do):
            return replay.attention_backward(*ctx.saved_tensors, do.contiguous(), causal=True)

    g = torch.Generator(device="cuda").manual_seed(2)
    q, k, v = (torch.randn(1, 130, 2, 64, generator=g, device="cuda").to(BF).requires_grad_() for _ in range(3))
    do = torch.randn(1, 130, 2, 64, generator=g, device="cuda").to(BF)
    for x in ((q, k.detach(), v.detach()), (q.detach(), k.detach(), v)):
        with pytest.raises(ValueError):
            replay.attention_forward(*x)
    with torch.no_grad():
        o, lse = replay.attention_forward(q, k, v, causal=True)
        want = replay.attention_backward(q, k, v, o, lse, do, causal=True)
    with pytest.raises(ValueError):
        replay.attention_backward(q, k, v, o, lse, do, causal=True)
    Attention.apply(q, k, v).backward(do)
    assert all(torch.equal(x.grad, y) for x, y in zip((q, k, v), want))
    codes, exps = replay.checkpoint_pack(q.view(130, 128))          # whole numbers: nothing to record
    dy = torch.randn(130, 8, device="cuda").to(BF)
    replay.checkpoint_wgrad(dy, codes, exps)
    with pytest.raises(ValueError):
        replay.checkpoint_wgrad(dy.requires_grad_(), codes, exps)


@pytest.mark.parametrize("B,T,Hq,Hk,D,bad", [(2, 131, 4, 2, 64, False), (2, 131, 4, 2, 64, True), (1, 300, 6, 3, 128, True), (2, 70, 4, 1, 80, True),
                                             (1, 2600, 1, 1, 64, False), (1, 2600, 1, 1, 64, True)])
def test_queries_keys_and_values_of_one_projection(B, T, Hq, Hk, D, bad):
    """Parts of one output, and their gradients into the same parts of one gradient: the bits of separate tensors, and nothing beside
    them is written; rows that are made again for a NaN included."""
    from paper_2608_11034_b200 import replay
    g = torch.Generator(device="cuda").manual_seed(3)
    width, gap = (Hq + 2 * Hk) * D, 24
    room = torch.randn(B, T, width + gap, generator=g, device="cuda").to(BF)
    do = torch.randn(B, T, Hq, D, generator=g, device="cuda").to(BF)
    if bad:
        room[0, T // 2, (Hq + Hk) * D + 3] = math.nan      # in the values of one token

    def parts(x):
        cut = [0, Hq * D, (Hq + Hk) * D, width]
        return [x[..., a:b].unflatten(-1, (-1, D)) for a, b in zip(cut, cut[1:])]

    q, k, v = parts(room)
    flat = [x.contiguous() for x in (q, k, v)]
    o, lse = replay.attention_forward(*flat, causal=True)
    want = replay.attention_backward(*flat, o, lse, do, causal=True)
    with pytest.raises(ValueError):
        replay.attention_backward(q, k, v, o, lse, do, causal=True)
    grad = torch.full_like(room, 7.0)
    got = replay.attention_backward(q, k, v, o, lse, do, causal=True, grads=parts(grad))
    same = lambda a, b: torch.equal(a.view(torch.int16), b.view(torch.int16))          # noqa: E731  - NaN included
    assert all(same(a.contiguous(), b) for a, b in zip(got, want)) and (grad[..., width:] == 7.0).all()
    assert any(x.isnan().any() for x in want) == bad
    for wrong in (parts(grad.half()), parts(grad[:, :-1]), [x.contiguous() for x in parts(grad)], parts(grad.cpu())):
        with pytest.raises(ValueError):
            replay.attention_backward(q, k, v, o, lse, do, causal=True, grads=wrong)
