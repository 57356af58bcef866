"""What the front ends refuse before they look at devices or the library."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2608_11034_b200 import replay, step


def calls(make):
    """One call of each function for each tensor that autograd could ask for, made by `make`."""
    m, n = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    w, q, s = torch.zeros(8), torch.zeros(1, 4, 2, 8), torch.zeros(2, 4)
    codes = torch.zeros(4, 8, dtype=torch.uint8)
    yield lambda: step.embedding_forward(n, make(m))
    yield lambda: step.embedding_backward(make(m), n, 4)
    yield lambda: step.embedding_backward(m, n, 4, grad=make(m))
    yield lambda: step.dropout(make(m), 0.1, seed=1)
    for i in range(5):
        a = [m, m, w, w, w]
        a[i] = make(a[i])
        yield lambda a=a: step.join_forward(a[0], a[1], gate=a[2], post_weight=a[3], norm_weight=a[4])
    for i in range(8):
        a = [m, m, m, m, s, w, w, w]
        a[i] = make(a[i])
        yield lambda a=a: step.join_backward(*a[:5], gate=a[5], post_weight=a[6], norm_weight=a[7])
    for i in range(2):
        a = [m, m]
        a[i] = make(a[i])
        yield lambda a=a: step.loss_forward(*a, n)
    for i in range(5):
        a = [m, m, s[0], s[0], m]
        a[i] = make(a[i])
        yield lambda a=a: step.loss_backward(a[0], a[1], n, a[2], a[3], grad=a[4])
    for i in range(3):
        a = [q, q, q]
        a[i] = make(a[i])
        yield lambda a=a: replay.attention_forward(*a)
    for i in range(5):
        a = [q, q, q, q, q]
        a[i] = make(a[i])
        yield lambda a=a: replay.attention_backward(*a[:4], torch.zeros(1, 2, 4), a[4])
    yield lambda: replay.checkpoint_wgrad(make(m), codes, codes)
    yield lambda: replay.checkpoint_wgrad(m, codes, codes, grad=make(m))


def test_gradients_in_forward_mode_are_not_dropped_silently():
    with forward_ad.dual_level():
        for call in calls(lambda t: forward_ad.make_dual(t, torch.ones_like(t))):
            with pytest.raises(ValueError, match="autograd"):
                call()
            with torch.no_grad(), pytest.raises(ValueError, match="autograd"):       # which forward mode does not heed
                call()


def test_gradients_in_reverse_mode_are_not_dropped_silently():
    for call in calls(lambda t: t.clone().requires_grad_()):
        with pytest.raises(ValueError, match="autograd"):
            call()


def test_a_function_with_a_jvp_may_call():
    class Twice(torch.autograd.Function):
        @staticmethod
        def forward(x):
            replay._no_autograd(x)
            return 2 * x

        @staticmethod
        def setup_context(ctx, inputs, output):
            pass

        @staticmethod
        def jvp(ctx, t):
            return 2 * t

    with forward_ad.dual_level():
        y = Twice.apply(forward_ad.make_dual(torch.ones(3), torch.ones(3)))
        assert torch.equal(forward_ad.unpack_dual(y).tangent, torch.full((3,), 2.0))
