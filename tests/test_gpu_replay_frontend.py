"""What the torch front end of the replay operators refuses rather than doing something other than was asked for."""
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
