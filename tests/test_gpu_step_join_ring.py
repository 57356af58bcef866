"""Rows of up to 512 columns, which a team of one warp takes through a ring in shared memory: so many rows that every place of the ring
is filled again many times, against the kernels that hold rows in registers (which the same values take where they lie off
16-byte boundaries) bit for bit."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, H, F = torch.bfloat16, torch.float16, torch.float32


@pytest.mark.parametrize("tb,ts,tw", [(BF, BF, BF), (H, F, F), (F, F, F)])
@pytest.mark.parametrize("dim", [8, 256, 264, 504, 512])
def test_places_are_filled_again(dim, tb, ts, tw):
    from paper_2608_11034_b200 import step
    rows, g = 30011, torch.Generator(device="cuda").manual_seed(dim)

    def normal(*shape, dtype):
        return torch.randn(*shape, generator=g, device="cuda").to(dtype)

    def off(t):
        room = torch.zeros(rows, dim + 1, dtype=t.dtype, device="cuda")
        room[:, 1:] = t
        return room[:, 1:]

    x, dy = normal(rows, dim, dtype=ts), normal(rows, dim, dtype=ts)
    block, dn = normal(rows, dim, dtype=tb), normal(rows, dim, dtype=tb)
    gate, post, norm = (normal(dim, dtype=tw) for _ in range(3))

    def both(x, block, dy, dn):
        how = dict(gate=gate, post_weight=post, norm_weight=norm, scale=0.7, p=0.1, seed=5, offset=6)
        y, n, stats = step.join_forward(x, block, **how)
        return (y, n, stats, *step.join_backward(dy, dn, block, y, stats, **how))

    want = both(off(x), off(block), off(dy), off(dn))
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(want, both(x, block, dy, dn)))
