"""Table gradients of many ids and many tokens: vocabularies whose ids take three radix passes, that several blocks mark, or whose ids
and places no longer fit into one number, and more tokens than sorting threads hold in registers."""
import math

import pytest
import torch

import step_defn as defn

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


@pytest.mark.parametrize("rows,vocab", [(2048, 300000), (2049, 300000), (40000, 300000), (40000, 700), (3000, (1 << 20) + 37), (100, (1 << 21) - 2),
                                        (100, (1 << 21) - 1), (100, (1 << 21) + 5), (40000, (1 << 18) - 1), (40000, 1 << 18)])
@pytest.mark.parametrize("dtype,out", [(BF, F), (F, F), (BF, BF)])
def test_gradient(rows, vocab, dtype, out):
    from paper_2608_11034_b200 import step
    dim, g = 8, torch.Generator(device="cuda").manual_seed(rows)
    # a third anywhere, a third around the middle of the vocabulary and its last ids, a third on a few ids
    part = torch.randint(0, 3, (rows,), generator=g, device="cuda")
    anywhere = torch.randint(-1, vocab + 1, (rows,), generator=g, device="cuda")
    near = torch.randint(-3, 4, (rows,), generator=g, device="cuda") + torch.where(anywhere % 2 == 0, min(vocab // 2, 1 << 20), vocab - 2)
    few = torch.randint(0, 5, (rows,), generator=g, device="cuda") * (vocab // 5)
    ids = torch.where(part == 0, anywhere, torch.where(part == 1, near, few))
    dy = torch.randn(rows, dim, generator=g, device="cuda").to(dtype)
    dy[(ids < 0) | (ids >= vocab)] = math.nan
    want, bound = defn.embedding_gradient(dy, ids, vocab, 0.5, out)
    got = step.embedding_backward(dy, ids, vocab, scale=0.5, out_dtype=out)
    assert defn.within(got, want, bound) <= 1
    assert torch.equal(step.embedding_backward(dy, ids.int(), vocab, scale=0.5, out_dtype=out), got)
    was = torch.randn(vocab, dim, generator=g, device="cuda").to(out)
    total = step.embedding_backward(dy, ids, vocab, scale=0.5, grad=was.clone())
    want, bound = defn.embedding_gradient(dy, ids, vocab, 0.5, out, was)
    assert defn.within(total, want, bound) <= 1
    idle = torch.ones(vocab, dtype=torch.bool, device="cuda")
    idle[ids[(ids >= 0) & (ids < vocab)]] = False
    assert torch.equal(total[idle], was[idle])


def test_dropout_of_rows_of_odd_lengths_past_the_first_launch():
    """More elements than one launch takes as one long row: the next one goes on with its own rows."""
    from paper_2608_11034_b200 import step
    cols = 1001
    first = (1 << 33) // cols // 8 * 8                      # rows of the first launch
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("not enough free memory")
    x = torch.ones(first + 11, cols, dtype=BF, device="cuda")
    y = step.dropout(x, 0.5, seed=11, offset=12)
    for row in (0, first - 3, first + 8):
        assert torch.equal(y[row:row + 3].double(), defn.mask(3, cols, 0.5, 11, 12, row).cuda())
