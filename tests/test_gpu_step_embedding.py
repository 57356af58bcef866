"""Token embedding and its gradient against the definition in 64 bits."""
import math

import pytest
import torch

import step_defn as defn

pytestmark = pytest.mark.gpu
BF, H, F = torch.bfloat16, torch.float16, torch.float32


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


@pytest.mark.parametrize("dtype,out", [(BF, BF), (BF, F), (H, H), (H, F), (F, F)])
@pytest.mark.parametrize("rows,dim,vocab,id_dtype", [((1,), 64, 10, torch.int64), ((2, 7), 1001, 333, torch.int32), ((129,), 8, 70000, torch.int64),
                                                     ((0,), 16, 5, torch.int64), ((5,), 4096, 2, torch.int32), ((3,), 1, 4, torch.int64)])
def test_lookup(rows, dim, vocab, id_dtype, dtype, out):
    from paper_2608_11034_b200 import step
    g = gen(1)
    table = torch.randn(vocab, dim, generator=g, device="cuda").to(dtype)
    ids = torch.randint(-2, vocab + 2, rows, generator=g, device="cuda").to(id_dtype)
    y = step.embedding_forward(ids, table, scale=1.7, out_dtype=out)
    live = (ids >= 0) & (ids < vocab)
    want = table.double()[ids.clamp(0, vocab - 1).long()] * float(torch.tensor(1.7)) * live[..., None]
    assert y.shape == (*rows, dim) and y.dtype == out
    assert defn.within(y, want, (2.0 ** -24 + defn.U[out]) * want.abs() + defn.TINY[out]) <= 1
    # a table whose rows lie apart and off 16-byte boundaries gives the same bits
    wide = torch.full((vocab, dim + 3), math.nan, dtype=dtype, device="cuda")
    wide[:, 1:dim + 1] = table
    assert torch.equal(step.embedding_forward(ids, wide[:, 1:dim + 1], scale=1.7, out_dtype=out), y)


def tokens(kind, rows, vocab, g):
    if kind == "spread":
        return torch.randint(-1, vocab + 1, (rows,), generator=g, device="cuda")
    if kind == "one":                                  # the same id everywhere
        return torch.full((rows,), vocab // 2, device="cuda")
    if kind == "none":
        return torch.full((rows,), -1, device="cuda")
    if kind == "few":                                  # runs that cross many pieces
        return torch.randint(0, min(vocab, 3), (rows,), generator=g, device="cuda")
    return torch.arange(rows, device="cuda").flip(0) % vocab      # every id in turn, backwards


@pytest.mark.parametrize("dtype,out", [(BF, F), (BF, BF), (H, H), (F, F)])
@pytest.mark.parametrize("kind", ["spread", "one", "none", "few", "turn"])
@pytest.mark.parametrize("rows,dim,vocab", [(1, 64, 10), (31, 8, 5), (32, 24, 700), (33, 1001, 3), (1000, 40, 50257), (5000, 136, 600), (70001, 8, 1)])
def test_gradient(rows, dim, vocab, kind, dtype, out):
    from paper_2608_11034_b200 import step
    g = gen(rows + dim)
    ids = tokens(kind, rows, vocab, g)
    dy = torch.randn(rows, dim, generator=g, device="cuda").to(dtype)
    dy[(ids < 0) | (ids >= vocab)] = math.nan           # padding's gradient is not read
    scale = 0.125
    want, bound = defn.embedding_gradient(dy, ids, vocab, scale, out)
    got = step.embedding_backward(dy, ids, vocab, scale=scale, out_dtype=out)
    assert got.dtype == out and defn.within(got, want, bound) <= 1
    assert torch.equal(step.embedding_backward(dy, ids.int(), vocab, scale=scale, out_dtype=out), got)      # the same bits again
    # added to what is there; rows without a token, and what lies between rows, stay as they are
    room = torch.randn(vocab, dim + 5, generator=g, device="cuda").to(out)
    was = room.clone()
    assert step.embedding_backward(dy, ids, vocab, scale=scale, grad=room[:, 2:dim + 2]).data_ptr() == room[:, 2:].data_ptr()
    want, bound = defn.embedding_gradient(dy, ids, vocab, scale, out, was[:, 2:dim + 2])
    assert defn.within(room[:, 2:dim + 2], want, bound) <= 1
    idle = torch.ones(vocab, dtype=torch.bool, device="cuda")
    idle[ids[(ids >= 0) & (ids < vocab)].long()] = False
    assert torch.equal(room[idle], was[idle]) and torch.equal(room[:, :2], was[:, :2]) and torch.equal(room[:, dim + 2:], was[:, dim + 2:])


def test_gradient_of_strided_and_shaped_gradients():
    from paper_2608_11034_b200 import step
    g = gen(5)
    ids = torch.randint(0, 50, (4, 9), generator=g, device="cuda")
    dy = torch.randn(4, 9, 72, generator=g, device="cuda").to(BF)
    want = step.embedding_backward(dy, ids, 50)
    wide = torch.full((36, 75), math.nan, dtype=BF, device="cuda")
    wide[:, 3:] = dy.view(36, 72)
    assert torch.equal(step.embedding_backward(wide[:, 3:], ids.view(36), 50), want)
    assert torch.equal(step.embedding_backward(dy.transpose(0, 1).contiguous().transpose(0, 1), ids, 50), want)
    assert torch.equal(step.embedding_backward(dy, ids.t().contiguous().t(), 50), want)
    assert (step.embedding_backward(dy[:0], ids[:0], 50) == 0).all()


def test_a_nan_reaches_its_own_row_alone():
    from paper_2608_11034_b200 import step
    ids = torch.randint(0, 20, (500,), generator=gen(6), device="cuda")
    dy = torch.randn(500, 64, generator=gen(7), device="cuda")
    dy[123, 5] = math.nan
    got = step.embedding_backward(dy, ids, 20)
    bad = torch.zeros(20, 64, dtype=torch.bool, device="cuda")
    bad[ids[123], 5] = True
    assert torch.equal(got.isnan(), bad)


def test_captured_and_on_another_stream():
    from paper_2608_11034_b200 import step
    g = gen(8)
    ids = torch.randint(0, 900, (3000,), generator=g, device="cuda")
    table, dy = (torch.randn(n, 128, generator=g, device="cuda").to(BF) for n in (900, 3000))
    step.embedding_backward(dy, ids, 900)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y, dw = step.embedding_forward(ids, table), step.embedding_backward(dy, ids, 900)
    for seed in (9, 10):
        ids.copy_(torch.randint(0, 900, (3000,), generator=gen(seed), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, table[ids]) and torch.equal(dw, step.embedding_backward(dy, ids, 900))


def test_refusals():
    from paper_2608_11034_b200 import step
    table, ids = torch.zeros(10, 8, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    dy = torch.zeros(4, 8, device="cuda")
    for bad in (lambda: step.embedding_forward(ids.float(), table), lambda: step.embedding_forward(ids, table.double()),
                lambda: step.embedding_forward(ids, table, out_dtype=BF), lambda: step.embedding_forward(ids.cpu(), table),
                lambda: step.embedding_forward(ids, table.t()), lambda: step.embedding_forward(ids, table, scale=math.inf),
                lambda: step.embedding_forward(ids, table.requires_grad_()), lambda: step.embedding_backward(dy[:3], ids, 10),
                lambda: step.embedding_backward(dy, ids, 10, out_dtype=BF), lambda: step.embedding_backward(dy, ids, -1),
                lambda: step.embedding_backward(dy, ids, 10, grad=torch.zeros(9, 8, device="cuda")),
                lambda: step.embedding_backward(dy.to(BF), ids, 10, grad=torch.zeros(10, 8, device="cuda"), out_dtype=BF),
                lambda: step.embedding_backward(dy.to(BF), ids, 10, grad=torch.zeros(10, 8, device="cuda").half())):
        with pytest.raises(ValueError):
            bad()
