"""Cross entropy over a vocabulary and its gradients against the definition in 64 bits."""
import math

import pytest
import torch

import step_defn as defn

pytestmark = pytest.mark.gpu
BF, H, F = torch.bfloat16, torch.float16, torch.float32


def inputs(rows, dim, vocab, dtype, seed=0, padding=0.0, lean=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = (torch.randn(vocab, dim, generator=g, device="cuda") * dim ** -0.5).to(dtype)
    targets = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    x = torch.randn(rows, dim, generator=g, device="cuda")
    if lean:
        x += torch.rand(rows, 1, generator=g, device="cuda") * 8 * w[targets].float()
    x = x.to(dtype)
    out = torch.rand(rows, generator=g, device="cuda") < padding
    targets[out] = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.5, -1, vocab)[out]
    x[out] = math.nan                                # what stands in padding reaches nothing
    return x, w, targets, torch.randn(rows, generator=g, device="cuda") * 1e-3


def check(x, w, targets, dloss, out=None):
    from paper_2608_11034_b200 import step
    r = defn.loss(torch.nan_to_num(x, 0.0), w, targets, dloss)
    loss, lse = step.loss_forward(x, w, targets)
    assert defn.within(lse, r["lse"], r["b_lse"]) <= 1 and defn.within(loss, r["loss"], r["b_loss"]) <= 1
    out = out or w.dtype
    dx, dw = step.loss_backward(x, w, targets, lse, dloss, out_dtype=out)
    assert dx.dtype == x.dtype and defn.within(dx, r["dx"], r["b_dx"]) <= 1
    assert dw.dtype == out and defn.within(dw, r["dw"], r["b_dw"] + defn.U[out] * r["dw"].abs() + defn.TINY[out]) <= 1
    # the same bits again, with ids of the other type
    again = step.loss_forward(x, w, targets.int())
    assert torch.equal(again[0], loss) and torch.equal(again[1], lse)
    assert all(torch.equal(a, b) for a, b in zip((dx, dw), step.loss_backward(x, w, targets.int(), lse, dloss, out_dtype=out)))
    return loss, lse, dx, dw


@pytest.mark.parametrize("dtype", [BF, H])
@pytest.mark.parametrize("rows,dim,vocab", [(1, 8, 1), (1, 64, 1000), (5, 72, 255), (127, 1024, 257), (128, 256, 512), (129, 1032, 130), (300, 520, 5003),
                                            (1000, 64, 777), (2, 4096, 20000), (700, 2056, 300)])
def test_sizes(rows, dim, vocab, dtype):
    check(*inputs(rows, dim, vocab, dtype))


@pytest.mark.parametrize("padding", [0.3, 0.99, 1.0])
@pytest.mark.parametrize("rows,dim,vocab", [(1, 64, 100), (257, 136, 1500), (3000, 64, 600)])
def test_padding_counts_for_nothing(rows, dim, vocab, padding):
    x, w, targets, dloss = inputs(rows, dim, vocab, BF, padding=padding)
    loss, lse, dx, dw = check(x, w, targets, dloss, F)
    out = (targets < 0) | (targets >= vocab)
    assert (loss[out] == 0).all() and (lse[out] == 0).all() and (dx[out] == 0).all() and (out.all() <= (dw == 0).all())


def test_one_number_for_all_rows_and_rows_that_lie_apart():
    from paper_2608_11034_b200 import step
    x, w, targets, _ = inputs(200, 264, 900, BF)
    one = torch.tensor(1 / 197.0, device="cuda")
    loss, lse, dx, dw = check(x, w, targets, one.expand(200))
    assert all(torch.equal(a, b) for a, b in zip((dx, dw), step.loss_backward(x, w, targets, lse, one.repeat(200), out_dtype=BF)))
    wide = torch.full((200, 264 + 3), math.nan, dtype=BF, device="cuda")
    wide[:, 1:265] = x
    table = torch.full((900, 264 + 8), math.nan, dtype=BF, device="cuda")
    table[:, :264] = w
    got = step.loss_forward(wide[:, 1:265], table[:, :264], targets)
    assert torch.equal(got[0], loss) and torch.equal(got[1], lse)
    room = torch.full((900, 264 + 11), 3.0, device="cuda")
    dx2, _ = step.loss_backward(wide[:, 1:265], table[:, :264], targets, lse, one.expand(200), grad=room[:, 5:269])
    r = defn.loss(x, w, targets, one.expand(200))
    assert torch.equal(dx2, dx) and defn.within(room[:, 5:269], r["dw"] + 3.0, r["b_dw"] + 2.0 ** -22) <= 1
    assert (room[:, :5] == 3.0).all() and (room[:, 269:] == 3.0).all()
    half = torch.full((900, 264), 3.0, dtype=BF, device="cuda")
    step.loss_backward(x, w, targets, lse, one.expand(200), grad=half)
    assert defn.within(half, r["dw"] + 3.0, r["b_dw"] + 2.0 ** -22 + defn.U[BF] * 3.1) <= 1


def test_gradients_are_what_differences_say():
    """Of the sum of the losses with weights; the loss is exact to 2^-20 or so, of which a step of 2^-3 leaves 2^-16 in a slope, and the
    third derivative of a log-sum-exp along a row of w, below |w_i|^3 / 2, puts 2^-8 |w_i|^3 into it."""
    from paper_2608_11034_b200 import step
    x, w, targets, dloss = inputs(6, 64, 50, BF, seed=3)
    dloss = dloss * 1000
    _, lse = step.loss_forward(x, w, targets)
    dx, dw = step.loss_backward(x, w, targets, lse, dloss)
    for t, grad, places in ((x, dx, (0, 70, 383)), (w, dw, (1, 64 * int(targets[2]) + 5, 3199))):
        for at in places:
            ends, steps = [], []
            for sign in (1, -1):
                moved = t.clone()
                moved.view(-1)[at] += sign * 0.125
                steps.append(float(moved.view(-1)[at]))
                loss, _ = step.loss_forward(*((moved, w) if t is x else (x, moved)), targets)
                ends.append(float((loss.double() * dloss.double()).sum()))
            slope = (ends[0] - ends[1]) / (steps[0] - steps[1])
            assert abs(slope - float(grad.reshape(-1)[at])) <= 2.0 ** -6 * (float(dloss.abs().sum()) + abs(slope))


def test_large_scores_infinities_and_nan():
    from paper_2608_11034_b200 import step
    x, w, targets, dloss = inputs(140, 64, 300, BF)
    x[3] *= 2.0 ** 7                                  # scores of some hundreds: the exponentials stay in range
    x[7, 5] = math.nan
    x[9, 1] = math.inf
    loss, lse = step.loss_forward(x, w, targets)
    ok = torch.ones(140, dtype=torch.bool, device="cuda")
    ok[[7, 9]] = False
    r = defn.loss(x[ok], w, targets[ok])
    assert defn.within(loss[ok], r["loss"], r["b_loss"]) <= 1 and defn.within(lse[ok], r["lse"], r["b_lse"]) <= 1
    assert loss[7].isnan() and not torch.isfinite(loss[9])
    dx, dw = step.loss_backward(x, w, targets, lse, dloss)
    assert torch.isfinite(dx[ok]).all() and dx[7].isnan().all() and dw.isnan().all()


def test_a_vocabulary_in_pieces():
    """So many rows that G of the whole vocabulary exceeds a piece: the pieces' sums meet in dx."""
    from paper_2608_11034_b200 import binding, step
    rows, dim, vocab = 33000, 64, 17000
    f, b = binding.scout_loss_workspace(binding.DT_BF16, rows, dim, vocab)
    assert b < rows * vocab * 2
    x, w, targets, dloss = inputs(rows, dim, vocab, BF, padding=0.1)
    loss, lse = step.loss_forward(x, w, targets)
    dx, dw = step.loss_backward(x, w, targets, lse, dloss, out_dtype=BF)
    want = torch.zeros(vocab, dim, dtype=torch.float64, device="cuda")
    bound = torch.zeros_like(want)
    for part in torch.arange(rows, device="cuda").split(4000):
        r = defn.loss(torch.nan_to_num(x[part], 0.0), w, targets[part], dloss[part])
        assert defn.within(loss[part], r["loss"], r["b_loss"]) <= 1 and defn.within(dx[part], r["dx"], r["b_dx"]) <= 1
        want += r["dw"]
        bound += r["b_dw"]
    assert defn.within(dw, want, bound + defn.U[BF] * want.abs()) <= 1


def test_no_rows_and_no_vocabulary():
    from paper_2608_11034_b200 import step
    x, w, targets, dloss = inputs(4, 64, 10, BF)
    loss, lse = step.loss_forward(x[:0], w, targets[:0])
    dx, dw = step.loss_backward(x[:0], w, targets[:0], lse, dloss[:0])
    assert loss.shape == (0,) and dx.shape == (0, 64) and (dw == 0).all()
    loss, lse = step.loss_forward(x, w[:0], targets)
    dx, dw = step.loss_backward(x, w[:0], targets, lse, dloss)
    assert (loss == 0).all() and (lse == 0).all() and (dx == 0).all() and dw.shape == (0, 64)


def test_captured_and_waits():
    from paper_2608_11034_b200 import binding, step
    x, w, targets, dloss = inputs(500, 128, 2000, BF, padding=0.2)

    def both():
        loss, lse = step.loss_forward(x, w, targets)
        return (loss, lse, *step.loss_backward(x, w, targets, lse, dloss))

    before = binding.scout_replay_waits()
    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for _ in range(2):
        targets.copy_(torch.where(torch.rand(500, device="cuda") < 0.5, targets.clamp(0, 1999), -1))    # fewer rows count from now on
        torch.nan_to_num(x, 0.5, out=x)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, both()))
    assert binding.scout_replay_waits() == before


def test_refusals():
    from paper_2608_11034_b200 import binding, step
    x, w, targets, dloss = inputs(6, 64, 10, BF)
    _, lse = step.loss_forward(x, w, targets)
    for bad in (lambda: step.loss_forward(x.float(), w.float(), targets), lambda: step.loss_forward(x, w.half(), targets),
                lambda: step.loss_forward(x[:, :56], w, targets), lambda: step.loss_forward(x, w, targets[:5]),
                lambda: step.loss_forward(x, w, targets.float()), lambda: step.loss_forward(x, w, targets.cpu()),
                lambda: step.loss_forward(x, w.t(), targets), lambda: step.loss_forward(x[0], w, targets),
                lambda: step.loss_forward(x.clone().requires_grad_(), w, targets), lambda: step.loss_backward(x, w, targets, lse[:5], dloss),
                lambda: step.loss_backward(x, w, targets, lse, dloss.double()), lambda: step.loss_backward(x, w, targets, lse, dloss, out_dtype=H),
                lambda: step.loss_backward(x, w, targets, lse, dloss, grad=torch.zeros(9, 64, device="cuda")),
                lambda: step.loss_backward(x, w, targets, lse, dloss, grad=torch.zeros(10, 64, device="cuda"), out_dtype=BF)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(binding.ScoutError) as e:                       # a row of w off 16-byte boundaries
        step.loss_forward(x, torch.zeros(10, 67, dtype=BF, device="cuda")[:, :64], targets)
    assert e.value.code == binding.ERR_ALIGN
    with pytest.raises(binding.ScoutError) as e:
        step.loss_forward(x[:, :60], w[:, :60], targets)
    assert e.value.code == binding.ERR_UNSUPPORTED
