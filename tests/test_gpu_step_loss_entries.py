"""Entries of the cross entropy that are made more exactly than the others, on inputs that show them alone."""
import math

import pytest
import torch

import step_defn as defn

pytestmark = pytest.mark.gpu
BF, H, F = torch.bfloat16, torch.float16, torch.float32
DIM = 1024


def truncated(dtype, score, rows, vocab):
    """x, w, targets: all rows alike, target 1, of which the exact score is `score` + 992 * 3 * 2^-16 (None: 2^13 instead of `score`), and all
    other scores 0.  The target's score has 2^13 as its first term, beside which the tensor cores lose what they add afterwards, less than
    2^-10 in 16 columns; they lose that of 48 to 64 times 16 columns.  In fp32 the warp adds it exactly: the lane that has columns 0 to 7 of
    each 256 has no small terms, the other lanes no large one."""
    x, w = torch.zeros(DIM, dtype=torch.float64), torch.zeros(DIM, dtype=torch.float64)
    c = torch.arange(DIM)
    small = (c // 8) % 32 != 0
    x[small], w[small] = 0.75 * 2.0 ** -7, 2.0 ** -7
    x[0], w[0] = 2.0 ** 7, 2.0 ** 6
    if score is not None:
        x[768], w[768] = -2.0 ** 7, 2.0 ** 6
        x[769], w[769] = 1.0, score
    table = torch.zeros(vocab, DIM, dtype=dtype, device="cuda")
    table[1] = w.to(dtype)
    exact = float((x * w).sum())
    assert exact == (2.0 ** 13 if score is None else score) + 992 * 3 * 2.0 ** -16
    return x.to(dtype).cuda().repeat(rows, 1), table, torch.ones(rows, dtype=torch.int64, device="cuda"), exact


@pytest.mark.parametrize("dtype", [BF, H])
@pytest.mark.parametrize("rows", [1, 70])
def test_a_sure_row_of_large_scores_loses_nothing(rows, dtype):
    """lse is the score here, and all that may part them is the rounding of either to fp32: half of 2^-10 around 2^13."""
    from paper_2608_11034_b200 import step
    x, w, targets, _ = truncated(dtype, None, rows, 300)
    loss, lse = step.loss_forward(x, w, targets)
    assert (loss.abs() <= 2.0 ** -11).all() and ((lse - 2.0 ** 13).abs() < 0.06).all()
    dx, _ = step.loss_backward(x, w, targets, lse, torch.ones(rows, device="cuda"))
    assert (dx.double().abs() <= 2.0 ** -10 * w[1].double().abs()).all()


@pytest.mark.parametrize("dtype", [BF, H])
@pytest.mark.parametrize("rows", [1, 70])
@pytest.mark.parametrize("score", [-3.0, 0.5, 8.0, 10.0, 14.0])
def test_what_the_tensor_cores_lose_of_a_targets_score(score, rows, dtype):
    """The score itself is exact in fp32 (multiples of 2^-16 below 2^6 once the large terms have met).  lse: exponentials and their sum
    are off by 2^-20 relative (2^-22 each, and as much for an argument of up to 2^4 that is rounded to fp32), and it is rounded to fp32."""
    from paper_2608_11034_b200 import step
    vocab = 20000
    x, w, targets, exact = truncated(dtype, score, rows, vocab)
    want = math.log(vocab - 1 + math.exp(exact))
    loss, lse = step.loss_forward(x, w, targets)
    off = 2.0 ** -20 + 2.0 ** -23 * abs(want)
    assert float((lse.double() - want).abs().max()) <= off
    assert float((loss.double() - (want - exact)).abs().max()) <= off + 2.0 ** -23 * abs(want - exact)


@pytest.mark.parametrize("rows", [1, 70])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_is_no_number_in_another_row_of_w(bad, rows):
    """A score that is NaN or Inf makes lse that; one of -Inf counts for nothing."""
    from paper_2608_11034_b200 import step
    x, w, targets, exact = truncated(BF, 8.0, rows, 2000)
    w[7, 9] = bad
    loss, lse = step.loss_forward(x, w, targets)
    if bad == -math.inf:
        assert ((lse - math.log(1998 + math.exp(exact))).abs() <= 2.0 ** -17).all()
    else:
        assert (lse.isnan() if bad != bad else lse == bad).all() and (loss.isnan() if bad != bad else loss == bad).all()


def half_step(x, dtype):
    """Half of the distance between numbers of this type around x."""
    return torch.exp2(torch.floor(torch.log2(x.abs()))) * defn.U[dtype]


@pytest.mark.parametrize("dtype", [BF, H])
@pytest.mark.parametrize("rows,count", [(1, 1), (64, 64), (65, 65), (100, 64), (100, 65), (300, 300), (1100, 1100)])
@pytest.mark.parametrize("tokens", [1, 2, 3, 100, 2000])
def test_the_gradient_at_a_target_is_not_rounded_to_16_bits(tokens, rows, count, dtype):
    """Row t alone has a number in column 64 + t of x, and its target alone in that of w: dx there is G at the target times w, dw is that
    times x, and the others' rounding does not reach them.  G at the target, g (p - 1), is off by what score and lse are off times g p, and
    by 2^-20 relative for expm1 and the products; 16 bits would be off by up to 2^-8 or 2^-11, which dw is at those of a target's
    tokens that come after two others."""
    from paper_2608_11034_b200 import step
    g = torch.Generator(device="cuda").manual_seed(rows + count)

    def rand(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    vocab, wide = 1500, 64 + -(-rows // 8) * 8
    x, w = torch.zeros(rows, wide, device="cuda"), torch.zeros(vocab, wide, device="cuda")
    x[:, :64] = torch.randn(rows, 64, generator=g, device="cuda")
    w[:, :64] = torch.randn(vocab, 64, generator=g, device="cuda") / 8
    t = torch.arange(rows, device="cuda")
    targets = torch.randperm(vocab, generator=g, device="cuda")[:rows]
    targets = targets[t // tokens]
    x[t, 64 + t], w[targets, 64 + t] = 0.5 + rand(rows), 0.5 + rand(rows)
    x, w = x.to(dtype), w.to(dtype)
    out = torch.randperm(rows, generator=g, device="cuda")[count:]
    dloss = 0.5 + rand(rows)
    marked = targets.clone()
    marked[out] = -1
    loss, lse = step.loss_forward(x, w, marked)
    r = defn.loss(x, w, marked)
    live = (marked >= 0).nonzero()[:, 0]
    t, v = t[live], targets[live]
    xd, wd = x.double(), w.double()
    p = torch.exp((xd[t] * wd[v]).sum(1) - r["lse"][t])
    at = dloss[t].double() * (p - 1)
    moved = r["b_lse"][t] + 24 * 2.0 ** -24 * (xd[t] * wd[v]).abs().sum(1)
    off = 2.0 ** -20 + moved * p / (1 - p)
    held = torch.zeros(vocab, dtype=torch.int64, device="cuda").index_add_(0, v, torch.ones_like(v))        # tokens of a target

    def check(got, want, room):
        """Within `room`, or beyond two of a target also within the rounding of G."""
        wrong = (got.double() - want).abs() - room
        assert bool((wrong <= torch.where(held[v] > 2, defn.U[dtype] * want.abs(), 0.0)).all())
        good = torch.zeros_like(held).index_add_(0, v, (wrong <= 0).long())
        assert bool((good >= held.clamp(max=2)).all())

    for out_dtype in (F, dtype):
        dx, dw = step.loss_backward(x, w, marked, lse, dloss, out_dtype=out_dtype)
        want = at * wd[v, 64 + t]
        assert bool(((dx[t, 64 + t].double() - want).abs() <= half_step(want, dtype) + off * want.abs()).all())
        want = at * xd[t, 64 + t]
        check(dw[v, 64 + t], want, off * want.abs() + (0 if out_dtype == F else half_step(want, dtype)))
    was = torch.full_like(dw, 0.5, dtype=F)
    step.loss_backward(x, w, marked, lse, dloss, grad=was)
    check(was[v, 64 + t].double() - 0.5, want, off * want.abs() + 2.0 ** -23)


def test_rows_that_weigh_little_have_gradients_of_their_own():
    """float16, half of the rows weighing 2^-27 of the others: their dx is as exact as if they were alone, and has the same bits whatever
    the others weigh."""
    from paper_2608_11034_b200 import step
    rows, dim, vocab = 200, 136, 1200
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(rows, dim, generator=g, device="cuda").to(H)
    w = (torch.randn(vocab, dim, generator=g, device="cuda") * dim ** -0.5).to(H)
    targets = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    _, lse = step.loss_forward(x, w, targets)
    light = torch.arange(rows, device="cuda") % 2 == 1
    dloss = torch.where(light, 2.0 ** -12, 2.0 ** 15) * (0.5 + torch.rand(rows, generator=g, device="cuda") / 2)
    dx, dw = step.loss_backward(x, w, targets, lse, dloss)
    r = defn.loss(x[light], w, targets[light], dloss[light])
    assert defn.within(dx[light], r["dx"], r["b_dx"]) <= 1
    r = defn.loss(x, w, targets, dloss)
    assert defn.within(dx, r["dx"], r["b_dx"]) <= 1 and defn.within(dw, r["dw"], r["b_dw"] + defn.U[F] * r["dw"].abs()) <= 1
    same, _ = step.loss_backward(x, w, targets, lse, torch.where(light, dloss, 2.0 ** -12))
    assert torch.equal(same[light], dx[light])


@pytest.mark.parametrize("rows", [40, 200])
@pytest.mark.parametrize("other", [0.0, -1.0, 2.0, math.inf, math.nan])
def test_rows_that_weigh_alike_and_one_that_does_not(other, rows):
    """float16: one number for all rows, or for all but the last."""
    from paper_2608_11034_b200 import step
    dim, vocab = 72, 700
    g = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn(rows, dim, generator=g, device="cuda").to(H)
    w = (torch.randn(vocab, dim, generator=g, device="cuda") * dim ** -0.5).to(H)
    targets = torch.randint(-50, vocab, (rows,), generator=g, device="cuda")
    targets[-1] = 5
    _, lse = step.loss_forward(x, w, targets)
    dloss = torch.ones(rows, device="cuda")
    dx, dw = step.loss_backward(x, w, targets, lse, dloss)
    r = defn.loss(x, w, targets, dloss)
    assert defn.within(dx, r["dx"], r["b_dx"]) <= 1 and defn.within(dw, r["dw"], r["b_dw"] + defn.U[F] * r["dw"].abs()) <= 1
    dloss[-1] = other
    mixed, dw = step.loss_backward(x, w, targets, lse, dloss)
    assert torch.equal(mixed[:-1], dx[:-1])
    if math.isfinite(other):
        r = defn.loss(x, w, targets, dloss)
        assert defn.within(mixed, r["dx"], r["b_dx"]) <= 1 and defn.within(dw, r["dw"], r["b_dw"] + defn.U[F] * r["dw"].abs()) <= 1
    else:
        assert not mixed[-1].isfinite().any() and not dw.isfinite().any()


def test_a_vocabulary_in_pieces_of_float16():
    """G is held in two forms there."""
    from paper_2608_11034_b200 import binding, step
    rows, dim, vocab = 33000, 64, 17000
    _, b = binding.scout_loss_workspace(binding.DT_F16, rows, dim, vocab)
    assert b < 2 * rows * vocab * 2
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn(rows, dim, generator=g, device="cuda").to(H)
    w = (torch.randn(vocab, dim, generator=g, device="cuda") / 8).to(H)
    targets = torch.randint(-100, vocab, (rows,), generator=g, device="cuda")
    dloss = torch.rand(rows, generator=g, device="cuda")
    _, lse = step.loss_forward(x, w, targets)
    dx, dw = step.loss_backward(x, w, targets, lse, dloss)
    want, bound = (torch.zeros(vocab, dim, dtype=torch.float64, device="cuda") for _ in range(2))
    for part in torch.arange(rows, device="cuda").split(4000):
        r = defn.loss(x[part], w, targets[part], dloss[part])
        assert defn.within(dx[part], r["dx"], r["b_dx"]) <= 1
        want += r["dw"]
        bound += r["b_dw"]
    assert defn.within(dw, want, bound + defn.U[F] * want.abs()) <= 1
