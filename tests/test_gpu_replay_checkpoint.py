"""8-bit activation checkpoints and the weight gradient taken from them.  Packing and restoring are exact, so they are
held to equality; the gradient's bound is the rounding of the stored result plus the fp32 sums' (2^-24 per addition,
taken over all additions of a sum in the worst order: rows * 2^-24 of the terms' magnitudes, at least 2^-18)."""
import math

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


def activation(seed, rows, cols, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, cols, generator=g, device="cuda")
    x *= torch.exp2(torch.randint(-12, 8, (rows, 1), generator=g, device="cuda").float())
    return x.to(dtype)


def hold(x):
    """pack, compare with the definition, restore in every type"""
    from paper_2608_11034_b200 import replay
    codes, exps = replay.checkpoint_pack(x)
    c, e = defn.pack(x)
    assert exps.tolist() == e
    assert codes.tolist() == c
    want = defn.restore(codes, exps)
    for t in (F32, BF, HF):
        got = replay.checkpoint_unpack(codes, exps, t)
        assert torch.equal(torch.nan_to_num(got, nan=12345.0), torch.nan_to_num(want.to(t), nan=12345.0)), t
        assert torch.equal(got.isnan(), want.isnan())
    # exact in the source's type, and a checkpoint of the restored tensor stands for the same values
    back = replay.checkpoint_unpack(codes, exps, x.dtype)
    fine = ~back.isnan()
    assert torch.equal(back.double()[fine], want[fine])
    again = replay.checkpoint_unpack(*replay.checkpoint_pack(back), x.dtype)
    assert torch.equal(again[fine], back[fine]) and torch.equal(again.isnan(), back.isnan())
    return codes, exps, back


@pytest.mark.parametrize("dtype", [F32, BF, HF])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (3, 32), (2, 33), (5, 64), (7, 100), (1, 255), (4, 256), (3, 264), (2, 1000), (67, 24)])
def test_pack_and_restore(dtype, rows, cols):
    x = activation(rows * 1000 + cols, rows, cols, dtype)
    _, exps, back = hold(x)
    # never further than half a step
    step = torch.exp2(exps.double()).repeat_interleave(32, 1)[:, :cols]
    assert ((back.double() - x.double()).abs() <= step / 2).all()


@pytest.mark.parametrize("dtype", [F32, BF, HF])
def test_extreme_values(dtype):
    f = torch.finfo(dtype)
    tiny = {F32: 2.0 ** -149, BF: 2.0 ** -133, HF: 2.0 ** -24}[dtype]
    rows = [[0.0] * 40, [-0.0] * 40, [f.max, f.min] * 20, [f.max * 0.99, 1.0] * 20, [tiny, -tiny, 0.0, 3 * tiny] * 10,
            [f.tiny, -3 * f.tiny] * 20, [127.0, 126.5, 0.5, 1.5, 2.5, -0.5, -1.5, 63.5] * 5, [127.5, 128.0, 1.0, 3.0] * 10,
            [63.5, 64.0, -63.75, 0.25] * 10]
    hold(torch.tensor(rows, dtype=torch.float64).to(dtype).cuda())


@pytest.mark.parametrize("dtype", [F32, BF, HF])
def test_non_finite_elements_stay_where_they_are(dtype):
    x = activation(3, 4, 100, dtype)
    x[0, 5], x[0, 40], x[1, 99] = math.nan, math.inf, -math.inf
    x[2] = math.nan
    clean = torch.nan_to_num(x, 0.0, 0.0, 0.0)
    codes, exps, back = hold(x)
    c2, e2, _ = hold(clean)
    assert torch.equal(exps, e2)
    bad = ~torch.isfinite(x)
    assert torch.equal(back.isnan(), bad) and torch.equal(codes[~bad], c2[~bad])


@pytest.mark.parametrize("dtype", [F32, BF, HF])
@pytest.mark.parametrize("offset,cols,stride", [(0, 96, 96), (1, 96, 97), (3, 70, 75), (8, 64, 72), (4, 128, 132), (0, 200, 201)])
def test_any_stride_and_alignment(dtype, offset, cols, stride):
    """A view into a larger tensor, at every alignment: same checkpoint as of its copy, nothing outside touched."""
    from paper_2608_11034_b200 import binding, replay
    rows = 9
    x = activation(offset + cols, rows, cols, dtype)
    room = torch.full((offset + rows * stride,), 7.0, dtype=dtype, device="cuda")
    view = room[offset:].as_strided((rows, cols), (stride, 1), offset)
    view.copy_(x)
    codes, exps = replay.checkpoint_pack(x)
    got = replay.checkpoint_pack(view)
    assert torch.equal(got[0], codes) and torch.equal(got[1], exps)
    # codes and restored values written into strided views too
    crm = torch.full((offset + rows * stride,), 0x5A, dtype=torch.int8, device="cuda")
    cv = crm.as_strided((rows, cols), (stride, 1), offset)
    s = torch.cuda.current_stream().cuda_stream
    code = {F32: binding.DT_F32, BF: binding.DT_BF16, HF: binding.DT_F16}[dtype]
    erm = torch.full((rows * exps.shape[1] + 64,), 0x5A, dtype=torch.int8, device="cuda")
    binding.scout_ckpt_pack(code, rows, cols, view.data_ptr(), stride, cv.data_ptr(), stride, erm.data_ptr(), s)
    assert torch.equal(cv, codes) and torch.equal(erm[:exps.numel()].view_as(exps), exps) and (erm[exps.numel():] == 0x5A).all()
    crm.as_strided((rows, cols), (stride, 1), offset).fill_(0x5A)
    assert (crm == 0x5A).all()
    back = torch.full_like(room, 7.0)
    bv = back.as_strided((rows, cols), (stride, 1), offset)
    crm.as_strided((rows, cols), (stride, 1), offset).copy_(codes)
    binding.scout_ckpt_unpack(code, rows, cols, cv.data_ptr(), stride, exps.data_ptr(), bv.data_ptr(), stride, s)
    assert torch.equal(bv, replay.checkpoint_unpack(codes, exps, dtype))
    bv.fill_(7.0)
    assert (back == 7.0).all()


def test_nothing_to_pack():
    from paper_2608_11034_b200 import replay
    for shape in ((0, 5), (5, 0), (0, 0)):
        codes, exps = replay.checkpoint_pack(torch.empty(shape, device="cuda"))
        assert replay.checkpoint_unpack(codes, exps).shape == shape


def grad_bound(dy, x, want, out_dtype):
    mag = dy.double().abs().t() @ x.abs()
    u = defn.U.get(out_dtype, 2.0 ** -24)
    tiny = defn.TINY.get(out_dtype, 0.0)
    return mag * max(dy.shape[0] * 2.0 ** -24, 2.0 ** -18) + u * want.abs() + tiny


@pytest.mark.parametrize("dtype,out", [(BF, F32), (BF, BF), (HF, F32), (HF, HF)])
@pytest.mark.parametrize("rows,outs,ins", [(1, 1, 1), (1, 64, 64), (33, 40, 72), (64, 128, 256), (100, 130, 257), (259, 96, 520),
                                           (500, 257, 128), (1000, 8, 8), (3000, 136, 48), (31, 999, 33), (129, 384, 512),
                                           (64, 128, 64), (65, 136, 67), (1030, 200, 264), (2500, 128, 300), (2049, 520, 1000), (5000, 1000, 72), (20, 1100, 1000), (1, 2048, 520)])
def test_weight_gradient(dtype, out, rows, outs, ins):
    from paper_2608_11034_b200 import replay
    x = activation(rows + outs, rows, ins, dtype)
    dy = activation(rows + ins, rows, outs, dtype)
    codes, exps = replay.checkpoint_pack(x)
    xd = defn.restore(codes, exps)
    want = dy.double().t() @ xd
    got = replay.checkpoint_wgrad(dy, codes, exps, out_dtype=out)
    assert got.dtype == out
    bound = grad_bound(dy, xd, want, out)
    # a sum beyond float16's range is Inf, which of the two results being judged by itself
    over = lambda r, w: torch.isinf(r) & (w.abs() > torch.finfo(out).max)          # noqa: E731
    assert (((got.double() - want).abs() <= bound) | over(got, want)).all()
    assert torch.equal(got, replay.checkpoint_wgrad(dy, codes, exps, out_dtype=out))
    # added in place to a gradient that is a view with gaps
    room = torch.full((outs, ins + 3), 0.5, dtype=out, device="cuda")
    grad = room[:, :ins]
    assert replay.checkpoint_wgrad(dy, codes, exps, grad=grad) is grad
    u = defn.U.get(out, 2.0 ** -24)
    assert (((grad.double() - want - 0.5).abs() <= bound + u * (want + 0.5).abs()) | over(grad, want + 0.5)).all()
    assert (room[:, ins:] == 0.5).all()


@pytest.mark.parametrize("dtype", [BF, HF])
def test_weight_gradient_of_views_and_of_non_finite_activations(dtype):
    from paper_2608_11034_b200 import replay
    x, dy = activation(1, 70, 203, dtype), activation(2, 70, 131, dtype)
    x[3, 7] = math.nan
    codes, exps = replay.checkpoint_pack(x)
    xd = defn.restore(codes, exps)
    want = dy.double().t() @ xd
    room = torch.full((70, 140), math.nan, dtype=dtype, device="cuda")
    room[:, 5:136] = dy
    croom = torch.full((70, 260), -128, dtype=torch.int8, device="cuda")
    croom[:, 9:212] = codes
    got = replay.checkpoint_wgrad(room[:, 5:136], croom[:, 9:212], exps)
    cols = [c for c in range(203) if c != 7]
    assert got[:, 7].isnan().all()
    ok = torch.nan_to_num(xd)
    assert ((got.double() - want).abs() <= grad_bound(dy, ok, torch.nan_to_num(want), F32))[:, cols].all()


def test_long_sums_round_to_nearest():
    """Sums of one sign over many tokens: the error stays that of fp32 additions, not of a chain that truncates."""
    from paper_2608_11034_b200 import replay
    x, dy = activation(7, 16384, 128, BF).abs(), activation(8, 16384, 256, BF).abs()
    codes, exps = replay.checkpoint_pack(x)
    want = dy.double().t() @ defn.restore(codes, exps)
    got = replay.checkpoint_wgrad(dy, codes, exps).double()
    # 64 truncating steps of at most 2^-23 each in a chain, then 16 additions
    assert ((got - want).abs() <= want * (64 * 2.0 ** -23 + 16 * 2.0 ** -24)).all()


def test_no_tokens():
    from paper_2608_11034_b200 import replay
    codes, exps = replay.checkpoint_pack(torch.empty(0, 40, device="cuda"))
    dy = torch.empty(0, 24, dtype=BF, device="cuda")
    assert (replay.checkpoint_wgrad(dy, codes, exps) == 0).all()
    grad = torch.full((24, 40), 3.0, device="cuda")
    assert (replay.checkpoint_wgrad(dy, codes, exps, grad=grad) == 3.0).all()


def test_weight_gradient_against_differences():
    """d/dW of sum(dy * (x W^T)) along random directions: linear, so one difference is exact up to rounding."""
    from paper_2608_11034_b200 import replay
    x, dy = activation(5, 200, 96, BF), activation(6, 200, 64, BF)
    codes, exps = replay.checkpoint_pack(x)
    xd = defn.restore(codes, exps)
    got = replay.checkpoint_wgrad(dy, codes, exps).double()
    g = torch.Generator(device="cuda").manual_seed(1)
    w, step = (torch.randn(64, 96, generator=g, device="cuda", dtype=torch.float64) for _ in range(2))
    loss = lambda z: (dy.double() * (xd @ z.t())).sum().item()          # noqa: E731
    want = (loss(w + step) - loss(w - step)) / 2
    mag = (dy.double().abs().t() @ xd.abs() * step.abs()).sum().item()
    assert abs((got * step).sum().item() - want) <= 2.0 ** -18 * mag


def test_refusals():
    from paper_2608_11034_b200 import binding, replay
    x = activation(1, 8, 64, BF)
    codes, exps = replay.checkpoint_pack(x)
    dy = activation(2, 8, 16, BF)
    for f in [lambda: replay.checkpoint_pack(x.double()), lambda: replay.checkpoint_pack(x.cpu()), lambda: replay.checkpoint_pack(x[0]),
              lambda: replay.checkpoint_pack(x[:, ::2]), lambda: replay.checkpoint_unpack(codes, exps[:, :1]),
              lambda: replay.checkpoint_unpack(codes, exps, torch.float64), lambda: replay.checkpoint_unpack(codes.int(), exps),
              lambda: replay.checkpoint_wgrad(dy[:4], codes, exps), lambda: replay.checkpoint_wgrad(dy.float(), codes, exps),
              lambda: replay.checkpoint_wgrad(dy, codes, exps, out_dtype=HF),
              lambda: replay.checkpoint_wgrad(dy, codes, exps, grad=torch.zeros(16, 63, device="cuda"))]:
        with pytest.raises(ValueError):
            f()
    s = torch.cuda.current_stream().cuda_stream
    flat = torch.zeros(600, dtype=torch.uint8, device="cuda")
    with pytest.raises(binding.ScoutError) as e:
        binding.scout_ckpt_pack(binding.DT_BF16, 8, 32, flat.data_ptr() + 1, 32, codes.data_ptr(), 64, exps.data_ptr(), s)
    assert e.value.code == binding.ERR_ALIGN
    with pytest.raises(binding.ScoutError) as e:
        binding.scout_ckpt_pack(binding.DT_BF16, 8, 64, x.data_ptr(), 63, codes.data_ptr(), 64, exps.data_ptr(), s)
    assert e.value.code == binding.ERR_INVALID
