"""Attention of the layer replay against its definition in 64 bits: sizes where tiles end, grouped heads, masks that
leave rows empty, padding and hidden places that hold NaN, strides, reproducibility, streams."""
import math

import pytest
import torch

import replay_defn as defn

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(autouse=True)
def no_wait_gives_up():
    yield
    from paper_2608_11034_b200 import binding
    assert binding.scout_replay_error() == 0


def make(seed, dtype, B, Tq, Tk, Hq, Hk, D, scale_do=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)          # noqa: E731
    return n(B, Tq, Hq, D), n(B, Tk, Hk, D), n(B, Tk, Hk, D), (n(B, Tq, Hq, D).float() * scale_do).to(dtype)


def lens(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def close(got, want, bound, name):
    assert got.shape == want.shape
    err = (got.double() - want).abs()
    assert torch.isfinite(got).all(), f"{name}: not finite"
    worst = (err - bound).max().item() if err.numel() else -1.0
    assert worst <= 0, f"{name}: off by {err.max().item():.3g}, {worst:.3g} beyond its bound"


def check(q, k, v, do, **kw):
    from paper_2608_11034_b200 import replay
    o, lse = replay.attention_forward(q, k, v, **kw)
    want = defn.attention(q, k, v, do, **kw)
    close(o, want["o"], want["b_o"], "o")
    empty = torch.isinf(want["lse"])
    assert torch.equal(empty, torch.isinf(lse)) and (lse[empty] < 0).all()
    assert ((lse.double() - want["lse"])[~empty].abs() <= 1e-5 * (1 + want["lse"][~empty].abs())).all()
    dq, dk, dv = replay.attention_backward(q, k, v, o, lse, do, **kw)
    for name, got in (("dq", dq), ("dk", dk), ("dv", dv)):
        close(got, want[name], want["b_" + name], name)
    return o, lse, dq, dk, dv


SIZES = [  # B, Tq, Tk, Hq, Hk, D, causal, window
    (1, 1, 1, 1, 1, 64, False, 0),
    (2, 1, 777, 8, 2, 128, True, 0),
    (3, 5, 64, 4, 4, 64, False, 0),
    (2, 63, 65, 4, 2, 64, True, 0),
    (1, 64, 64, 3, 1, 128, True, 0),
    (2, 129, 129, 6, 2, 128, True, 0),
    (1, 200, 131, 2, 1, 64, True, 0),       # more rows than keys: the first 69 rows see nothing
    (2, 257, 300, 4, 1, 128, False, 0),
    (1, 333, 333, 5, 5, 80, True, 0),
    (2, 130, 130, 2, 2, 8, True, 0),
    (1, 96, 300, 4, 2, 120, True, 1),       # a row sees its own position alone
    (2, 300, 300, 4, 2, 64, True, 50),
    (1, 520, 520, 2, 1, 128, True, 128),
    (1, 7, 4000, 4, 1, 96, True, 0),
    (1, 2000, 9, 2, 2, 64, False, 0),       # few keys, many rows
    (1, 1100, 1100, 2, 1, 128, False, 0),
    (1, 3000, 3000, 1, 1, 64, True, 0),     # one head: its keys go in parts
    (2, 130, 2600, 1, 1, 128, False, 0),
]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_against_the_definition(size, dtype):
    B, Tq, Tk, Hq, Hk, D, causal, window = size
    check(*make(hash(size) & 0xFFFF, dtype, B, Tq, Tk, Hq, Hk, D), causal=causal, window=window)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_padded_sequences_and_empty_rows(dtype, D, causal):
    B, T, Hq, Hk = 5, 150, 4, 2
    q, k, v, do = make(11, dtype, B, T, T, Hq, Hk, D)
    ql, kl = lens(150, 64, 1, 0, 77), lens(150, 65, 140, 20, 0)
    for b in range(B):       # whatever stands in the padding must not matter
        q[b, int(ql[b]):] = math.nan
        do[b, int(ql[b]):] = math.inf
        k[b, int(kl[b]):] = math.nan
        v[b, int(kl[b]):] = -math.inf
    o, lse, dq, dk, dv = check(q, k, v, do, causal=causal, q_lens=ql, kv_lens=kl)
    for b in range(B):
        assert (o[b, int(ql[b]):] == 0).all() and (dq[b, int(ql[b]):] == 0).all()
        assert (dk[b, int(kl[b]):] == 0).all() and (dv[b, int(kl[b]):] == 0).all()
    assert (o[4] == 0).all() and (dk[3] == 0).all()


def test_lengths_outside_the_tensors_are_clamped():
    q, k, v, do = make(12, BF, 3, 70, 70, 2, 1, 64)
    check(q, k, v, do, causal=True, q_lens=lens(-5, 1000, 70), kv_lens=lens(3, 99999, -1))


def test_zero_tokens():
    from paper_2608_11034_b200 import replay
    q, k, v, do = make(13, BF, 2, 6, 6, 2, 1, 64)
    o, lse = replay.attention_forward(q, k[:, :0].contiguous(), v[:, :0].contiguous())
    assert (o == 0).all() and torch.isinf(lse).all()
    dq, dk, dv = replay.attention_backward(q, k[:, :0].contiguous(), v[:, :0].contiguous(), o, lse, do)
    assert (dq == 0).all() and dk.numel() == dv.numel() == 0
    e = q[:, :0].contiguous()
    o, lse = replay.attention_forward(e, k, v)
    assert o.numel() == lse.numel() == 0
    dq, dk, dv = replay.attention_backward(e, k, v, o, lse, e)
    assert dq.numel() == 0 and (dk == 0).all() and (dv == 0).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_what_a_row_does_not_see_never_reaches_it(D, value):
    """A non-finite token poisons the rows that see it and no others, also inside a tile."""
    from paper_2608_11034_b200 import replay
    B, T, Hq, Hk, at = 1, 300, 2, 1, 171
    q, k, v, do = make(14, BF, B, T, T, Hq, Hk, D)
    clean = defn.attention(q, k, v, do, causal=True)
    kb, vb = k.clone(), v.clone()
    vb[0, at] = value
    o, lse = replay.attention_forward(q, k, vb, causal=True)
    close(o[:, :at], clean["o"][:, :at], clean["b_o"][:, :at], "o before the bad value")
    assert not torch.isfinite(o[:, at:]).any()
    assert torch.isfinite(lse).all()
    kb[0, at] = value
    o, lse = replay.attention_forward(q, kb, v, causal=True)
    close(o[:, :at], clean["o"][:, :at], clean["b_o"][:, :at], "o before the bad key")
    # a gradient that no earlier key is hidden from poisons the keys its row sees: rows 0..at see keys 0..at
    gb = do.clone()
    gb[0, at] = value
    o, lse = replay.attention_forward(q, k, v, causal=True)
    dq, dk, dv = replay.attention_backward(q, k, v, o, lse, gb, causal=True)
    for got, name in ((dk, "dk"), (dv, "dv")):
        close(got[:, at + 1:], clean[name][:, at + 1:], clean["b_" + name][:, at + 1:], name + " after the bad row")
    assert not torch.isfinite(dv[:, :at + 1]).any()
    others = [i for i in range(T) if i != at]
    close(dq[:, others], clean["dq"][:, others], clean["b_dq"][:, others], "dq of the other rows")
    # keys hidden from a row
    dq, dk, dv = replay.attention_backward(q, kb, vb, o, lse, do, causal=True)
    close(dq[:, :at], clean["dq"][:, :at], clean["b_dq"][:, :at], "dq before the bad key")


def test_scores_far_apart_and_types_lowest_values():
    """Rows whose scores differ by thousands, and inputs at the type's lowest value in hidden places."""
    q, k, v, do = make(15, BF, 1, 140, 140, 2, 2, 64)
    q[0, 5] *= 1000
    k[0, 100] *= -100
    low = torch.finfo(BF).min
    k[0, 139], v[0, 139] = low, low
    check(q, k, v, do, causal=True, kv_lens=lens(139), q_lens=lens(139), scale=0.03125)


@pytest.mark.parametrize("layout", ["heads_first", "packed", "gaps"])
def test_strides(layout):
    from paper_2608_11034_b200 import replay
    B, T, Hq, Hk, D = 2, 131, 4, 2, 64
    q, k, v, do = make(16, BF, B, T, T, Hq, Hk, D)
    want = replay.attention_forward(q, k, v, causal=True) + replay.attention_backward(
        q, k, v, *replay.attention_forward(q, k, v, causal=True), do, causal=True)
    if layout == "heads_first":
        qs, ks, vs, gs = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (q, k, v, do))
    elif layout == "packed":     # one projection's output, queries, keys and values side by side
        both = torch.cat([x.reshape(B, T, -1) for x in (q, k, v)], -1)
        qs = both[..., :Hq * D].view(B, T, Hq, D)
        ks = both[..., Hq * D:(Hq + Hk) * D].view(B, T, Hk, D)
        vs = both[..., (Hq + Hk) * D:].view(B, T, Hk, D)
        gs = do
        o, lse = replay.attention_forward(qs, ks, vs, causal=True)
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
        with pytest.raises(ValueError):
            replay.attention_backward(qs, ks, vs, o, lse, gs, causal=True)
        return
    else:
        qs, ks, vs, gs = (torch.zeros(B, T, x.shape[2], D + 8, dtype=BF, device="cuda")[..., :D].copy_(x) for x in (q, k, v, do))
        o, lse = replay.attention_forward(qs, ks, vs, causal=True)
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
        return
    o, lse = replay.attention_forward(qs, ks, vs, causal=True)
    got = (o, lse) + replay.attention_backward(qs, ks, vs, o, lse, gs, causal=True)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("size", [(2, 700, 700, 8, 2, 128, True, 0), (1, 3, 5000, 4, 1, 128, True, 0), (1, 900, 900, 3, 3, 64, True, 100)], ids=str)
def test_same_bits_every_time_and_in_every_batch(size):
    """What consensus rests on: the same inputs give the same bits, run after run."""
    from paper_2608_11034_b200 import replay
    B, Tq, Tk, Hq, Hk, D, causal, window = size
    q, k, v, do = make(17, BF, B, Tq, Tk, Hq, Hk, D)
    first = None
    for _ in range(4):
        o, lse = replay.attention_forward(q, k, v, causal=causal, window=window)
        got = (o, lse) + replay.attention_backward(q, k, v, o, lse, do, causal=causal, window=window)
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(got, first))


def test_what_else_runs_does_not_show():
    """The same bits while another stream keeps memory and SMs busy: loads come late, blocks start late, warps fall behind."""
    import random
    from paper_2608_11034_b200 import replay
    rng, side, noise = random.Random(5), torch.cuda.Stream(), torch.empty(1 << 27, device="cuda")

    def run(q, k, v, do, causal):
        o, lse = replay.attention_forward(q, k, v, causal=causal)
        return (o, lse) + replay.attention_backward(q, k, v, o, lse, do, causal=causal)

    for _ in range(60):
        Hk, G, D, T = rng.choice([1, 2, 8]), rng.choice([1, 2, 4]), rng.choice([64, 128]), rng.randint(100, 1500)
        case = make(rng.randrange(1 << 16), BF, rng.randint(1, 3), T, T, Hk * G, Hk, D) + (rng.random() < 0.7,)
        want = run(*case)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(rng.randint(1, 6)):
                noise[:rng.randint(1 << 16, 1 << 27)].add_(1.0)
        for _ in range(3):
            assert all(torch.equal(a, b) for a, b in zip(run(*case), want))


def test_gradients_against_differences():
    """Directional derivatives of the definition's loss, by central differences in 64 bits."""
    from paper_2608_11034_b200 import replay
    kw = dict(causal=True, q_lens=lens(90, 40), kv_lens=lens(97, 40))
    q, k, v, do = make(18, HF, 2, 90, 97, 4, 2, 64)
    o, lse = replay.attention_forward(q, k, v, **kw)
    grads = replay.attention_backward(q, k, v, o, lse, do, **kw)
    g = torch.Generator(device="cuda").manual_seed(5)

    def loss(qd, kd, vd):
        total = 0.0
        for b in range(2):
            nq, nk = int(kw["q_lens"][b]), int(kw["kv_lens"][b])
            at = torch.arange(nq, device="cuda")[:, None] + nk - nq
            hide = torch.arange(nk, device="cuda")[None] > at
            for h in range(4):
                s = (qd[b, :nq, h] @ kd[b, :nk, h // 2].t() / 8.0).masked_fill(hide, -math.inf)
                total += ((torch.softmax(s, 1) @ vd[b, :nk, h // 2]) * do[b, :nq, h].double()).sum().item()
        return total

    x = [t.double() for t in (q, k, v)]
    for n in range(3):
        step = torch.randn(x[n].shape, generator=g, device="cuda", dtype=torch.float64)
        h = 1e-4
        up, down = list(x), list(x)
        up[n], down[n] = x[n] + h * step, x[n] - h * step
        want = (loss(*up) - loss(*down)) / (2 * h)
        got = (grads[n].double() * step).sum().item()
        # the gradient's elementwise error (about 2^-10 of its size) summed over random signs
        tol = 4 * 2.0 ** -10 * grads[n].double().norm().item() + 1e-4
        assert abs(got - want) <= tol, (n, got, want)


def test_outputs_stay_inside_their_buffers():
    """Every output and the scratch between guard bands, at sizes no tile divides."""
    import numpy as np
    from paper_2608_11034_b200 import binding
    B, Tq, Tk, Hq, Hk, D = 2, 77, 141, 6, 2, 72
    q, k, v, do = make(19, BF, B, Tq, Tk, Hq, Hk, D)
    a = np.zeros(1, dtype=binding.ATTN_DTYPE)
    st = [tuple(x.stride()[:3]) for x in (q, k, v, q, do)]
    a[0] = (binding.DT_BF16, B, Tq, Tk, Hq, Hk, D, 1, 0, 0.125) + tuple(st)
    fb, bb = binding.scout_attn_workspace(a.ctypes.data)
    bufs = []

    def band(nbytes):
        x = torch.full((nbytes + 1024,), 0x5A, dtype=torch.uint8, device="cuda")
        bufs.append((x, nbytes))
        return x.data_ptr() + 512

    o, lse = band(q.numel() * 2), band(B * Hq * Tq * 4)
    s = torch.cuda.current_stream().cuda_stream
    binding.scout_attn_forward(a.ctypes.data, q.data_ptr(), k.data_ptr(), v.data_ptr(), 0, 0, o, lse, band(fb) if fb else 0, fb, s)
    binding.scout_attn_backward(a.ctypes.data, q.data_ptr(), k.data_ptr(), v.data_ptr(), o, lse, do.data_ptr(), 0, 0,
                                band(q.numel() * 2), band(k.numel() * 2), band(v.numel() * 2), band(bb), bb, s)
    torch.cuda.synchronize()
    for x, n in bufs:
        assert bool((x[:512] == 0x5A).all()) and bool((x[512 + n:] == 0x5A).all())


def test_another_stream_and_a_graph():
    from paper_2608_11034_b200 import replay
    q, k, v, do = make(20, BF, 1, 260, 260, 4, 2, 128)
    o, lse = replay.attention_forward(q, k, v, causal=True)
    want = (o, lse) + replay.attention_backward(q, k, v, o, lse, do, causal=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        o2, lse2 = replay.attention_forward(q, k, v, causal=True)
        got = (o2, lse2) + replay.attention_backward(q, k, v, o2, lse2, do, causal=True)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o3, lse3 = replay.attention_forward(q, k, v, causal=True)
        got = (o3, lse3) + replay.attention_backward(q, k, v, o3, lse3, do, causal=True)
    for x in got:
        x.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_rows_beyond_32_bit_offsets():
    """A cache whose last tokens lie beyond 2^32 elements from its start."""
    from paper_2608_11034_b200 import replay
    T, D = 300, 64
    stride = (1 << 32) // (T - 100) // 8 * 8            # elements between tokens: token 201 starts beyond 2^32
    room = torch.empty((T - 1) * stride + D, dtype=BF, device="cuda")
    k = room.as_strided((1, T, 1, D), (room.numel() // 8 * 8, stride, D, 1))
    q, small, v, do = make(21, BF, 1, 40, T, 2, 1, D)
    k.copy_(small)
    assert (T - 1) * stride > 1 << 32
    o, lse = replay.attention_forward(q, k, v, causal=True)
    want = replay.attention_forward(q, small, v, causal=True)
    assert torch.equal(o, want[0]) and torch.equal(lse, want[1])


def test_refusals():
    from paper_2608_11034_b200 import binding, replay
    q, k, v, do = make(22, BF, 1, 16, 16, 4, 2, 64)
    o, lse = replay.attention_forward(q, k, v)
    bad = [lambda: replay.attention_forward(q.float(), k.float(), v.float()),
           lambda: replay.attention_forward(q, k.half(), v),
           lambda: replay.attention_forward(q, k, v[:, :8]),
           lambda: replay.attention_forward(q.cpu(), k.cpu(), v.cpu()),
           lambda: replay.attention_forward(q[..., ::2], k[..., ::2], v[..., ::2]),
           lambda: replay.attention_forward(q, k, v, q_lens=torch.zeros(1, device="cuda")),
           lambda: replay.attention_backward(q, k, v, o, lse[:, :, :8], do),
           lambda: replay.attention_backward(q, k, v, o, lse, do[:, :8])]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f, code in [(lambda: replay.attention_forward(q[:, :, :3], k, v), binding.ERR_INVALID),          # 3 heads on 2
                    (lambda: replay.attention_forward(q, k, v, window=4), binding.ERR_INVALID),           # window without causal
                    (lambda: replay.attention_forward(q, k, v, scale=0.0), binding.ERR_INVALID),
                    (lambda: replay.attention_forward(q, k, v, scale=math.nan), binding.ERR_INVALID),
                    (lambda: replay.attention_forward(q, k.expand(1, 16, 2, 64)[:, :, :1].expand(1, 16, 2, 64), v), binding.ERR_INVALID),
                    (lambda: replay.attention_forward(q[..., :12].contiguous(), k[..., :12].contiguous(), v[..., :12].contiguous()),
                     binding.ERR_UNSUPPORTED)]:
        with pytest.raises(binding.ScoutError) as e:
            f()
        assert e.value.code == code
    flat = torch.zeros(q.numel() + 8, dtype=BF, device="cuda")
    with pytest.raises(binding.ScoutError) as e:
        replay.attention_forward(flat[1:1 + q.numel()].view(q.shape), k, v)
    assert e.value.code == binding.ERR_ALIGN
