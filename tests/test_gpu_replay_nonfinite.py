"""NaN and Inf in what a row sees, at every place of a tile and in every kernel of attention: they reach the rows that see them.
Which kernel a call takes is a matter of its sizes: few rows, a tile of rows, whole tiles on tcgen05, with its keys in parts or not."""
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


def make(seed, dtype, B, Tq, Tk, Hq, Hk, D):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)          # noqa: E731
    return n(B, Tq, Hq, D), n(B, Tk, Hk, D), n(B, Tk, Hk, D), n(B, Tq, Hq, D)


KERNELS = {  # B, Tq, Tk, Hq, Hk
    "few": (1, 2, 400, 4, 2),
    "few_join": (1, 1, 3000, 2, 1),
    "tile": (1, 40, 300, 2, 1),
    "tile_parts": (1, 70, 900, 1, 1),
    "whole": (1, 260, 420, 2, 2),
    "whole_parts": (1, 200, 2600, 1, 1),
}


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("kernel", list(KERNELS))
def test_a_key_that_is_nan_poisons_the_rows_that_see_it(kernel, causal, D, dtype):
    """One NaN element in one key, its value finite; the key stands at each of 32 places in a row of a tile in turn."""
    from paper_2608_11034_b200 import replay
    B, Tq, Tk, Hq, Hk = KERNELS[kernel]
    q, k, v, _ = make(41, dtype, B, Tq, Tk, Hq, Hk, D)
    clean = defn.attention(q, k, v, causal=causal)
    for at in list(range(128, 160)) + [0, 5, Tk - 1]:
        bad = k.clone()
        bad[0, at, 0, at % D] = math.nan
        o, lse = replay.attention_forward(q, bad, v, causal=causal)
        first = max(0, at - (Tk - Tq)) if causal else 0
        heads = Hq // Hk                                      # those of the first key head
        assert o[0, first:, :heads].isnan().all() and lse[0, :heads, first:].isnan().all(), at
        assert ((o.double() - clean["o"]).abs() <= clean["b_o"])[0, :first].all(), at
        assert ((o.double() - clean["o"]).abs() <= clean["b_o"])[0, :, heads:].all(), at
        assert torch.isfinite(lse[0, :heads, :first]).all() and torch.isfinite(lse[0, heads:]).all(), at


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kernel", list(KERNELS))
def test_scores_that_are_all_minus_infinity_weigh_nothing(kernel, D, dtype):
    """All keys hold -Inf where the queries are positive: as if the row saw nothing.  One finite key among them has all the weight."""
    from paper_2608_11034_b200 import replay
    B, Tq, Tk, Hq, Hk = KERNELS[kernel]
    q, k, v, do = make(42, dtype, B, Tq, Tk, Hq, Hk, D)
    q[..., 3], k[..., 3] = 1.0, -math.inf
    o, lse = replay.attention_forward(q, k, v)
    assert (o == 0).all() and (lse == -math.inf).all()
    dv = replay.attention_backward(q, k, v, o, lse, do)[2]
    assert (dv == 0).all()
    for at in (0, 4, 134, Tk - 1):
        one = k.clone()
        one[:, at, :, 3] = 0.0
        o, lse = replay.attention_forward(q, one, v)
        assert torch.equal(o, v[:, at:at + 1].repeat_interleave(Hq // Hk, 2).expand_as(o))
        want = (q.double() * one[:, at:at + 1].double().repeat_interleave(Hq // Hk, 2)).sum(-1).transpose(1, 2) / math.sqrt(D)
        assert ((lse.double() - want).abs() <= 1e-5 * (1 + want.abs())).all()


BACKWARD = {"tile": (1, 80, 90, 2, 1), "whole": (1, 300, 260, 2, 2), "whole_parts": (1, 2600, 200, 1, 1), "keys_in_parts": (1, 200, 2600, 1, 1)}


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kernel", list(BACKWARD))
def test_a_row_statistic_that_is_nan_or_far_off_shows_in_every_gradient_it_enters(kernel, D, dtype):
    """lse of one row is NaN, or so low that its probabilities overflow: dq of that row, dk and dv of all keys are not finite."""
    from paper_2608_11034_b200 import replay
    B, Tq, Tk, Hq, Hk = BACKWARD[kernel]
    q, k, v, do = make(43, dtype, B, Tq, Tk, Hq, Hk, D)
    o, lse = replay.attention_forward(q, k, v)
    want = defn.attention(q, k, v, do)
    for value in (math.nan, -300.0):
        for row in list(range(32, 64)) + [0, Tq - 1]:
            bad = lse.clone()
            bad[0, 0, row] = value
            dq, dk, dv = replay.attention_backward(q, k, v, o, bad, do)
            for x in (dq[0, row, 0], dk[0, :, 0], dv[0, :, 0]):
                assert not torch.isfinite(x).any(), (value, row)
            rest = torch.ones(Tq, dtype=torch.bool, device="cuda")
            rest[row] = False
            assert ((dq.double() - want["dq"]).abs() <= want["b_dq"])[0, rest].all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_what_a_row_does_not_see_never_reaches_it_in_float16(D, causal, value):
    """Non-finite keys, values, queries and gradients in float16: rows and keys that see none of them keep their results."""
    from paper_2608_11034_b200 import replay
    B, T, Hq, Hk, at = 1, 300, 2, 1, 171
    q, k, v, do = make(44, HF, B, T, T, Hq, Hk, D)
    clean = defn.attention(q, k, v, do, causal=True)
    o, lse = replay.attention_forward(q, k, v, causal=True)
    kb, vb, gb = k.clone(), v.clone(), do.clone()
    kb[0, at], vb[0, at], gb[0, at] = value, value, value
    for kk, vv in ((kb, v), (k, vb)):
        o2, l2 = replay.attention_forward(q, kk, vv, causal=True)
        assert ((o2.double() - clean["o"]).abs() <= clean["b_o"])[:, :at].all() and torch.isfinite(l2[..., :at]).all()
        dq, dk, dv = replay.attention_backward(q, kk, vv, o, lse, do, causal=True)
        assert ((dq.double() - clean["dq"]).abs() <= clean["b_dq"])[:, :at].all()
    assert not torch.isfinite(replay.attention_forward(q, k, vb, causal=True)[0][:, at:]).any()
    dq, dk, dv = replay.attention_backward(q, k, v, o, lse, gb, causal=True)
    assert ((dk.double() - clean["dk"]).abs() <= clean["b_dk"])[:, at + 1:].all()
    assert ((dv.double() - clean["dv"]).abs() <= clean["b_dv"])[:, at + 1:].all()
    assert not torch.isfinite(dv[:, :at + 1]).any()


def test_powers_of_two_by_multiply_adds():
    """The sum of a row's weights, where one score is 0 and the others lie a known distance below, over two binades in small
    steps.  Bound on the natural logarithm: 2.7e-6 of the polynomial, 2^-24 relative for each of the score (up to 2^4 on powers of
    two, times ln 2), the scale, the sums (eight roundings) and the logarithm, the result up to 6 in size."""
    from paper_2608_11034_b200 import replay
    Tq, Tk, D = 512, 128, 64
    q, k, v = (torch.zeros(1, t, 1, D, dtype=HF, device="cuda") for t in (Tq, Tk, Tk))
    depth = torch.arange(Tq, device="cuda", dtype=torch.float64) * (2.0 / Tq)     # exact in float16: multiples of 2^-8
    q[0, :, 0, 0] = depth.to(HF)
    k[0, 1:, 0, 0] = -1.0
    # scores 0 and -depth, natural units
    _, lse = replay.attention_forward(q, k, v, scale=1.0)
    want = torch.log(1.0 + (Tk - 1) * torch.exp(-depth))
    bound = 2.7e-6 + 2.0 ** -24 * (16 * math.log(2) * 2 + 8 + 2 * 6)
    assert ((lse[0, 0].double() - want).abs() <= bound).all()


def where_nan_belongs(q, k, v, do, see, group):
    """Truth values in [batch, heads, tokens, head_dim]: which elements of o, dq, dk, dv (and of lse) the formulas make NaN, from
    where the inputs are.  see: [batch, 1, q_len, kv_len]."""
    up = lambda x: x.isnan().permute(0, 2, 1, 3)                                      # noqa: E731
    Q, G = up(q), up(do)
    K, V = (up(x).repeat_interleave(group, 1) for x in (k, v))
    see = see.expand(-1, Q.shape[1], -1, -1)
    reach = lambda a, b: (a.float() @ b.float()) > 0                                  # noqa: E731
    score = see & (Q.any(-1)[..., :, None] | K.any(-1)[..., None, :])
    lse = score.any(-1)
    o = lse[..., None] | reach(see, V)
    p = see & (score | lse[..., None])
    delta = see.any(-1) & (o | G).any(-1)
    ds = see & (p | G.any(-1)[..., :, None] | V.any(-1)[..., None, :] | delta[..., None])
    dq = ds.any(-1)[..., None] | reach(see, K)
    back = lambda x: x.view(x.shape[0], -1, group, *x.shape[2:]).any(2)               # noqa: E731
    dk = back(ds.any(-2)[..., None] | reach(see.transpose(-1, -2), Q))
    dv = back(p.any(-2)[..., None] | reach(see.transpose(-1, -2), G))
    return lse, o, dq, dk, dv


@pytest.mark.parametrize("seed", range(1150, 1310))
def test_nan_is_where_the_formulas_put_it_and_nowhere_else(seed):
    """A few NaN anywhere in the inputs, single elements and whole tokens, under every mask and in every kernel."""
    import random
    from paper_2608_11034_b200 import replay
    r = random.Random(seed)
    dtype, B, Hk, group, D = r.choice([BF, HF]), r.randint(1, 2), r.choice([1, 2]), r.choice([1, 2, 3]), r.choice([8, 64, 72, 128])
    Tk = r.choice([r.randint(1, 40), r.randint(90, 500)])
    Tq = r.choice([Tk, Tk, r.randint(1, 500), r.randint(1, 20)])
    causal = r.random() < 0.65
    window = r.choice([0, 0, 1, r.randint(2, 300)]) if causal else 0
    q, k, v, do = make(seed, dtype, B, Tq, Tk, Hk * group, Hk, D)
    for x in (q, k, v, do):
        for _ in range(r.choice([0, 1, 1, 3])):
            at = tuple(r.randrange(s) for s in x.shape)
            x[at if r.random() < 0.7 else at[:3]] = math.nan
    ql = kl = None
    if r.random() < 0.4:
        ql, kl = (torch.tensor([r.randint(0, t) for _ in range(B)], dtype=torch.int32, device="cuda") for t in (Tq, Tk))
    see = torch.zeros(B, 1, Tq, Tk, dtype=torch.bool, device="cuda")
    for b in range(B):
        nq, nk = Tq if ql is None else int(ql[b]), Tk if kl is None else int(kl[b])
        for i in range(nq):
            keys = defn.seen_by_row(i, nq, nk, causal, window)
            see[b, 0, i, keys.start:keys.stop] = True
    kw = dict(causal=causal, window=window, q_lens=ql, kv_lens=kl)
    o, lse = replay.attention_forward(q, k, v, **kw)
    got = (o,) + replay.attention_backward(q, k, v, o, lse, do, **kw)
    want = where_nan_belongs(q, k, v, do, see, group)
    assert torch.equal(lse.isnan(), want[0])
    for name, x, w in zip(("o", "dq", "dk", "dv"), got, want[1:]):
        assert torch.equal(x.permute(0, 2, 1, 3).isnan(), w), name
