"""A block joins the residual stream: results and gradients against the definition in 64 bits, and gradients against differences."""
import math

import pytest
import torch

import step_defn as defn

pytestmark = pytest.mark.gpu
BF, H, F = torch.bfloat16, torch.float16, torch.float32
SEED, OFFSET, EPS = 77, (1 << 35) + 3, 1e-5


def inputs(rows, dim, groups, tb, ts, tw, parts, seed=0, strided=False):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype, scale=1.0, mean=0.0):
        t = (torch.randn(*shape, generator=g, device="cuda") * scale + mean).to(dtype)
        if strided and len(shape) == 2 and shape[0] == rows:
            room = torch.full((rows, dim + 5), math.nan, dtype=dtype, device="cuda")
            room[:, 3:dim + 3] = t
            return room[:, 3:dim + 3]
        return t

    s = dict(x=normal(rows, dim, dtype=ts) if "x" in parts else None, block=normal(rows, dim, dtype=tb, scale=0.6), dy=normal(rows, dim, dtype=ts),
             dn=normal(rows, dim, dtype=tb))
    s["gate"] = (torch.randn(groups, dim, generator=g, device="cuda") * 0.3 + 0.7).to(tw) if "g" in parts else None
    if groups == 1 and s["gate"] is not None:
        s["gate"] = s["gate"][0]
    s["post"], s["norm"] = ((torch.randn(dim, generator=g, device="cuda") * 0.2 + 1).to(tw) if c in parts else None for c in "pn")
    return s


def check(rows, dim, groups, tb, ts, tw, parts, p, scale=0.7, seed=0, strided=False):
    from paper_2608_11034_b200 import step
    s = inputs(rows, dim, groups, tb, ts, tw, parts, seed, strided)
    drop = defn.mask(rows, dim, p, SEED, OFFSET).cuda() if p else None
    how = dict(gate=s["gate"], post_weight=s["post"], norm_weight=s["norm"], scale=scale, p=p, seed=SEED, offset=OFFSET)
    scale = float(torch.tensor(scale))                  # as the library gets it
    y, n, stats = step.join_forward(s["x"], s["block"], eps=EPS, **how)
    r = defn.join(s["x"], s["block"], s["gate"], s["post"], s["norm"], scale, float(torch.tensor(EPS)), drop)
    assert y.dtype == (tb if s["x"] is None else ts) and defn.within(y, r["y"], r["b_y"]) <= 1
    assert (n is None) == (s["norm"] is None)
    if n is not None:
        assert n.dtype == tb and defn.within(n, r["n"], r["b_n"]) <= 1
    for k, name in enumerate(("rb", "ry")):
        assert defn.within(stats[k], r[name][:, 0], 4 * defn.ROW * r[name][:, 0]) <= 1
    dy = s["dy"].to(y.dtype) if "d" in parts else None
    dn = s["dn"] if n is not None else None
    got = step.join_backward(dy, dn, s["block"], y, stats, **how)
    w = defn.join_gradient(dy, dn, s["block"], y, stats, s["gate"], s["post"], s["norm"], scale, drop)
    for x, name, like in zip(got, ("dx", "db", "dgate", "dpost", "dnorm"), (y, s["block"], s["gate"], s["post"], s["norm"])):
        assert (x is None) == (like is None), name
        if x is not None:
            assert x.shape == like.shape and x.dtype == like.dtype and defn.within(x, w[name], w["b_" + name]) <= 1, name
    # the same bits again
    assert all(a is None or torch.equal(a, b) for a, b in zip((y, n, stats, *got), (*step.join_forward(s["x"], s["block"], eps=EPS, **how),
                                                                                    *step.join_backward(dy, dn, s["block"], y, stats, **how))))


@pytest.mark.parametrize("rows,dim", [(1, 1), (1, 4096), (2, 8), (3, 65), (7, 256), (300, 264), (33, 1000), (64, 1001), (150, 4096), (9, 4104),
                                      (5, 8192), (4, 16383), (3, 16384), (1000, 96), (2500, 512)])
@pytest.mark.parametrize("p", [0.0, 0.2])
def test_sizes(rows, dim, p):
    check(rows, dim, 1, BF, BF, BF, "xgpnd", p)


@pytest.mark.parametrize("tb,ts,tw", [(BF, F, F), (BF, F, BF), (BF, BF, F), (H, H, H), (H, F, H), (H, H, F), (H, F, F), (F, F, F)])
@pytest.mark.parametrize("rows,dim,groups,strided", [(66, 520, 3, False), (40, 777, 40, True), (18, 4224, 2, True)])
def test_types_and_rows_that_lie_apart(rows, dim, groups, strided, tb, ts, tw):
    check(rows, dim, groups, tb, ts, tw, "xgpnd", 0.1, strided=strided)


@pytest.mark.parametrize("tb,ts,tw", [(BF, BF, BF), (H, F, F), (F, F, F)])
@pytest.mark.parametrize("rows,dim", [(301, 6144), (5, 7168), (310, 8192), (150, 8200)])
def test_wide_rows_through_shared_memory_and_not(rows, dim, tb, ts, tw):
    """Two rows of eight thousand fp32 columns and their gradients do not fit into shared memory; those of six thousand do."""
    check(rows, dim, 1, tb, ts, tw, "xgpnd", 0.1)


@pytest.mark.parametrize("parts", ["", "x", "n", "xn", "xp", "xg", "xgnd", "xpnd", "gpnd", "gpn", "xgpn", "pd", "xgd"])
@pytest.mark.parametrize("rows,dim", [(37, 200), (12, 2048), (6, 9000)])
def test_parts_that_are_left_out(parts, rows, dim):
    check(rows, dim, 2 if rows % 2 == 0 else 1, BF, BF, BF, parts, 0.3)


@pytest.mark.parametrize("rows,dim,groups", [(1200, 64, 1), (1200, 64, 3), (1200, 64, 100), (1200, 64, 1200), (1110, 2048, 5), (1184, 512, 37), (999, 4096, 333)])
def test_gates_of_sequences_whose_rows_are_dealt_to_several_blocks(rows, dim, groups):
    check(rows, dim, groups, BF, BF, F, "xgpnd", 0.1)


def test_gradients_are_what_differences_say():
    """Of a sum of the results with fixed weights, in fp32; a central difference over 2^-6 is off by its third order, 2^-12, and by 2^-24
    of the sum's terms over the step: 64 numbers of a few units, 2^-24 * 2^8 * 2^6 = 2^-10."""
    from paper_2608_11034_b200 import step
    rows, dim = 4, 16
    s = inputs(rows, dim, 2, F, F, F, "xgpnd", seed=5)
    how = dict(scale=0.7, p=0.25, seed=SEED, offset=OFFSET)

    def value(t):
        y, n, _ = step.join_forward(t["x"], t["block"], gate=t["gate"], post_weight=t["post"], norm_weight=t["norm"], eps=EPS, **how)
        return float((y.double() * s["dy"].double()).sum() + (n.double() * s["dn"].double()).sum())

    y, _, stats = step.join_forward(s["x"], s["block"], gate=s["gate"], post_weight=s["post"], norm_weight=s["norm"], eps=EPS, **how)
    got = step.join_backward(s["dy"], s["dn"], s["block"], y, stats, gate=s["gate"], post_weight=s["post"], norm_weight=s["norm"], **how)
    for name, grad in zip(("x", "block", "gate", "post", "norm"), got):
        for at in (0, 5, s[name].numel() - 1):
            ends = []
            for sign in (1, -1):
                t = dict(s, **{name: s[name].clone()})
                t[name].view(-1)[at] += sign * 2.0 ** -6
                ends.append(value(t))
            slope = (ends[0] - ends[1]) / 2.0 ** -5
            assert abs(slope - float(grad.view(-1)[at])) <= 2.0 ** -7 * (1 + abs(slope)), (name, at)


def test_a_bad_row_stays_a_bad_row():
    from paper_2608_11034_b200 import step
    s = inputs(50, 264, 50, BF, BF, BF, "xgpnd")
    s["block"][20, 7] = math.nan
    s["x"][30, 9] = math.inf
    y, n, stats = step.join_forward(s["x"], s["block"], gate=s["gate"], post_weight=s["post"], norm_weight=s["norm"])
    ok = torch.ones(50, dtype=torch.bool, device="cuda")
    ok[[20, 30]] = False
    assert torch.isfinite(y[ok]).all() and torch.isfinite(n[ok]).all() and y[20].isnan().all() and n[20].isnan().all()
    assert torch.isfinite(y[30]).sum() == 263 and n[30, 9].isnan()
    dx, db, dgate, _, _ = step.join_backward(s["dy"], s["dn"], s["block"], y, stats, gate=s["gate"], post_weight=s["post"], norm_weight=s["norm"])
    assert all(torch.isfinite(t[ok]).all() for t in (dx, db, dgate)) and dx[20].isnan().all()


def test_no_rows():
    from paper_2608_11034_b200 import step
    s = inputs(0, 64, 1, BF, BF, F, "xgpnd")
    y, n, stats = step.join_forward(s["x"], s["block"], gate=s["gate"], post_weight=s["post"], norm_weight=s["norm"])
    got = step.join_backward(s["dy"], s["dn"], s["block"], y, stats, gate=s["gate"], post_weight=s["post"], norm_weight=s["norm"])
    assert y.shape == n.shape == (0, 64) and all((g == 0).all() for g in got[2:])


def test_captured():
    from paper_2608_11034_b200 import step
    s, at = inputs(600, 512, 3, BF, F, F, "xgpnd"), torch.tensor([4], device="cuda")
    how = dict(gate=s["gate"], post_weight=s["post"], norm_weight=s["norm"], scale=0.5, p=0.2, seed=3)

    def both(offset):
        y, n, stats = step.join_forward(s["x"], s["block"], offset=offset, **how)
        return (y, n, *step.join_backward(s["dy"], s["dn"], s["block"], y, stats, offset=offset, **how))

    both(at)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both(at)
    for n in (4, 5):
        at.fill_(n)
        s["block"].mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, both(n)))


def test_refusals():
    from paper_2608_11034_b200 import step
    s = inputs(6, 64, 2, BF, F, F, "xgpnd")
    x, b, gate, w = s["x"], s["block"], s["gate"], s["norm"]
    y, n, stats = step.join_forward(x, b, gate=gate, post_weight=w, norm_weight=w)
    for bad in (lambda: step.join_forward(x.half(), b), lambda: step.join_forward(x[:5], b), lambda: step.join_forward(x, b.t()),
                lambda: step.join_forward(x, b, gate=gate[:, :63]), lambda: step.join_forward(x, b, gate=torch.ones(4, 64, device="cuda")),
                lambda: step.join_forward(x, b, post_weight=w, norm_weight=w.to(BF)), lambda: step.join_forward(x, b, norm_weight=w.half()),
                lambda: step.join_forward(x, b, norm_weight=w[:8]), lambda: step.join_forward(x, b, eps=-1.0), lambda: step.join_forward(x, b, p=1.0),
                lambda: step.join_forward(x, b, scale=math.inf), lambda: step.join_forward(x, b, norm_weight=torch.ones(128, device="cuda")[::2]),
                lambda: step.join_forward(x.cpu(), b), lambda: step.join_forward(x, b[:, :0]), lambda: step.join_forward(x.clone().requires_grad_(), b),
                lambda: step.join_backward(y, n, b, y, stats), lambda: step.join_backward(y.to(BF), n, b, y, stats, norm_weight=w),
                lambda: step.join_backward(y, n.float(), b, y, stats, norm_weight=w), lambda: step.join_backward(y, n, b, y, stats[:1], norm_weight=w)):
        with pytest.raises(ValueError):
            bad()
    from paper_2608_11034_b200 import binding
    with pytest.raises(binding.ScoutError):
        step.join_forward(None, torch.zeros(2, 16392, device="cuda"))


@pytest.mark.parametrize("tb,ts,tw", [(BF, BF, BF), (H, F, F), (F, F, F)])
@pytest.mark.parametrize("rows,dim,groups,parts", [(70, 520, 5, "xgpnd"), (41, 2048, 41, "xgpnd"), (700, 64, 1, "xpnd"), (37, 4096, 1, "gnd"), (12, 4224, 3, "xgpnd"),
                                                   (33, 777, 3, "xgpnd"), (9, 9001, 1, "xgpnd")])
def test_bits_do_not_depend_on_where_rows_lie(rows, dim, groups, parts, tb, ts, tw):
    from paper_2608_11034_b200 import step

    def moved(t, gap):
        if t is None or t.dim() != 2 or t.shape[0] != rows:
            return t
        room = torch.full((rows, dim + gap), math.nan, dtype=t.dtype, device="cuda")
        room[:, 1:dim + 1] = t
        return room[:, 1:dim + 1]

    s = inputs(rows, dim, groups, tb, ts, tw, parts)
    weights = {n: s[n] for n in ("gate", "post", "norm")}

    def both(s, w):
        how = dict(gate=w["gate"], post_weight=w["post"], norm_weight=w["norm"], scale=0.7, p=0.2, seed=SEED, offset=OFFSET)
        y, n, stats = step.join_forward(s["x"], s["block"], **how)
        dy = None if s["dy"] is None else s["dy"].to(y.dtype)
        return (y, n, stats, *step.join_backward(dy, s["dn"] if n is not None else None, s["block"], y, stats, **how))

    want = both(s, weights)
    # weights off 16-byte boundaries too
    off = {n: None if w is None else torch.cat([w.new_zeros(1), w.reshape(-1)])[1:].view(w.shape) for n, w in weights.items()}
    for gap, w in ((9, weights), (8, weights), (0, off), (9, off)):
        there = {n: moved(t, gap) if gap else t for n, t in s.items() if n in ("x", "block", "dy", "dn")}
        assert all(a is None or torch.equal(a, b) for a, b in zip(want, both(there, w))), gap
