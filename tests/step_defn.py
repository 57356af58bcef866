"""The step operators written out in 64 bits, with the error bounds that follow from the roundings they document.  Shares nothing with
the library.

Bounds.  u is the unit roundoff of the stored type (2^-8 bfloat16, 2^-11 float16, 2^-24 float32); float16 also loses what lies below
2^-24 (half of that, TINY), and so do sums there.  fp32 arithmetic: a sum of k terms is off by at most k 2^-24 of the sum of
their magnitudes, in whatever order; a sum over a row runs over at most 16 terms a thread and then over a tree of at most ten levels,
which with the roundings of the terms themselves, the mean, a reciprocal root (2 ulp) and the products around it stays within
ROW = 64 * 2^-24 of the magnitudes that enter."""
import math

import numpy as np
import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}
ROW = 64 * 2.0 ** -24


def philox(counter, key):
    """Philox 4x32 with ten rounds, one counter at a time, in Python's whole numbers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def numbers(rows, cols, seed, offset, first_row=0):
    """uint16 [rows, cols]: the same, all places at once"""
    m, s32 = np.uint64(0xFFFFFFFF), np.uint64(32)
    col, row = np.meshgrid(np.arange(-(-cols // 8), dtype=np.uint64), np.arange(first_row, first_row + rows, dtype=np.uint64))
    c = [col, row, np.full_like(col, offset & 0xFFFFFFFF), np.full_like(col, offset >> 32)]
    k = [np.uint64(seed & 0xFFFFFFFF), np.uint64(seed >> 32)]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> s32) ^ c[1] ^ k[0], b & m, (a >> s32) ^ c[3] ^ k[1], a & m]
        k = [(k[0] + np.uint64(0x9E3779B9)) & m, (k[1] + np.uint64(0xBB67AE85)) & m]
    return np.stack(c, -1).astype("<u4").view("<u2").reshape(rows, 8 * (-(-cols // 8)))[:, :cols]


def mask(rows, cols, p, seed, offset, first_row=0):
    """float64 [rows, cols]: 0, or the factor of a place that is kept"""
    cut = min(65535, math.floor(65536 * p + 0.5))
    return torch.from_numpy(np.where(numbers(rows, cols, seed, offset, first_row) >= cut, 65536 / (65536 - cut), 0.0))


def embedding_gradient(dy, ids, vocab, scale, out_dtype, grad=None):
    """-> float64 [vocab, dim], bound"""
    live = (ids >= 0) & (ids < vocab)
    at, d = ids[live].long(), dy[live].double()
    total, mag = (torch.zeros(vocab, dy.shape[-1], dtype=torch.float64, device=dy.device) for _ in range(2))
    total.index_add_(0, at, d * scale)
    mag.index_add_(0, at, d.abs() * abs(scale))
    count = torch.bincount(at, minlength=vocab)[:, None]
    if grad is not None:
        total += grad.double()
    # the sum, the product with the scale, and its addition to what was there
    bound = (count + 2) * 2.0 ** -24 * mag + (2.0 ** -24 + U[out_dtype]) * total.abs() + TINY[out_dtype]
    return total, bound


def join(x, block, gate, post, norm, scale, eps, drop):
    """drop: float64 mask or None -> dict of y, n, rb, ry, u and bounds b_y, b_n"""
    rows, dim = block.shape
    b = block.double()
    one = torch.ones(dim, dtype=torch.float64, device=block.device)
    rb = (b.square().mean(1, keepdim=True) + eps).rsqrt() if post is not None else torch.zeros_like(b[:, :1])
    u = b * rb * post.double() if post is not None else b
    if drop is not None:
        u = torch.where(drop == 0, 0.0, u * drop)
    g = (one[None] if gate is None else gate.double().view(-1, dim))
    add = scale * g.repeat_interleave(rows // g.shape[0], 0) * u
    y = add + (0 if x is None else x.double())
    off = ROW * add.abs() + 2.0 ** -24 * y.abs()
    r = dict(y=y, u=u, rb=rb, gate=g, b_y=off + U[(block if x is None else x).dtype] * y.abs() + TINY[(block if x is None else x).dtype])
    r["ry"] = (y.square().mean(1, keepdim=True) + eps).rsqrt() if norm is not None else torch.zeros_like(b[:, :1])
    if norm is not None:
        w = norm.double()
        r["n"] = y * r["ry"] * w
        # ry is off by what the row's sum is off: its own rounding and twice the relative error of the y that enter it
        slip = ROW + (y.abs() * off).sum(1, keepdim=True) / y.square().sum(1, keepdim=True).clamp(min=1e-300)
        r["b_n"] = off * r["ry"] * w.abs() + (slip + U[block.dtype]) * r["n"].abs() + TINY[block.dtype]
    return r


def join_gradient(dy, dn, block, y, stats, gate, post, norm, scale, drop):
    """From what the call is given (y and stats as they are) -> dict of dx, db, dgate, dpost, dnorm and bounds b_*"""
    rows, dim = block.shape
    rb, ry = stats.double()[0][:, None], stats.double()[1][:, None]
    b, z = block.double(), y.double() * ry
    zero = torch.zeros_like(b)
    g = zero.clone() if dy is None else dy.double()
    e = ROW * g.abs()
    r = {}
    if dn is not None:
        t = dn.double() * norm.double()
        g = g + ry * (t - z * (t * z).mean(1, keepdim=True))
        e = e + ROW * ry * (t.abs() + z.abs() * (t * z).abs().mean(1, keepdim=True))
        r["dnorm"] = (dn.double() * z).sum(0)
        mag = (dn.double() * z).abs().sum(0)
        r["b_dnorm"] = (rows + 4) * 2.0 ** -24 * mag + U[norm.dtype] * r["dnorm"].abs() + TINY[norm.dtype]
    r["dx"], r["b_dx"] = g, e + U[y.dtype] * g.abs() + TINY[y.dtype]
    m = torch.ones_like(b) if drop is None else drop.to(b.device)
    gt = torch.ones(1, dim, dtype=torch.float64, device=b.device) if gate is None else gate.double().view(-1, dim)
    per = gt.repeat_interleave(rows // gt.shape[0], 0)
    c = b * rb if post is not None else b
    w = post.double() if post is not None else torch.ones(dim, dtype=torch.float64, device=b.device)
    h, eh = scale * g, abs(scale) * e + 4 * 2.0 ** -24 * (scale * g).abs()
    u = torch.where(m == 0, 0.0, c * w * m)
    if gate is not None:
        fold = lambda q: q.view(gt.shape[0], -1, dim).sum(1).view(gate.shape)        # noqa: E731
        r["dgate"] = fold(h * u)
        r["b_dgate"] = fold(eh * u.abs()) + (rows + 8) * 2.0 ** -24 * fold((h * u).abs()) + U[gate.dtype] * r["dgate"].abs() + TINY[gate.dtype]
    du = torch.where(m == 0, 0.0, h * per * m)
    edu = eh * (per * m).abs() + 4 * 2.0 ** -24 * du.abs()
    if post is None:
        r["db"], r["b_db"] = du, edu + U[block.dtype] * du.abs() + TINY[block.dtype]
        return r
    r["dpost"] = (du * c).sum(0)
    r["b_dpost"] = (edu * c.abs()).sum(0) + (rows + 8) * 2.0 ** -24 * (du * c).abs().sum(0) + U[post.dtype] * r["dpost"].abs() + TINY[post.dtype]
    s, es = du * w, edu * w.abs() + 4 * 2.0 ** -24 * (du * w).abs()
    r["db"] = rb * (s - c * (s * c).mean(1, keepdim=True))
    r["b_db"] = rb * (es + c.abs() * ((es * c.abs()).mean(1, keepdim=True) + ROW * (s * c).abs().mean(1, keepdim=True)) + ROW * s.abs()) + \
        U[block.dtype] * r["db"].abs() + TINY[block.dtype]
    return r


def within(got, want, bound):
    """Largest |got - want| / bound; NaN places must agree."""
    got = got.double()
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan)
    d = torch.where(nan | (got == want), 0.0, (got - want).abs() / bound.clamp(min=1e-300))
    return float(d.max()) if d.numel() else 0.0


def loss(x, w, targets, dloss=None):
    """-> dict of loss, lse (and dx, dw) and bounds b_*.

    Scores are sums of `dim` exact products: chains of at most 1024 added by the tensor cores, which truncate (2^-23 of the running
    sum for each 16 products that enter it, taken as 2^-23 * 64 of the sum of magnitudes), then fp32 additions; SCORE covers both.
    lse moves by no more than the largest error of a score, and its own sum, exponentials (2 ulp) and logarithm by 2^-20; G by its
    rounding and by exp of what scores and lse are off, and its products as the scores are."""
    u, tiny = U[x.dtype], TINY[x.dtype]
    live = (targets >= 0) & (targets < w.shape[0])
    at = torch.where(live, targets, 0).long()
    xd, wd = torch.where(live[:, None], x.double(), 0.0), w.double()
    s = xd @ wd.t()
    off = 2.0 ** -17 * (xd.abs() @ wd.abs().t()).amax(1)
    lse = torch.logsumexp(s, 1)
    st = s.gather(1, at[:, None])[:, 0]
    r = dict(lse=torch.where(live, lse, 0.0), loss=torch.where(live, lse - st, 0.0))
    r["b_lse"] = off + 2.0 ** -20 + 2.0 ** -23 * lse.abs()
    r["b_loss"] = r["b_lse"] + off + 2.0 ** -23 * st.abs()
    if dloss is None:
        return r
    g = torch.where(live, dloss.double(), 0.0)
    p = torch.exp(s - lse[:, None])
    e = g.abs()[:, None] * p * (off[:, None] * 2 + 2.0 ** -19)
    p[torch.arange(len(p), device=p.device), at] -= 1
    gs = g[:, None] * p
    # the least that float16 holds is 2^-24 of what is held 2^13 times over, with the largest g as one
    least = g.abs().max() * (2.0 ** -38 if x.dtype == torch.float16 else 0.0)
    e = e + (u + 2.0 ** -17) * gs.abs() + least
    r["dx"], r["dw"] = gs @ wd, gs.t() @ xd
    r["b_dx"] = torch.where(live[:, None], e @ wd.abs() + u * r["dx"].abs() + tiny, 0.0)
    r["b_dw"] = e.t() @ xd.abs()            # and the rounding of what is stored
    return r
