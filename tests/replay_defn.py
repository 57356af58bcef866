"""The layer-replay operators written out in 64 bits, one sequence and head at a time, with the error bounds that
follow from the roundings the operators document.  Shares nothing with the library.

Bounds.  u is the unit roundoff of the 16-bit type (2^-8 for bfloat16, 2^-11 for float16).  Products of 16-bit
numbers are exact in fp32; what rounds is (a) each probability, and each dS, once to the 16-bit type before its
product, (b) the stored result, (c) the saved o that delta = g . o is taken from, (d) the fp32 arithmetic, taken as
FP32 = 3e-5 of the sum of the terms' magnitudes (scores of up to 2^4 on powers of two carry 2^-20 absolute, which a
power of two turns into 7e-7 relative; sums of a few thousand terms add a few 1e-6).  float16 also loses what lies
below 2^-24: 2^-25 per factor, TINY."""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
FP32 = 3e-5
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


def seen_by_row(i, nq, nk, causal, window):
    """keys row i sees, as a range"""
    if i >= nq:
        return range(0)
    p = i + nk - nq
    hi = min(nk, p + 1) if causal else nk
    lo = max(0, p - window + 1) if window else 0
    return range(lo, max(hi, lo))


def attention(q, k, v, do=None, *, causal=False, window=0, scale=None, q_lens=None, kv_lens=None):
    """-> dict of float64 o, lse (and dq, dk, dv) and elementwise bounds under 'b_' + name.  Masked places are never read."""
    B, Tq, Hq, D = q.shape
    Tk, Hk = k.shape[1], k.shape[2]
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    u, tiny, dev = U[q.dtype], TINY[q.dtype], q.device
    z = lambda *s: torch.zeros(*s, dtype=torch.float64, device=dev)      # noqa: E731
    r = {n: z(B, Tq, Hq, D) for n in ("o", "b_o", "dq", "b_dq")}
    r.update({n: z(B, Tk, Hk, D) for n in ("dk", "b_dk", "dv", "b_dv")})
    r["lse"] = torch.full((B, Hq, Tq), -math.inf, dtype=torch.float64, device=dev)
    for b in range(B):
        nq = Tq if q_lens is None else min(max(int(q_lens[b]), 0), Tq)
        nk = Tk if kv_lens is None else min(max(int(kv_lens[b]), 0), Tk)
        see = torch.zeros(nq, nk, dtype=torch.bool, device=dev)
        for i in range(nq):
            keys = seen_by_row(i, nq, nk, causal, window)
            see[i, keys.start:keys.stop] = True
        some = see.any(1)
        for h in range(Hq):
            g = h // (Hq // Hk)
            qd, kd, vd = q[b, :nq, h].double(), k[b, :nk, g].double(), v[b, :nk, g].double()
            # a hidden place must not turn a product into NaN: every product runs over visible places only
            keep = lambda m, x: torch.where(m, x, 0.0)                   # noqa: E731
            s = torch.where(see, qd @ torch.nan_to_num(kd, 0.0, 0.0, 0.0).t() * scale, -math.inf)
            bad_k, bad_v = ~torch.isfinite(kd).all(1), ~torch.isfinite(vd).all(1)
            assert not (see & (bad_k | bad_v)[None, :]).any(), "this oracle takes finite visible values"
            vd = torch.where(bad_v[:, None], 0.0, vd)
            kd = torch.where(bad_k[:, None], 0.0, kd)
            lse = torch.logsumexp(s, 1) if nk else torch.full((nq,), -math.inf, dtype=torch.float64, device=dev)
            p = keep(see, torch.exp(s - torch.where(some, lse, 0.0)[:, None]))
            o = p @ vd
            r["lse"][b, h, :nq] = lse
            r["o"][b, :nq, h] = o
            mag = p @ vd.abs()
            r["b_o"][b, :nq, h] = u * (mag + o.abs()) + FP32 * mag + tiny * (1 + vd.abs().sum(0))
            if do is None:
                continue
            gd = torch.where(some[:, None], do[b, :nq, h].double(), 0.0)
            qd = torch.where(some[:, None], qd, 0.0)
            dp = gd @ vd.t()
            delta = (gd * o).sum(1, keepdim=True)
            ds = p * (dp - delta)
            dq, dk, dv = scale * (ds @ kd), scale * (ds.t() @ qd), p.t() @ gd
            # dS: its own rounding, delta's error from the rounded o, and the fp32 terms it is the difference of
            off = (gd.abs() * (u * o.abs() + r["b_o"][b, :nq, h])).sum(1, keepdim=True)
            e_ds = u * ds.abs() + p * off + FP32 * p * (gd.abs() @ vd.abs().t() + (gd.abs() * o.abs()).sum(1, keepdim=True)) + \
                keep(see, torch.full_like(ds, tiny))
            e_p = (u + FP32) * p + keep(see, torch.full_like(p, tiny))
            r["dq"][b, :nq, h] = dq
            r["b_dq"][b, :nq, h] = scale * (e_ds @ kd.abs() + FP32 * ds.abs() @ kd.abs()) + u * dq.abs() + tiny
            r["dk"][b, :nk, g] += dk
            r["b_dk"][b, :nk, g] += scale * (e_ds.t() @ qd.abs() + FP32 * ds.abs().t() @ qd.abs())
            r["dv"][b, :nk, g] += dv
            r["b_dv"][b, :nk, g] += e_p.t() @ gd.abs()
    r["b_dk"] += u * r["dk"].abs() + tiny
    r["b_dv"] += u * r["dv"].abs() + tiny
    return r


# ---- 8-bit activation checkpoints: exact, so there is nothing to bound --------------------------------

TOP_STEP = {torch.float32: 122, torch.bfloat16: 122, torch.float16: 10}


def pack(x):
    """Element by element in Python floats (which hold every input exactly) -> nested lists codes, exps."""
    top_step = TOP_STEP[x.dtype]
    codes, exps = [], []
    for row in x.double().cpu().tolist():
        crow, erow = [], []
        for c0 in range(0, len(row), 32):
            part = row[c0:c0 + 32]
            amax = max([abs(y) for y in part if math.isfinite(y)], default=0.0)
            e = -126
            while amax > 127 * 2.0 ** e:
                e += 1
            top = 63 if e == top_step else 127
            erow.append(e)
            # Python's round() of a float is to nearest, ties to even; y / 2^e is exact in a double
            crow += [max(-top, min(top, round(y / 2.0 ** e))) if math.isfinite(y) else -128 for y in part]
        codes.append(crow)
        exps.append(erow)
    return codes, exps


def restore(codes, exps):
    """int8 codes [rows, cols], exps -> float64 values (exact)"""
    step = torch.exp2(exps.double()).repeat_interleave(32, 1)[:, :codes.shape[1]]
    return torch.where(codes == -128, math.nan, codes.double() * step)
