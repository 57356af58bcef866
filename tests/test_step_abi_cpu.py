"""Arguments of the step entry points are validated before any device work."""
import numpy as np
import pytest

from paper_2608_11034_b200 import binding, build

B, F, H, I32, I64 = binding.DT_BF16, binding.DT_F32, binding.DT_F16, binding.DT_I32, binding.DT_I64
BAD, ALIGN, NOT = binding.ERR_INVALID, binding.ERR_ALIGN, binding.ERR_UNSUPPORTED


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return binding.lib()


def test_embedding_arguments_are_checked(lib):
    f, b = lib.scout_embed_forward, lib.scout_embed_backward

    def fwd(idt=I64, t=B, o=B, rows=4, dim=8, vocab=10, ids=256, table=256, ts=8, scale=1.0, y=256, ys=8):
        return f(idt, t, o, rows, dim, vocab, ids, table, ts, scale, y, ys, 0)

    assert fwd(idt=B) == fwd(t=I64) == fwd(o=H) == NOT and fwd(t=99) == BAD
    assert fwd(scale=float("nan")) == fwd(scale=float("inf")) == BAD
    assert fwd(ids=0) == fwd(table=0) == fwd(y=0) == fwd(ts=7) == fwd(ys=7) == BAD
    assert fwd(ids=260) == fwd(table=257) == fwd(y=255) == ALIGN and fwd(o=F, y=258) == ALIGN
    assert fwd(rows=0, ids=0, table=0, y=0) == fwd(dim=0) == binding.OK
    assert fwd(rows=2 ** 31) == fwd(vocab=2 ** 31) == NOT
    n = binding.scout_embed_backward_workspace(100, 64, 1000)
    assert n % 256 == 0 and n >= 4 * 100 * 4 + 4 * 2 * 64 * 4

    def bwd(idt=I64, t=B, o=F, rows=100, dim=64, vocab=1000, ids=256, dy=256, ds=64, scale=1.0, w=256, wst=64, acc=0, ws=256, nb=n):
        return b(idt, t, o, rows, dim, vocab, ids, dy, ds, scale, w, wst, acc, ws, nb, 0)

    assert bwd(nb=n - 1) == bwd(ws=0) == bwd(acc=2) == bwd(dy=0) == bwd(w=0) == bwd(ids=0) == bwd(ds=63) == bwd(wst=63) == BAD
    assert bwd(ws=264) == bwd(w=258) == bwd(ids=252) == ALIGN
    assert bwd(o=H) == bwd(idt=F) == NOT
    assert bwd(vocab=0) == bwd(dim=0) == bwd(rows=0, acc=1) == binding.OK


def test_dropout_arguments_are_checked(lib):
    def call(t=B, rows=4, cols=8, x=256, xs=8, y=256, ys=8, p=0.1, off=0):
        return lib.scout_dropout(t, rows, cols, x, xs, y, ys, p, 1, 2, off, 0)

    assert call(t=I64) == NOT and call(t=77) == BAD
    assert call(p=-0.1) == call(p=1.0) == call(p=float("nan")) == BAD
    assert call(x=0) == call(y=0) == call(xs=7) == call(ys=7) == BAD
    assert call(x=257) == call(y=257) == call(off=4) == ALIGN
    assert call(rows=2 ** 33) == call(cols=2 ** 34) == NOT
    assert call(rows=0, x=0, y=0) == call(cols=0) == binding.OK


def join(**kw):
    a = np.zeros(1, dtype=binding.JOIN_DTYPE)
    d = dict(dtype=B, stream_dtype=F, weight_dtype=B, scale=1.0, eps=1e-6, rows=12, dim=64, groups=3, x_stride=64, b_stride=64, y_stride=64,
             n_stride=64, dy_stride=64, dn_stride=64, dx_stride=64, db_stride=64)
    d.update(kw)
    for n, x in d.items():
        a[0][n] = x
    return a


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=99), BAD), (dict(dtype=I32), NOT), (dict(stream_dtype=H), NOT), (dict(weight_dtype=H), NOT), (dict(scale=float("nan")), BAD),
    (dict(eps=-1.0), BAD), (dict(eps=float("inf")), BAD), (dict(dim=0), BAD), (dict(dim=16385), NOT), (dict(groups=0), BAD),
    (dict(groups=5), BAD), (dict(rows=3 * 2 ** 31), NOT), (dict(x_stride=2 ** 32), NOT), (dict(reserved=1), BAD), (dict(dtype=F, weight_dtype=B), NOT)])
def test_join_descriptions_are_checked(kw, code):
    with pytest.raises(binding.ScoutError) as e:
        binding.scout_join_backward_workspace(join(**kw).ctypes.data)
    assert e.value.code == code


def test_join_pointers_are_checked(lib):
    a = join()
    at = a.ctypes.data
    n = binding.scout_join_backward_workspace(at)

    def fwd(x=256, b=256, gate=256, post=256, norm=256, p=0.0, off=0, y=256, nn=256, stats=256, j=at):
        return lib.scout_join_forward(j, x, b, gate, post, norm, p, 1, 2, off, y, nn, stats, 0)

    assert fwd(j=0) == fwd(b=0) == fwd(y=0) == fwd(nn=0) == fwd(norm=0) == fwd(stats=0) == fwd(p=1.0) == BAD
    assert fwd(x=258) == fwd(b=257) == fwd(gate=257) == fwd(stats=258) == fwd(off=12) == ALIGN
    short = join(y_stride=63)
    assert fwd(j=short.ctypes.data) == BAD

    def bwd(dy=256, dn=256, b=256, y=256, stats=256, gate=256, post=256, norm=256, p=0.0, dx=256, db=256, dg=256, dp=256, dnm=256, ws=256, nb=n):
        return lib.scout_join_backward(at, dy, dn, b, y, stats, gate, post, norm, p, 1, 2, 0, dx, db, dg, dp, dnm, ws, nb, 0)

    assert bwd(gate=0) == bwd(post=0) == bwd(norm=0) == bwd(dn=0) == bwd(b=0) == bwd(y=0) == bwd(stats=0) == bwd(db=0) == bwd(nb=n - 1) == bwd(ws=0) == BAD
    assert bwd(dy=258) == bwd(dx=258) == bwd(dg=257) == bwd(ws=128) == ALIGN
    empty = join(rows=0)
    assert lib.scout_join_forward(empty.ctypes.data, 0, 0, 0, 0, 0, 0.0, 0, 0, 0, 0, 0, 0, 0) == binding.OK


def test_loss_arguments_are_checked(lib):
    f, b = binding.scout_loss_workspace(B, 100, 64, 1000)
    assert f % 256 == 0 and b % 256 == 0 and b >= 128 * 1000 * 2 + 128 * 64 * 6
    for bad, code in (((F, 4, 8, 4), NOT), ((99, 4, 8, 4), BAD), ((B, 4, 12, 4), NOT), ((B, 4, 0, 4), BAD), ((B, 2 ** 25, 8, 4), NOT),
                      ((B, 4, 8, 2 ** 25), NOT), ((B, 4, 65544, 4), NOT), ((B, 2 ** 23, 8, 2 ** 24), NOT)):
        with pytest.raises(binding.ScoutError) as e:
            binding.scout_loss_workspace(*bad)
        assert e.value.code == code, bad

    def fwd(t=B, idt=I64, rows=100, dim=64, vocab=1000, x=256, xs=64, w=256, wst=64, tg=256, loss=256, lse=256, ws=256, nb=f):
        return lib.scout_loss_forward(t, idt, rows, dim, vocab, x, xs, w, wst, tg, loss, lse, ws, nb, 0)

    assert fwd(idt=F) == NOT
    assert fwd(x=0) == fwd(w=0) == fwd(tg=0) == fwd(loss=0) == fwd(lse=0) == fwd(ws=0) == fwd(nb=f - 1) == fwd(xs=63) == fwd(wst=56) == BAD
    assert fwd(x=257) == fwd(w=264) == fwd(wst=68) == fwd(tg=260) == fwd(loss=258) == fwd(ws=128) == ALIGN
    assert fwd(rows=0, x=0, w=0, tg=0, loss=0, lse=0) == binding.OK

    def bwd(out=B, x=256, w=256, tg=256, lse=256, dl=256, dls=0, dx=256, dxs=64, dw=256, dws=64, acc=0, ws=256, nb=b):
        return lib.scout_loss_backward(B, I64, out, 100, 64, 1000, x, 64, w, 64, tg, lse, dl, dls, dx, dxs, dw, dws, acc, ws, nb, 0)

    assert bwd(out=H) == bwd(acc=2) == bwd(x=0) == bwd(w=0) == bwd(tg=0) == bwd(lse=0) == bwd(dl=0) == bwd(dx=0) == bwd(dw=0) == BAD
    assert bwd(dxs=63) == bwd(dws=63) == bwd(ws=0) == bwd(nb=b - 1) == BAD
    assert bwd(dx=257) == bwd(dw=257) == bwd(lse=258) == bwd(dl=258) == bwd(ws=128) == ALIGN and bwd(out=F, dw=258) == ALIGN
