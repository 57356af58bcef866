"""Outputs and scratch of the step entry points between bands of a fixed pattern, which no call may change; and calls that overlap."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, H, F = torch.bfloat16, torch.float16, torch.float32
BAND = 256


class Room:
    def __init__(self):
        self.outer = []

    def take(self, *shape, dtype):
        n = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
        whole = torch.full((n + 2 * BAND,), 0x5A, dtype=torch.uint8, device="cuda")
        self.outer.append((whole, n))
        return whole[BAND:BAND + n].view(dtype).view(*shape)

    def intact(self):
        torch.cuda.synchronize()
        return all(bool((w[:BAND] == 0x5A).all()) and bool((w[BAND + n:] == 0x5A).all()) for w, n in self.outer)


def stream():
    return torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("rows,dim,vocab", [(1, 8, 3), (33, 95, 700), (2500, 264, 1000), (500, 1001, 17)])
@pytest.mark.parametrize("accumulate", [0, 1])
def test_embedding(rows, dim, vocab, accumulate):
    from paper_2608_11034_b200 import binding as b
    room = Room()
    ids = torch.randint(-1, vocab + 1, (rows,), device="cuda")
    table, dy = torch.randn(vocab, dim, device="cuda").to(BF), torch.randn(rows, dim, device="cuda").to(BF)
    y, dw = room.take(rows, dim, dtype=BF), room.take(vocab, dim, dtype=F)
    dw.zero_()
    n = b.scout_embed_backward_workspace(rows, dim, vocab)
    ws = room.take(n, dtype=torch.uint8)
    b.scout_embed_forward(b.DT_I64, b.DT_BF16, b.DT_BF16, rows, dim, vocab, ids.data_ptr(), table.data_ptr(), dim, 1.0, y.data_ptr(), dim, stream())
    b.scout_embed_backward(b.DT_I64, b.DT_BF16, b.DT_F32, rows, dim, vocab, ids.data_ptr(), dy.data_ptr(), dim, 1.0, dw.data_ptr(), dim, accumulate,
                           ws.data_ptr(), n, stream())
    assert room.intact()


@pytest.mark.parametrize("rows,dim,groups", [(1, 8, 1), (7, 95, 7), (65, 256, 5), (31, 1001, 1), (40, 4096, 2), (6, 4104, 1), (3, 16384, 3)])
@pytest.mark.parametrize("dtype", [BF, F])
def test_join_and_dropout(rows, dim, groups, dtype):
    from paper_2608_11034_b200 import binding as b
    room, code = Room(), {BF: b.DT_BF16, F: b.DT_F32}[dtype]
    x, blk, dy, dn = (torch.randn(rows, dim, device="cuda").to(dtype) for _ in range(4))
    gate, post, norm = (torch.randn(*s, device="cuda").to(dtype) for s in ((groups, dim), (dim,), (dim,)))
    y, n, dx, db, z = (room.take(rows, dim, dtype=dtype) for _ in range(5))
    stats, dgate, dpost, dnorm = room.take(2, rows, dtype=F), room.take(groups, dim, dtype=dtype), room.take(dim, dtype=dtype), room.take(dim, dtype=dtype)
    j = np.zeros(1, dtype=b.JOIN_DTYPE)
    j[0] = (code, code, code, 0.5, 1e-6, 0, rows, dim, groups) + (dim,) * 8
    at = j.ctypes.data
    nb = b.scout_join_backward_workspace(at)
    ws = room.take(nb, dtype=torch.uint8)
    p = lambda t: t.data_ptr()                                     # noqa: E731
    b.scout_join_forward(at, p(x), p(blk), p(gate), p(post), p(norm), 0.1, 1, 2, 0, p(y), p(n), p(stats), stream())
    b.scout_join_backward(at, p(dy), p(dn), p(blk), p(y), p(stats), p(gate), p(post), p(norm), 0.1, 1, 2, 0, p(dx), p(db), p(dgate), p(dpost),
                          p(dnorm), p(ws), nb, stream())
    b.scout_dropout(code, rows, dim, p(x), dim, p(z), dim, 0.3, 1, 2, 0, stream())
    assert room.intact()
    assert all(torch.isfinite(t.float()).all() for t in (y, n, stats, dx, db, dgate, dpost, dnorm, z))
    b.scout_dropout(code, rows, dim, p(x), dim, p(x), dim, 0.3, 1, 2, 0, stream())          # in place
    assert torch.equal(x, z)


@pytest.mark.parametrize("rows,dim,vocab", [(1, 8, 1), (130, 72, 300), (257, 264, 1025)])
def test_loss(rows, dim, vocab):
    from paper_2608_11034_b200 import binding as b
    room = Room()
    x, w = torch.randn(rows, dim, device="cuda").to(BF), torch.randn(vocab, dim, device="cuda").to(BF)
    targets, dloss = torch.randint(-1, vocab, (rows,), device="cuda"), torch.ones(1, device="cuda")
    loss, lse = room.take(rows, dtype=F), room.take(rows, dtype=F)
    dx, dw = room.take(rows, dim, dtype=BF), room.take(vocab, dim, dtype=BF)
    f, nb = b.scout_loss_workspace(b.DT_BF16, rows, dim, vocab)
    wf, wb = room.take(f, dtype=torch.uint8), room.take(nb, dtype=torch.uint8)
    p = lambda t: t.data_ptr()                                     # noqa: E731
    b.scout_loss_forward(b.DT_BF16, b.DT_I64, rows, dim, vocab, p(x), dim, p(w), dim, p(targets), p(loss), p(lse), p(wf), f, stream())
    b.scout_loss_backward(b.DT_BF16, b.DT_I64, b.DT_BF16, rows, dim, vocab, p(x), dim, p(w), dim, p(targets), p(lse), p(dloss), 0, p(dx), dim, p(dw),
                          dim, 0, p(wb), nb, stream())
    assert room.intact() and torch.isfinite(loss).all() and torch.isfinite(dx.float()).all() and torch.isfinite(dw.float()).all()


def test_calls_on_several_streams_at_once():
    from paper_2608_11034_b200 import step
    g = torch.Generator(device="cuda").manual_seed(1)
    x, w = torch.randn(600, 256, generator=g, device="cuda").to(BF), torch.randn(3000, 256, generator=g, device="cuda").to(BF)
    ids, dl = torch.randint(0, 3000, (600,), generator=g, device="cuda"), torch.rand(600, generator=g, device="cuda")
    gain = torch.rand(256, generator=g, device="cuda").to(BF)

    def all_of_them():
        e = step.embedding_forward(ids, w)
        y, n, stats = step.join_forward(x, e, gate=gain, post_weight=gain, norm_weight=gain, p=0.1, seed=1)
        loss, lse = step.loss_forward(n, w, ids)
        dn, dw = step.loss_backward(n, w, ids, lse, dl)
        grads = step.join_backward(None, dn, e, y, stats, gate=gain, post_weight=gain, norm_weight=gain, p=0.1, seed=1)
        return [loss, dw, *grads, step.embedding_backward(grads[1], ids, 3000, grad=dw.clone()), step.dropout(y, 0.2, seed=3)]

    want = all_of_them()
    streams = [torch.cuda.Stream() for _ in range(4)]
    torch.cuda.synchronize()
    for _ in range(20):
        got = []
        for s in streams:
            with torch.cuda.stream(s):
                got.append(all_of_them())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for one in got for a, b in zip(one, want))


def test_from_a_thread_that_has_made_no_call_yet():
    import threading

    from paper_2608_11034_b200 import step
    x, w = torch.randn(40, 64, device="cuda").to(BF), torch.randn(90, 64, device="cuda").to(BF)
    t = torch.randint(0, 90, (40,), device="cuda")
    want, got = step.loss_forward(x, w, t), []
    torch.cuda.synchronize()
    th = threading.Thread(target=lambda: got.append(step.loss_forward(x, w, t)))
    th.start()
    th.join()
    torch.cuda.synchronize()
    assert torch.equal(got[0][0], want[0]) and torch.equal(got[0][1], want[1])
