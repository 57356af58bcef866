"""Operators of a replayed training step around its layers, on torch tensors.

A replay from the step's tokens to its loss leaves surfaces that ``replay`` does not make: the embedding's
gradient, the activations between blocks, the loss of every token and the output projection's gradients.
As there, the same values give the same bits on every healthy GPU: no floating-point atomics, every sum in
an order that the sizes and the token ids fix, random numbers from a counter.

    embedding_forward, embedding_backward   rows of a table by token id, and the table's gradient
    dropout                                 with a mask that is made again from a counter, never stored
    join_forward, join_backward             a block's output joins the residual stream: norm, dropout, gate,
                                            scale, sum and the next block's norm in one pass
    loss_forward, loss_backward             softmax cross entropy over a vocabulary, from hidden states and
                                            output projection; the scores are never kept

``include/scout_step.h`` has the definitions.  What ``replay`` says of streams, autograd (the calls raise where
it would have to record them, or to give their results a tangent) and bounded waits (``replay.waits_checked``;
join and loss have such waits) holds here too.
"""
from __future__ import annotations

import functools
import math
from typing import Optional

import numpy as np
import torch

from . import binding
from .replay import _CODE, _enqueue, _fail, _no_autograd, _row_stride

_IDS = {torch.int32: binding.DT_I32, torch.int64: binding.DT_I64}
_MASK64 = (1 << 64) - 1


def _flat_ids(ids: torch.Tensor, device, name: str) -> torch.Tensor:
    if ids.dtype not in _IDS or ids.device != device:
        _fail(f"{name}: int32 or int64, on the other tensors' device")
    return ids if ids.is_contiguous() else ids.contiguous()


def _finite(x, name: str) -> float:
    x = float(x)
    if not math.isfinite(x):
        _fail(f"{name}: a finite number is wanted")
    return x


# ---- token embedding ------------------------------------------------------------------------------------

@functools.lru_cache(maxsize=1024)
def _lookup(shape, stride, dtype, device, out_dtype):
    """Checks a description of a table -> codes of its and the result's type, row stride."""
    if dtype not in _CODE or out_dtype not in (dtype, torch.float32):
        _fail("a table is float32, bfloat16 or float16, what is looked up of its dtype or float32")
    return _CODE[dtype], _CODE[out_dtype], _row_stride(shape, stride, device, "table")


def embedding_forward(ids: torch.Tensor, table: torch.Tensor, *, scale: float = 1.0, out_dtype: Optional[torch.dtype] = None):
    """scale * table[ids].  ids: int32 or int64 of any shape; table: [vocab, dim]; ids outside 0..vocab-1 (padding, or another part of
    the vocabulary) give zeros.  -> [*ids.shape, dim] in out_dtype (the table's, which is the default, or float32)."""
    _no_autograd(table)
    code, out_code, stride = _lookup(table.shape, table.stride(), table.dtype, table.device, out_dtype or table.dtype)
    ids = _flat_ids(ids, table.device, "ids")
    vocab, dim = table.shape
    y = table.new_empty((*ids.shape, dim), dtype=out_dtype or table.dtype)
    _enqueue("scout_embed_forward", table.device.index, _IDS[ids.dtype], code, out_code, ids.numel(), dim, vocab, ids.data_ptr(),
             table.data_ptr(), stride, _finite(scale, "scale"), y.data_ptr(), max(dim, 1))
    return y


@functools.lru_cache(maxsize=1024)
def _table_gradient(shape, stride, dtype, device, ids_shape, vocab, dw_shape, dw_stride, dw_dtype, dw_device):
    """Checks a description of dy and the table's gradient -> codes, rows, dim, row strides, scratch bytes."""
    if dtype not in _CODE or len(shape) != len(ids_shape) + 1 or shape[:-1] != ids_shape:
        _fail("dy: float32, bfloat16 or float16, [*ids.shape, dim]")
    rows, dim = math.prod(ids_shape), shape[-1]
    if len(shape) == 2:
        row = _row_stride(shape, stride, device, "dy")
    else:
        row = max(dim, 1)
        if device.type != "cuda":
            _fail("tensors must be on a CUDA device")
    if dw_dtype not in (dtype, torch.float32) or dw_shape != (vocab, dim) or dw_device != device:
        _fail("the gradient is [vocab, dim], float32 or of dy's dtype, on dy's device")
    dw_row = _row_stride(dw_shape, dw_stride, dw_device, "grad")
    return _CODE[dtype], _CODE[dw_dtype], rows, dim, row, dw_row, binding.scout_embed_backward_workspace(rows, dim, vocab)


def embedding_backward(dy: torch.Tensor, ids: torch.Tensor, vocab: int, *, scale: float = 1.0, out_dtype: Optional[torch.dtype] = None,
                       grad: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of embedding_forward's table from the gradient dy [*ids.shape, dim] of what was looked up.
    -> [vocab, dim] in out_dtype (float32, which is the default, or dy's), zeros for ids that do not occur; with `grad` (of those
    dtypes, of a tied output projection, say) it is added to that in place, rows of ids that do not occur are left alone, and
    out_dtype may only repeat its dtype."""
    _no_autograd(dy, grad)
    ids = _flat_ids(ids, dy.device, "ids")
    if dy.dim() == 0 or vocab < 0:
        _fail("dy: [*ids.shape, dim]; vocab: the table's rows")
    if grad is None:
        dw = dy.new_empty((vocab, dy.shape[-1]), dtype=out_dtype or torch.float32)
    else:
        if out_dtype not in (None, grad.dtype):
            _fail("grad is added to in its own dtype; out_dtype names another")
        dw = grad
    if dy.dim() != 2 and not dy.is_contiguous():
        dy = dy.contiguous()
    code, dw_code, rows, dim, row, dw_row, nbytes = _table_gradient(dy.shape, dy.stride(), dy.dtype, dy.device, ids.shape, vocab, dw.shape,
                                                                   dw.stride(), dw.dtype, dw.device)
    ws = dy.new_empty(nbytes, dtype=torch.uint8) if nbytes else None
    _enqueue("scout_embed_backward", dy.device.index, _IDS[ids.dtype], code, dw_code, rows, dim, vocab, ids.data_ptr(), dy.data_ptr(), row,
             _finite(scale, "scale"), dw.data_ptr(), dw_row, int(grad is not None), ws.data_ptr() if ws is not None else 0, nbytes)
    return dw


# ---- dropout --------------------------------------------------------------------------------------------

def _counter(p: float, seed: int, offset, device):
    """-> p, seed, offset on the host, address of an offset on the device"""
    p = float(p)
    if not 0.0 <= p < 1.0:
        _fail("p: at least 0 and below 1")
    if isinstance(offset, torch.Tensor):
        if offset.dtype != torch.int64 or offset.numel() != 1 or offset.device != device:
            _fail("offset: a whole number, or one int64 on the other tensors' device")
        return p, int(seed) & _MASK64, 0, offset.data_ptr()
    return p, int(seed) & _MASK64, int(offset) & _MASK64, 0


@functools.lru_cache(maxsize=1024)
def _matrix(shape, stride, dtype, device):
    if dtype not in _CODE:
        _fail("x: float32, bfloat16 or float16")
    return _CODE[dtype], _row_stride(shape, stride, device, "x")


def dropout(x: torch.Tensor, p: float, *, seed: int, offset=0) -> torch.Tensor:
    """x [rows, cols] with each place kept with probability 1 - p (in steps of 2^-16) and divided by that, or 0.  Which places are kept
    follows from their row and column, seed and offset alone, so the gradient of x is dropout(dy, p) with the same two numbers,
    and a replay on another GPU drops the same places.
    offset: a whole number (of the training step, layer and place in it, say), or one int64 on the device, which is read when
    the kernel runs: a captured graph then drops other places each time that number has changed."""
    _no_autograd(x)
    if x.dim() != 2:
        _fail("x: a matrix with adjacent row elements is wanted")
    code, stride = _matrix(x.shape, x.stride(), x.dtype, x.device)
    p, seed, host, dev = _counter(p, seed, offset, x.device)
    rows, cols = x.shape
    y = torch.empty_like(x)             # rows one behind the other
    _enqueue("scout_dropout", x.device.index, code, rows, cols, x.data_ptr(), stride, y.data_ptr(), max(cols, 1), p, seed, host, dev)
    return y


# ---- a block joins the residual stream ----------------------------------------------------------------------

class _Join:
    """What a call needs to know of its arguments' sizes: the library's record and the backward pass's scratch."""
    __slots__ = ("record", "at", "bytes", "rows", "dim", "index")


def _like(a, b) -> bool:
    """Whether b (None, or shape, stride, dtype, device) has the shape and device of a."""
    return b is None or (b[0] == a[0] and b[3] == a[3])


@functools.lru_cache(maxsize=1024)
def _join(block, stream, dn, weights, scale, eps, backward):
    """Checks descriptions (shape, stride, dtype, device, or None) of block; of x, or y and dy; of dn; of gate, post and norm -> _Join."""
    shape, stride, dtype, device = block
    if dtype not in _CODE or len(shape) != 2:
        _fail("block: a float32, bfloat16 or float16 matrix [rows, dim]")
    _row_stride(shape, stride, device, "block")
    types = {s[2] for s in stream if s is not None} or {dtype}
    if len(types) != 1 or not types <= {dtype, torch.float32} or not all(_like(block, s) for s in stream):
        _fail("the residual stream (x, y, dy) has the block's shape and device, and one dtype: the block's or float32")
    for s, name in zip(stream, ("y", "dy") if backward else ("x",)):
        if s is not None:
            _row_stride(s[0], s[1], s[3], name)
    if dn is not None:
        if not _like(block, dn) or dn[2] != dtype:
            _fail("dn has the block's shape, dtype and device")
        _row_stride(dn[0], dn[1], dn[3], "dn")
    rows, dim = shape
    gate, post, norm = weights
    given = [w for w in weights if w is not None]
    wtypes = {w[2] for w in given} or {dtype}
    if len(wtypes) != 1 or not wtypes <= {dtype, torch.float32} or any(w[3] != device or not w[4] for w in given):
        _fail("gate, post_weight and norm_weight are contiguous, on the block's device, and of one dtype: the block's or float32")
    groups = 1
    if gate is not None:
        if len(gate[0]) not in (1, 2) or gate[0][-1] != dim:
            _fail("gate: [dim] or [groups, dim]")
        groups = gate[0][0] if len(gate[0]) == 2 else 1
        if groups == 0 or rows % groups:
            _fail("gate: [groups, dim], the rows being a multiple of groups")
    if any(w is not None and w[0] != (dim,) for w in (post, norm)):
        _fail("post_weight and norm_weight: [dim]")
    if not math.isfinite(scale) or not math.isfinite(eps) or eps < 0:
        _fail("scale and eps: finite, eps not negative")
    if dim == 0:
        _fail("block: a row has at least one element")
    r = _Join()
    row = lambda t: max(t[1][0], dim) if t is not None else dim        # noqa: E731  - a single row's stride says nothing
    r.record = np.zeros(1, dtype=binding.JOIN_DTYPE)
    x, y, dy = (None, *stream) if backward else (stream[0], None, None)
    r.record[0] = (_CODE[dtype], _CODE[next(iter(types))], _CODE[next(iter(wtypes))], scale, eps, 0, rows, dim, groups, row(x), row(block),
                   row(y), dim, row(dy), row(dn), dim, dim)
    r.at = r.record.ctypes.data
    r.bytes = binding.scout_join_backward_workspace(r.at)
    r.rows, r.dim, r.index = rows, dim, device.index
    return r


def _say(x):
    return None if x is None else (x.shape, x.stride(), x.dtype, x.device)


def _say_weight(x):
    return None if x is None else (x.shape, None, x.dtype, x.device, x.is_contiguous())


def _at(x) -> int:
    return 0 if x is None else x.data_ptr()


def join_forward(x: Optional[torch.Tensor], block: torch.Tensor, *, gate: Optional[torch.Tensor] = None,
                 post_weight: Optional[torch.Tensor] = None, norm_weight: Optional[torch.Tensor] = None, scale: float = 1.0,
                 eps: float = 1e-6, p: float = 0.0, seed: int = 0, offset=0):
    """A block's output joins the residual stream, and what the next block reads, in one pass over memory:

        u = dropout(rms_norm(block) * post_weight)      y = x + scale * gate * u      n = rms_norm(y) * norm_weight

    x [rows, dim]: the stream, of block's dtype or float32 (None: 0, y is then of block's dtype).  gate: [dim], or [groups, dim] with
    one row for every rows / groups rows in turn (one per sequence, one per token).  Without post_weight the block is not normed,
    without norm_weight n is None.  p, seed, offset: as in dropout.  dim: up to 16384.
    -> (y, n, stats); stats [2, rows] float32 are the two norms' factors, for the backward pass."""
    _no_autograd(x, block, gate, post_weight, norm_weight)
    j = _join(_say(block), (_say(x),), None, (_say_weight(gate), _say_weight(post_weight), _say_weight(norm_weight)), float(scale),
              float(eps), False)
    p, seed, host, dev = _counter(p, seed, offset, block.device)
    y = torch.empty_like(block if x is None else x)             # rows one behind the other
    n = None if norm_weight is None else torch.empty_like(block)
    stats = block.new_empty((2, j.rows), dtype=torch.float32)
    _enqueue("scout_join_forward", j.index, j.at, _at(x), block.data_ptr(), _at(gate), _at(post_weight), _at(norm_weight), p, seed, host, dev,
             y.data_ptr(), _at(n), stats.data_ptr())
    return y, n, stats


def join_backward(dy: Optional[torch.Tensor], dn: Optional[torch.Tensor], block: torch.Tensor, y: torch.Tensor, stats: torch.Tensor, *,
                  gate: Optional[torch.Tensor] = None, post_weight: Optional[torch.Tensor] = None,
                  norm_weight: Optional[torch.Tensor] = None, scale: float = 1.0, p: float = 0.0, seed: int = 0, offset=0):
    """Gradients of join_forward from dy and dn, those of y and n (None: zero; dn needs norm_weight), block, and what the forward
    pass returned; the other arguments as there.
    -> (dx, dblock, dgate, dpost_weight, dnorm_weight): dx of the stream's dtype, the weights' gradients like the weights, None
    where there is no such weight."""
    _no_autograd(dy, dn, block, y, stats, gate, post_weight, norm_weight)
    if dn is not None and norm_weight is None:
        _fail("dn: without norm_weight there was no n")
    j = _join(_say(block), (_say(y), _say(dy)), _say(dn), (_say_weight(gate), _say_weight(post_weight), _say_weight(norm_weight)),
              float(scale), 0.0, True)
    if stats.dtype != torch.float32 or stats.shape != (2, j.rows) or not stats.is_contiguous() or stats.device != block.device:
        _fail("stats: the forward pass's, a contiguous float32 tensor [2, rows]")
    p, seed, host, dev = _counter(p, seed, offset, block.device)
    dx, db = torch.empty_like(y), torch.empty_like(block)             # rows one behind the other
    dgate = None if gate is None else torch.empty_like(gate)
    dpost = None if post_weight is None else torch.empty_like(post_weight)
    dnorm = None if norm_weight is None else torch.empty_like(norm_weight) if dn is not None else torch.zeros_like(norm_weight)
    ws = block.new_empty(j.bytes, dtype=torch.uint8)
    _enqueue("scout_join_backward", j.index, j.at, _at(dy), _at(dn), block.data_ptr(), y.data_ptr(), stats.data_ptr(), _at(gate),
             _at(post_weight), _at(norm_weight), p, seed, host, dev, dx.data_ptr(), db.data_ptr(), _at(dgate), _at(dpost),
             dnorm.data_ptr() if dnorm is not None and dn is not None else 0, ws.data_ptr(), j.bytes)
    return dx, db, dgate, dpost, dnorm


# ---- cross entropy over a vocabulary ------------------------------------------------------------------------

@functools.lru_cache(maxsize=1024)
def _scores(x_shape, x_stride, w_shape, w_stride, dtype, w_dtype, device, w_device, targets_shape):
    """Checks a description of x, w and targets -> their type's code, rows, dim, vocab, row strides, scratch of both passes."""
    if dtype not in (torch.bfloat16, torch.float16) or w_dtype != dtype or w_device != device:
        _fail("x and w: bfloat16 or float16, of one dtype and on one device")
    x_row, w_row = _row_stride(x_shape, x_stride, device, "x"), _row_stride(w_shape, w_stride, device, "w")
    if x_shape[1] != w_shape[1]:
        _fail("x is [rows, dim], w is [vocab, dim]")
    if targets_shape != x_shape[:1]:
        _fail("targets: one for each row of x")
    code, (rows, dim), vocab = _CODE[dtype], x_shape, w_shape[0]
    if dim == 0:
        _fail("x: a row has at least one element")
    return (code, rows, dim, vocab, x_row, w_row) + binding.scout_loss_workspace(code, rows, dim, vocab)


def _describe_scores(x, w, targets):
    if x.dim() != 2 or w.dim() != 2:
        _fail("x is [rows, dim], w is [vocab, dim]")
    return _scores(x.shape, x.stride(), w.shape, w.stride(), x.dtype, w.dtype, x.device, w.device, targets.shape)


def loss_forward(x: torch.Tensor, w: torch.Tensor, targets: torch.Tensor):
    """Softmax cross entropy of the scores x w^T, which are not kept.  x: [rows, dim] hidden states, w: [vocab, dim] output
    projection (bfloat16 or float16, dim a multiple of 8, rows of w on 16-byte boundaries); targets: int32 or int64 [rows].
    Rows whose target is outside 0..vocab-1 (padding) do not count, and nothing is read from them.
    -> (loss, lse), float32 [rows]: lse is the logarithm of the sum of exponentials, for the backward pass; both are 0 for rows
    that do not count."""
    _no_autograd(x, w)
    code, rows, dim, vocab, x_row, w_row, nbytes, _ = _describe_scores(x, w, targets)
    targets = _flat_ids(targets, x.device, "targets")
    loss = x.new_empty(rows, dtype=torch.float32)
    lse = torch.empty_like(loss)
    ws = x.new_empty(nbytes, dtype=torch.uint8)
    _enqueue("scout_loss_forward", x.device.index, code, _IDS[targets.dtype], rows, dim, vocab, x.data_ptr(), x_row, w.data_ptr(), w_row,
             targets.data_ptr(), loss.data_ptr(), lse.data_ptr(), ws.data_ptr(), nbytes)
    return loss, lse


def loss_backward(x: torch.Tensor, w: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor, dloss: torch.Tensor, *,
                  out_dtype: Optional[torch.dtype] = None, grad: Optional[torch.Tensor] = None):
    """Gradients of loss_forward's loss with respect to x and w, from its lse and the gradient dloss (float32 [rows], of any stride:
    a mean over the batch has one number, expanded).
    -> (dx like x, dw [vocab, dim] in out_dtype: float32, which is the default, or w's); with `grad` (of those dtypes, of a tied
    embedding, say) dw is added to it in place, and out_dtype may only repeat its dtype.
    The gradient of the scores is rounded to x's type for its products, so a float32 dw is as exact as its terms are (2^-8 of
    each in bfloat16, 2^-11 in float16), not as float32 is.  What that takes from a token's own target is given back: all of it to
    dx, and to a row of dw that of two of its tokens.  In float16 dw's terms are rounded relative to the largest dloss: of a row that weighs
    2^-27 of that little is left there, and all of it in its dx."""
    _no_autograd(x, w, lse, dloss, grad)
    code, rows, dim, vocab, x_row, w_row, _, nbytes = _describe_scores(x, w, targets)
    targets = _flat_ids(targets, x.device, "targets")
    for t, name in ((lse, "lse"), (dloss, "dloss")):
        if t.dtype != torch.float32 or t.shape != (rows,) or t.device != x.device:
            _fail(f"{name}: float32 [rows], on x's device")
    if not lse.is_contiguous():
        lse = lse.contiguous()
    if grad is None:
        dw = w.new_empty((vocab, dim), dtype=out_dtype or torch.float32)
    else:
        if out_dtype not in (None, grad.dtype):
            _fail("grad is added to in its own dtype; out_dtype names another")
        dw = grad
    if dw.dtype not in (torch.float32, w.dtype) or dw.shape != (vocab, dim) or dw.device != x.device:
        _fail("the gradient is [vocab, dim], float32 or of w's dtype, on x's device")
    dw_row = _row_stride(dw.shape, dw.stride(), dw.device, "grad")
    dx = torch.empty_like(x)             # rows one behind the other
    ws = x.new_empty(nbytes, dtype=torch.uint8)
    _enqueue("scout_loss_backward", x.device.index, code, _IDS[targets.dtype], _CODE[dw.dtype], rows, dim, vocab, x.data_ptr(), x_row,
             w.data_ptr(), w_row, targets.data_ptr(), lse.data_ptr(), dloss.data_ptr(), dloss.stride(0), dx.data_ptr(), dim, dw.data_ptr(),
             dw_row, int(grad is not None), ws.data_ptr(), nbytes)
    return dx, dw
