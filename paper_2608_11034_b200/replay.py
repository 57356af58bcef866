"""Operators of one replayed transformer layer, on torch tensors.

In-situ replay (Sec. 6 of the paper) runs a layer again on every peer from the
same captured inputs; exact consensus then compares the output and the gradients
bit by bit.  The operators here give the same bits on every healthy GPU: no
floating-point atomics, every sum in an order that the sizes alone fix.

    attention_forward, attention_backward   softmax attention and its gradient
    checkpoint_pack, checkpoint_unpack      captured activations held in 8 bits
    checkpoint_wgrad                        a projection's weight gradient, straight
                                            from such a checkpoint

Each call checks its arguments, allocates outputs and scratch from torch's
allocator on the current stream and enqueues the library's kernels there
(``include/scout_replay.h`` has the definitions).  Tensors are used where they
lie: as usual in torch, one made on another stream needs that stream's work
waited for, and ``record_stream`` if it is freed early.

None of the calls is recorded by autograd.  Where it would be asked to (grad mode on,
an input of attention or of the weight gradient that requires a gradient), they raise
instead of dropping the gradient: call them under torch.no_grad(), or from the
forward and backward of a torch.autograd.Function, where grad mode is off.

The kernels' waits are bounded.  A call in which one gave up has no valid results, and
cannot say so itself, since it only enqueues: ``with waits_checked(device):`` around
the calls raises WaitGaveUp before anybody signs or votes on what they left.
"""
from __future__ import annotations

import contextlib
import functools
import math
from typing import Optional

import numpy as np
import torch

from . import binding

_CODE = {torch.float32: binding.DT_F32, torch.bfloat16: binding.DT_BF16, torch.float16: binding.DT_F16}
_SIXTEEN = (torch.bfloat16, torch.float16)


class WaitGaveUp(RuntimeError):
    """A wait of a replay kernel ran into its limit: what the calls since the last check left is not valid."""


@contextlib.contextmanager
def waits_checked(device: torch.device):
    """Raises WaitGaveUp if a wait of the replay kernels gave up on `device` between entry and exit, on any of its streams
    (synchronises the device at both).  While a CUDA graph is captured nothing runs and nothing is checked: that is for
    whoever replays the graph."""
    if torch.cuda.is_initialized() and torch.cuda.is_current_stream_capturing():
        yield
        return
    with torch.cuda.device(device):
        before = binding.scout_replay_waits()
    yield
    with torch.cuda.device(device):
        n = (binding.scout_replay_waits() - before) % (1 << 32)
    if n:
        raise WaitGaveUp(f"{n} waits of the replay kernels gave up on {device}: the results are not valid")


def _fail(what: str):
    raise ValueError(what)


def _no_autograd(*tensors) -> None:
    if torch.is_grad_enabled() and any(x.requires_grad for x in tensors):
        _fail("autograd does not record this call: use torch.no_grad() or a torch.autograd.Function")


class _Attention:
    """What a call needs to know of its arguments' sizes: the library's record and the scratch of both passes."""
    __slots__ = ("record", "at", "forward_bytes", "backward_bytes", "batch", "rows", "index")


@functools.lru_cache(maxsize=1024)
def _attention(dtypes, devices, qs, ks, vs, os, gs, q_stride, k_stride, v_stride, o_stride, g_stride, causal, window, scale):
    """Checks a description of q, k, v, o, do (sizes only, no data) -> _Attention."""
    if len(qs) != 4 or len(ks) != 4 or ks != vs:
        _fail("q is [batch, q_len, q_heads, head_dim], k and v are [batch, kv_len, kv_heads, head_dim]")
    b, tq, hq, d = qs
    if ks[0] != b or ks[3] != d:
        _fail("q and k differ in batch or head_dim")
    if os != qs or gs != qs:
        _fail("o and do must have the shape of q")
    if dtypes[0] not in _SIXTEEN:
        _fail("attention takes bfloat16 or float16")
    if len(set(dtypes)) != 1 or len(set(devices)) != 1:
        _fail("q, k, v, o and do must share one dtype and device")
    if devices[0].type != "cuda":
        _fail("tensors must be on a CUDA device")
    if window < 0:
        _fail("window: 0 (all) or a number of tokens")
    strides = (q_stride, k_stride, v_stride, o_stride, g_stride)
    if d > 1 and any(st[3] != 1 for st in strides):
        _fail("a head's elements must be adjacent (last stride 1)")
    r = _Attention()
    r.record = np.zeros(1, dtype=binding.ATTN_DTYPE)
    r.record[0] = (_CODE[dtypes[0]], b, tq, ks[1], hq, ks[2], d, int(bool(causal)), int(window),
                   1.0 / math.sqrt(d) if scale is None and d else float(scale or 0.0)) + tuple(st[:3] for st in strides)
    r.at = r.record.ctypes.data
    r.forward_bytes, r.backward_bytes = binding.scout_attn_workspace(r.at)
    r.batch, r.rows, r.index = b, (b, hq, tq), devices[0].index
    return r


def _lens(x, batch, device, name) -> int:
    if x is None:
        return 0
    if x.dtype != torch.int32 or x.shape != (batch,) or x.device != device or not x.is_contiguous():
        _fail(f"{name}: a contiguous int32 tensor [batch] on the queries' device is wanted")
    return x.data_ptr()


def _enqueue(name: str, index: int, *args) -> None:
    """The library's call `name` with args and the current stream of the tensors' device, which is made current for it."""
    now = torch._C._cuda_getDevice()
    if now == index:
        rc = getattr(binding.lib(), name)(*args, torch._C._cuda_getCurrentRawStream(index))
    else:
        torch.cuda.set_device(index)
        try:
            rc = getattr(binding.lib(), name)(*args, torch._C._cuda_getCurrentRawStream(index))
        finally:
            torch.cuda.set_device(now)
    if rc:
        raise binding.ScoutError(rc, name)


def attention_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *, causal: bool = False, window: int = 0,
                      scale: Optional[float] = None, q_lens: Optional[torch.Tensor] = None,
                      kv_lens: Optional[torch.Tensor] = None):
    """Softmax attention.  q: [batch, q_len, q_heads, head_dim], k, v: [batch, kv_len, kv_heads, head_dim]
    (bfloat16 or float16; any strides that are multiples of 8 elements, last axis adjacent); query head h
    reads key head h // (q_heads // kv_heads).

    causal: a row sees the keys up to its own position, the last row standing at the last key.
    window: with causal, only its own position and the window - 1 before it (0: all).
    q_lens, kv_lens: int32 [batch], the tokens in use of padded sequences.
    -> (o like q, lse float32 [batch, q_heads, q_len]); rows that see nothing give 0 and -inf."""
    _no_autograd(q, k, v)
    o = torch.empty_like(q)
    shape = q.shape
    t = _attention((q.dtype, k.dtype, v.dtype), (q.device, k.device, v.device), shape, k.shape, v.shape, shape, shape,
                   q.stride(), k.stride(), v.stride(), o.stride(), o.stride(), causal, window, scale if scale is None else float(scale))
    lse = q.new_empty(t.rows, dtype=torch.float32)
    ql, kl = _lens(q_lens, t.batch, q.device, "q_lens"), _lens(kv_lens, t.batch, q.device, "kv_lens")
    ws = q.new_empty(t.forward_bytes, dtype=torch.uint8) if t.forward_bytes else None
    _enqueue("scout_attn_forward", t.index, t.at, q.data_ptr(), k.data_ptr(), v.data_ptr(), ql, kl, o.data_ptr(), lse.data_ptr(),
             ws.data_ptr() if ws is not None else 0, t.forward_bytes)
    return o, lse


def attention_backward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor, lse: torch.Tensor,
                       do: torch.Tensor, *, causal: bool = False, window: int = 0, scale: Optional[float] = None,
                       q_lens: Optional[torch.Tensor] = None, kv_lens: Optional[torch.Tensor] = None, grads=None):
    """Gradients of attention_forward's o with respect to q, k and v, from the gradient `do` of o and what the
    forward pass returned; the other arguments as there.  Gradients of key heads that several query heads share are
    summed over those.  -> (dq, dk, dv), laid out like q, k, v.

    grads: the three tensors to write, which q, k and v that are parts of one projection's output need: the same parts of a
    gradient laid out like that output.  They do not overlap."""
    _no_autograd(q, k, v, o, do, *(grads or ()))
    t = _attention((q.dtype, k.dtype, v.dtype, o.dtype, do.dtype), (q.device, k.device, v.device, o.device, do.device), q.shape,
                   k.shape, v.shape, o.shape, do.shape, q.stride(), k.stride(), v.stride(), o.stride(), do.stride(), causal, window,
                   scale if scale is None else float(scale))
    dq, dk, dv = (torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)) if grads is None else grads
    for x, y, name in ((q, dq, "q"), (k, dk, "k"), (v, dv, "v")):
        if grads is not None and (y.shape != x.shape or y.dtype != x.dtype or y.device != x.device):
            _fail(f"grads: d{name} has the shape, dtype and device of {name}")
        if x.stride() != y.stride():
            _fail(f"{name}: overlapping or gapped memory has no gradient laid out like it; pass {name}.contiguous(), or grads")
    if lse.dtype != torch.float32 or lse.shape != t.rows or not lse.is_contiguous() or lse.device != q.device:
        _fail("lse: the forward pass's, a contiguous float32 tensor [batch, q_heads, q_len]")
    ql, kl = _lens(q_lens, t.batch, q.device, "q_lens"), _lens(kv_lens, t.batch, q.device, "kv_lens")
    ws = q.new_empty(t.backward_bytes, dtype=torch.uint8) if t.backward_bytes else None
    _enqueue("scout_attn_backward", t.index, t.at, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(),
             do.data_ptr(), ql, kl, dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), ws.data_ptr() if ws is not None else 0,
             t.backward_bytes)
    return dq, dk, dv


def _row_stride(shape, stride, device, name) -> int:
    if len(shape) != 2 or (shape[1] > 1 and stride[1] != 1) or (shape[0] > 1 and stride[0] < shape[1]):
        _fail(f"{name}: a matrix with adjacent row elements is wanted")
    if device.type != "cuda":
        _fail("tensors must be on a CUDA device")
    return max(stride[0], shape[1], 1)


@functools.lru_cache(maxsize=1024)
def _activation(shape, stride, dtype, device):
    """Checks a description of x (sizes only) -> its type's code, rows, columns, row stride, shape of the exponents."""
    if dtype not in _CODE:
        _fail("activations are float32, bfloat16 or float16")
    row = _row_stride(shape, stride, device, "x")
    return _CODE[dtype], shape[0], shape[1], row, (shape[0], -(-shape[1] // binding.CKPT_BLOCK))


@functools.lru_cache(maxsize=1024)
def _checkpoint(shape, stride, dtype, device, exps_shape, exps_stride, exps_dtype, exps_device):
    """Checks a description of a checkpoint -> rows, columns, row stride of the codes."""
    row = _row_stride(shape, stride, device, "codes")
    blocks = -(-shape[1] // binding.CKPT_BLOCK)
    if dtype != torch.int8 or exps_dtype != torch.int8 or exps_device != device or exps_shape != (shape[0], blocks) or \
            (shape[0] > 1 and blocks > 0 and exps_stride[0] != blocks) or (blocks > 1 and exps_stride[1] != 1):
        _fail("codes: int8 [rows, cols], exps: contiguous int8 [rows, ceil(cols / 32)]")
    return shape[0], shape[1], row


def checkpoint_pack(x: torch.Tensor):
    """Hold the activation x [rows, cols] (float32, bfloat16 or float16) in 8 bits.
    -> (codes int8 [rows, cols], exps int8 [rows, ceil(cols / 32)]): x is about codes * 2**exps, exps per block of 32 columns."""
    code, rows, cols, stride, exps_shape = _activation(x.shape, x.stride(), x.dtype, x.device)
    codes, exps = x.new_empty((rows, cols), dtype=torch.int8), x.new_empty(exps_shape, dtype=torch.int8)
    _enqueue("scout_ckpt_pack", x.device.index, code, rows, cols, x.data_ptr(), stride, codes.data_ptr(), max(cols, 1),
             exps.data_ptr())
    return codes, exps


def checkpoint_unpack(codes: torch.Tensor, exps: torch.Tensor, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """The activation a checkpoint stands for, in `dtype`."""
    rows, cols, stride = _checkpoint(codes.shape, codes.stride(), codes.dtype, codes.device, exps.shape, exps.stride(), exps.dtype,
                                     exps.device)
    if dtype not in _CODE:
        _fail("activations are float32, bfloat16 or float16")
    x = codes.new_empty((rows, cols), dtype=dtype)
    _enqueue("scout_ckpt_unpack", codes.device.index, _CODE[dtype], rows, cols, codes.data_ptr(), stride, exps.data_ptr(),
             x.data_ptr(), max(cols, 1))
    return x


@functools.lru_cache(maxsize=1024)
def _product(shape, stride, dtype, device, rows, codes_device, ins, dw_shape, dw_stride, dw_dtype, dw_device):
    """Checks a description of dy and the gradient -> their codes, outputs, row strides, scratch bytes."""
    row = _row_stride(shape, stride, device, "dy")
    if dtype not in _SIXTEEN or shape[0] != rows or device != codes_device:
        _fail("dy: a bfloat16 or float16 matrix with the checkpoint's rows, on its device")
    outs = shape[1]
    if dw_dtype not in (torch.float32, dtype) or dw_shape != (outs, ins) or dw_device != device:
        _fail("the gradient is [outs, ins], float32 or of dy's dtype, on dy's device")
    dw_row = _row_stride(dw_shape, dw_stride, dw_device, "grad")
    return _CODE[dtype], _CODE[dw_dtype], outs, row, dw_row, binding.scout_ckpt_wgrad_workspace(_CODE[dtype], rows, outs, ins)


def checkpoint_wgrad(dy: torch.Tensor, codes: torch.Tensor, exps: torch.Tensor, *, out_dtype: Optional[torch.dtype] = None,
                     grad: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Weight gradient dW = dy^T x of y = x W^T, x taken from its checkpoint.  dy: [rows, outs], bfloat16 or float16.
    -> dW [outs, ins] in out_dtype (float32, which is the default, or dy's); with `grad` (of those dtypes) dW is added to it in
    place, and out_dtype may only repeat its dtype."""
    rows, ins, code_stride = _checkpoint(codes.shape, codes.stride(), codes.dtype, codes.device, exps.shape, exps.stride(),
                                         exps.dtype, exps.device)
    _no_autograd(dy) if grad is None else _no_autograd(dy, grad)
    if dy.dim() != 2:
        _fail("dy: a matrix with adjacent row elements is wanted")
    if grad is None:
        dw = dy.new_empty((dy.shape[1], ins), dtype=out_dtype or torch.float32)
    else:
        if out_dtype not in (None, grad.dtype):
            _fail("grad is added to in its own dtype; out_dtype names another")
        dw = grad
    code, dw_code, outs, dy_stride, dw_stride, nbytes = _product(dy.shape, dy.stride(), dy.dtype, dy.device, rows, codes.device, ins,
                                                                 dw.shape, dw.stride(), dw.dtype, dw.device)
    ws = dy.new_empty(nbytes, dtype=torch.uint8) if nbytes else None
    _enqueue("scout_ckpt_wgrad", dy.device.index, code, dw_code, rows, outs, ins, dy.data_ptr(), dy_stride, codes.data_ptr(),
             code_stride, exps.data_ptr(), dw.data_ptr(), dw_stride, int(grad is not None),
             ws.data_ptr() if ws is not None else 0, nbytes)
    return dw
