"""Operators of a training step around the optimizer, on libmalt's HIP kernels:

  embedding, embedding_grad            rows of a token table, scaled, and the table's gradient
  distill_loss, distill_step           loss against a teacher's top logits (and labels), and its gradient
  fp8_linear                           a linear layer in 8-bit floating point, with its backward pass
  fp8_quantize_weight, fp8_forward     the same layer on kept 8-bit weights
  linear_cross_entropy, linear_cross_entropy_step
                                       loss of a linear head over a large vocabulary without its logits, and its gradients
  rms_norm, rms_norm_fp8               norm of x + residual, with its backward pass, and with its output in 8 bits
  adamw_state, adamw_step, adamw_moments
                                       one AdamW step over many tensors, moments in 32 bits or in 8

The definitions stand in include/libmalt.h.  This module checks arguments,
allocates outputs and workspaces with torch, and calls the library; there is
no CPU fallback.  Wrong arguments raise ValueError (TypeError for what is no
tensor) before anything is enqueued, what only the library tells (buffers that
overlap, sizes past its limits) libmalt's MaltError.  "Differentiable" means reverse mode, once; a
tangent of forward mode is refused there.  A captured backward pass of the head's loss or the norm is
refused where it would go on in a graph of the default stream (an eager graph of the same leaves
that still lives): no capture survives that.

Work runs on the current stream of the tensors' device, or on `stream`; the
caller orders that stream after whatever produces the inputs.  Outputs and
workspaces belong to the stream the work runs on.  Tensors whose rows are not
contiguous are copied first, on that stream too; row pitches larger than a row are
taken as they are up to 2^31 - 1 elements, as are those of outputs.
"""
from __future__ import annotations

import functools
from ctypes import byref, c_size_t
from typing import List, NamedTuple, Optional, Sequence, Tuple, Union

import torch
from torch.autograd import forward_ad as _forward_ad

from . import libmalt as lm

_DTYPES = {torch.float32: lm.MALT_FLOAT32, torch.bfloat16: lm.MALT_BFLOAT16}
_INDEX = {torch.int32: lm.MALT_INT32, torch.int64: lm.MALT_INT64}
BLOCK = 128   # values that share a scale
MAX_PITCH = (1 << 31) - 1   # elements between two rows


# ------------------------------------------------------------------ arguments
def _tensor(name: str, x, types, device=None) -> None:
    try:
        if x.dtype in types and x.is_cuda and (device is None or x.device == device):
            return
    except AttributeError:
        pass
    if not isinstance(x, torch.Tensor):
        raise TypeError(f"{name} must be a tensor (got {type(x).__name__})")
    if x.dtype not in types:
        raise ValueError(f"{name} must be {' or '.join(str(t).replace('torch.', '') for t in types)} (got {x.dtype})")
    if not x.is_cuda:
        raise ValueError(f"{name} must be on a GPU (got {x.device})")
    if device is not None and x.device != device:
        raise ValueError(f"{name} is on {x.device}, the other tensors on {device}")


def _type(name: str, dtype) -> int:
    if dtype not in _DTYPES:
        raise ValueError(f"{name} must be float32 or bfloat16 (got {dtype})")
    return _DTYPES[dtype]


def _rows(x: torch.Tensor) -> Tuple[torch.Tensor, int]:
    """A 2-D tensor whose rows are contiguous, do not overlap and lie no further apart
    than the library takes, and its row pitch."""
    r, c = x.shape
    if x.is_contiguous():
        return x, c
    if (c > 1 and x.stride(1) != 1) or (r > 1 and not c <= x.stride(0) <= MAX_PITCH):
        x = x.contiguous()
    return x, (x.stride(0) if r > 1 else c)


def _no_stream(stream) -> None:
    """A differentiable call follows the current stream, as its backward pass will."""
    if stream is not None:
        raise ValueError("a differentiable call takes no stream: make it within torch.cuda.stream(...)")


def _no_tangent(name: str, x) -> None:
    """Forward-mode derivatives are not defined: a tangent would be lost without a word."""
    # The level is -1 outside forward mode; asked first, it costs 0.05 us a call instead of 0.3.
    if _forward_ad._current_level >= 0 and _forward_ad.unpack_dual(x).tangent is not None:
        raise ValueError(f"{name} has a tangent, but only reverse-mode derivatives are defined")


def _flat(x: torch.Tensor) -> torch.Tensor:
    """All but the last dimension as one."""
    return x if x.dim() == 2 else x.reshape(-1, x.shape[-1])


# The current device and its current stream, as numbers.
_current_device = torch.cuda.current_device
_current_stream = torch._C._cuda_getCurrentRawStream


def _on(device: torch.device, stream, inputs, work):
    """work(stream handle) with `device` and `stream` current, so that what it
    allocates and copies belongs to them.  `inputs` are the caller's tensors."""
    if stream is None:
        if device.index == _current_device():
            return work(_current_stream(device.index))
        with torch.cuda.device(device):
            return work(_current_stream(device.index))
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=device)
    if stream.device != device:
        raise ValueError(f"the stream belongs to {stream.device}, the tensors to {device}")
    for x in inputs:   # their memory is not handed out again before this work is done
        if x is not None:
            x.record_stream(stream)
    with torch.cuda.stream(stream):
        return work(stream.cuda_stream)


def _written(out: Optional[torch.Tensor]) -> None:
    """Tells autograd that a caller's tensor holds new values, so that a backward
    pass which had saved it raises.  (What was made in inference mode is never saved.)"""
    if out is not None and not out.is_inference():
        torch.autograd.graph.increment_version(out)


# ------------------------------------------------------------------ embedding
def _lookup(ids, weight, scale, out_dtype, stream):
    v, w = weight.shape
    dev = weight.device

    def work(s):
        flat = ids if ids.is_contiguous() else ids.contiguous()
        table, ld = _rows(weight)
        out = torch.empty((*ids.shape, w), dtype=out_dtype, device=dev)
        lm._check(lm.lib().malt_embed_lookup(flat.data_ptr(), _INDEX[flat.dtype], flat.numel(), table.data_ptr(),
                                             _DTYPES[table.dtype], v, w, ld, scale, out.data_ptr(), _DTYPES[out_dtype],
                                             w, s))
        return out

    return _on(dev, stream, (ids, weight), work)


@functools.lru_cache(maxsize=4096)
def _embed_grad_size(tokens: int, vocab: int, width: int) -> int:
    size = c_size_t(0)
    lm._check(lm.lib().malt_embed_grad_size(tokens, vocab, width, byref(size)))
    return size.value


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ids, weight, scale, out_dtype):
        ctx.save_for_backward(ids)
        ctx.args = (weight.shape[0], scale, weight.dtype)
        return _lookup(ids, weight, scale, out_dtype, None)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        (ids,) = ctx.saved_tensors
        rows, scale, dtype = ctx.args
        if grad.dtype not in _DTYPES:
            grad = grad.float()
        return None, embedding_grad(ids, grad, rows, scale=scale, dtype=dtype), None, None


def embedding(ids: torch.Tensor, weight: torch.Tensor, scale: float = 1.0, out_dtype: Optional[torch.dtype] = None,
              stream=None) -> torch.Tensor:
    """scale * weight[ids], shape ids.shape + (width,); zeros for ids outside
    the table.  weight: (vocab, width) float32 or bfloat16; ids: int32 or int64
    of any shape; out_dtype: weight's unless given.  Differentiable in weight
    (the gradient is dense, of weight's type, see embedding_grad)."""
    _tensor("weight", weight, _DTYPES)
    if weight.dim() != 2 or weight.numel() < 1:
        raise ValueError(f"weight must be (vocab, width) (got {tuple(weight.shape)})")
    _no_tangent("weight", weight)
    _tensor("ids", ids, _INDEX, weight.device)
    if out_dtype is None:
        out_dtype = weight.dtype
    else:
        _type("out_dtype", out_dtype)
    scale = float(scale)
    if weight.requires_grad and torch.is_grad_enabled():
        _no_stream(stream)
        return _Embedding.apply(ids, weight, scale, out_dtype)
    return _lookup(ids, weight, scale, out_dtype, stream)


def embedding_grad(ids: torch.Tensor, grad: torch.Tensor, num_rows: int, scale: float = 1.0,
                   dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None, accumulate: bool = False,
                   stream=None) -> torch.Tensor:
    """Gradient of a (num_rows, width) table: row v is scale times the sum of
    grad over the tokens with id v, in float32 and in the tokens' order (equal
    inputs give equal bits).  grad: ids.shape + (width,).  Written to `out`
    (contiguous rows) when given, with accumulate added to it; otherwise to a
    new tensor of `dtype` (default: grad's).  To autograd, `out` is changed in place."""
    _tensor("grad", grad, _DTYPES)
    dev = grad.device
    _tensor("ids", ids, _INDEX, dev)
    if grad.dim() < 1 or tuple(grad.shape[:-1]) != tuple(ids.shape):
        raise ValueError(f"grad must be ids.shape + (width,) (got {tuple(grad.shape)} for ids {tuple(ids.shape)})")
    w = grad.shape[-1]
    if num_rows < 1 or w < 1:
        raise ValueError(f"the table must have rows and columns (got {num_rows} x {w})")
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs out")
        dtype = grad.dtype if dtype is None else dtype
        _type("dtype", dtype)
    else:
        _tensor("out", out, _DTYPES, dev)
        if tuple(out.shape) != (num_rows, w) or (w > 1 and out.stride(1) != 1) or (num_rows > 1 and out.stride(0) < w):
            raise ValueError(f"out must be ({num_rows}, {w}) with contiguous rows (got {tuple(out.shape)}, "
                             f"strides {out.stride()})")
        if dtype is not None and dtype != out.dtype:
            raise ValueError(f"dtype {dtype} differs from out's {out.dtype}")
    n = ids.numel()
    size = _embed_grad_size(n, num_rows, w)

    def work(s):
        flat = ids.reshape(-1).contiguous()
        g, ld = _rows(grad.reshape(-1, w))
        d = torch.empty((num_rows, w), dtype=dtype, device=dev) if out is None else out
        ws = torch.empty(size, dtype=torch.uint8, device=dev) if size else None
        lm._check(lm.lib().malt_embed_grad(flat.data_ptr(), _INDEX[flat.dtype], n, g.data_ptr(), _DTYPES[g.dtype], ld,
                                           float(scale), int(bool(accumulate)), d.data_ptr(), _DTYPES[d.dtype],
                                           num_rows, w, d.stride(0) if num_rows > 1 else w,
                                           None if ws is None else ws.data_ptr(), size, s))
        return d

    result = _on(dev, stream, (ids, grad, out), work)
    _written(out)
    return result


# --------------------------------------------------------------- distillation
def _distill(logits, top_logits, top_ids, labels, tau, alpha, weight, want_loss, want_grad, out, stream):
    _tensor("logits", logits, _DTYPES)
    dev = logits.device
    if logits.dim() < 1 or logits.shape[-1] < 1:
        raise ValueError(f"logits must be (..., vocab) (got {tuple(logits.shape)})")
    lead, v = logits.shape[:-1], logits.shape[-1]
    tau, alpha = float(tau), float(alpha)
    if not 2.0 ** -60 <= tau <= 2.0 ** 60:
        raise ValueError(f"tau must be in [2^-60, 2^60] (got {tau})")
    if not 0 <= alpha <= 1:
        raise ValueError(f"alpha must be in [0, 1] (got {alpha})")
    n = lead.numel()
    k = 0
    if (top_logits is None) != (top_ids is None):
        raise ValueError("top_logits and top_ids come together")
    if top_logits is not None:
        _tensor("top_logits", top_logits, _DTYPES, dev)
        _tensor("top_ids", top_ids, _INDEX, dev)
        if top_logits.shape[:-1] != lead or top_logits.shape != top_ids.shape:
            raise ValueError(f"top_logits and top_ids must be {tuple(lead)} + (k,) (got {tuple(top_logits.shape)}, "
                             f"{tuple(top_ids.shape)})")
        k = top_logits.shape[-1]
        if k > lm.DISTILL_MAX_TOP:
            raise ValueError(f"at most {lm.DISTILL_MAX_TOP} teacher entries a row (got {k})")
    if labels is not None:
        _tensor("labels", labels, _INDEX, dev)
        if labels.shape != lead:
            raise ValueError(f"labels must be {tuple(lead)} (got {tuple(labels.shape)})")
    weights = None
    if isinstance(weight, torch.Tensor):
        _tensor("grad", weight, (torch.float32,), dev)
        if weight.dim() > 0 and weight.shape != lead:
            raise ValueError(f"grad must be a number, a scalar tensor or {tuple(lead)} (got {tuple(weight.shape)})")
        weights, weight = weight, 1.0
    else:
        weight = float(weight)
    d, dld = None, v
    if out is not None:
        _tensor("out", out, (logits.dtype,), dev)
        if out.shape != logits.shape:
            raise ValueError(f"out must be {tuple(logits.shape)} (got {tuple(out.shape)})")
        d = out if out.dim() == 2 else out.view(-1, v)   # a view, or an error: the result is written through it
        if (v > 1 and d.stride(1) != 1) or (n > 1 and d.stride(0) < v):
            raise ValueError(f"out must have contiguous rows (got strides {out.stride()})")
        dld = d.stride(0) if n > 1 else v

    def work(s):
        losses = torch.empty(lead, dtype=torch.float32, device=dev) if want_loss else None
        grad = out
        if want_grad and out is None:
            grad = torch.empty_like(logits, memory_format=torch.contiguous_format)
        if n == 0:
            return losses, grad
        z, ld = _rows(_flat(logits) if logits.dim() > 1 else logits.reshape(1, v))
        # Teacher, labels and weights: pointers, types and pitches.
        tp = ip = yp = wp = None
        tt = it = tld = ild = yt = y_stride = w_stride = 0
        if k > 0:
            t, tld = _rows(top_logits if top_logits.dim() == 2 else top_logits.reshape(n, k))
            i, ild = _rows(top_ids if top_ids.dim() == 2 else top_ids.reshape(n, k))
            tp, tt, ip, it = t.data_ptr(), _DTYPES[t.dtype], i.data_ptr(), _INDEX[i.dtype]
        if labels is not None:
            y = labels if labels.dim() == 1 else labels.reshape(-1)
            yp, yt, y_stride = y.data_ptr(), _INDEX[y.dtype], (y.stride(0) if n > 1 else 0)
        if weights is not None:
            w = weights if weights.dim() < 2 else weights.reshape(-1)
            wp, w_stride = w.data_ptr(), (w.stride(0) if n > 1 and w.dim() else 0)
        a = lm.malt_distill_t(z.data_ptr(), _DTYPES[z.dtype], n, v, ld, tp, tt, ip, it, k, tld, ild, yp, yt, y_stride,
                              tau, alpha, wp, w_stride, weight, losses.data_ptr() if want_loss else None,
                              (grad if d is None else d).data_ptr() if want_grad else None, dld)
        lm._check(lm.lib().malt_distill(byref(a), s))
        return losses, grad

    result = _on(dev, stream, (logits, top_logits, top_ids, labels, weights, out), work)
    _written(out)
    return result


class _DistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, top_logits, top_ids, labels, tau, alpha):
        ctx.save_for_backward(logits, top_logits, top_ids, labels)
        ctx.args = (tau, alpha)
        return _distill(logits, top_logits, top_ids, labels, tau, alpha, 1.0, True, False, None, None)[0]

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        logits, top_logits, top_ids, labels = ctx.saved_tensors
        # The row is read once for its sums and gradient together: nothing but the inputs was kept.
        d = _distill(logits, top_logits, top_ids, labels, *ctx.args, grad.float(), False, True, None, None)[1]
        return d, None, None, None, None, None


def distill_loss(logits: torch.Tensor, top_logits: Optional[torch.Tensor], top_ids: Optional[torch.Tensor],
                 labels: Optional[torch.Tensor] = None, tau: float = 1.0, alpha: float = 0.0,
                 stream=None) -> torch.Tensor:
    """Loss of each row of student logits (..., vocab) against a teacher's top
    logits (..., k) at top_ids, float32 of shape (...):
    (1 - alpha) tau^2 KL(p || q) + alpha * cross entropy of `labels`, where
    p = softmax(top_logits / tau) over the valid entries and
    q = softmax(logits / tau) over the vocabulary.  Ids and labels outside the
    vocabulary (-1, -100) are no entries and no labels; a part that a row lacks
    is zero.  Differentiable in logits."""
    if isinstance(logits, torch.Tensor):
        _no_tangent("logits", logits)
    if isinstance(logits, torch.Tensor) and logits.requires_grad and torch.is_grad_enabled():
        _no_stream(stream)
        return _DistillLoss.apply(logits, top_logits, top_ids, labels, tau, alpha)
    return _distill(logits, top_logits, top_ids, labels, tau, alpha, 1.0, True, False, None, stream)[0]


def distill_step(logits: torch.Tensor, top_logits: Optional[torch.Tensor], top_ids: Optional[torch.Tensor],
                 labels: Optional[torch.Tensor] = None, tau: float = 1.0, alpha: float = 0.0,
                 grad: Union[float, torch.Tensor] = 1.0, out: Optional[torch.Tensor] = None,
                 stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The losses of distill_loss and the gradient of sum(grad * losses) to the
    logits, in one pass over the logits.  grad: a number, a float32 scalar
    tensor or one weight for each row (0: no gradient).  The gradient goes to
    `out` when given, which may be `logits` itself and is changed in place to autograd:
    a backward pass that saved it raises."""
    if isinstance(logits, torch.Tensor) and logits.requires_grad:
        logits = logits.detach()
    return _distill(logits, top_logits, top_ids, labels, tau, alpha, grad, True, True, out, stream)


# --------------------------------------------------------------- 8-bit linear
def _pad(n: int, to: int) -> int:
    return -(-n // to) * to


def _quantize_weight(w, s) -> Tuple[torch.Tensor, torch.Tensor]:
    """A weight's values and block scales."""
    w, ld = _rows(w)
    r, c = w.shape
    values = torch.empty((r, _pad(c, BLOCK)), dtype=torch.uint8, device=w.device)
    scales = torch.empty((-(-r // BLOCK), -(-c // BLOCK)), dtype=torch.uint8, device=w.device)
    lm._check(lm.lib().malt_block_quantize_weight(w.data_ptr(), _DTYPES[w.dtype], r, c, ld, values.data_ptr(),
                                                  scales.data_ptr(), None, s))
    return values, scales


@functools.lru_cache(maxsize=4096)
def _linear_size(m: int, n: int, k: int, out_type: int) -> int:
    size = c_size_t(0)
    lm._check(lm.lib().malt_block_linear_size(m, n, k, out_type, byref(size)))
    return size.value


@functools.lru_cache(maxsize=4096)
def _layer_sizes(m: int, n: int, k: int, transposed: bool, types: Tuple[int, int, int], need_x: bool,
                 need_w: bool) -> Tuple[int, int, int]:
    """Bytes kept for the backward pass, and of the workspaces of both passes."""
    sizes = (c_size_t(0), c_size_t(0), c_size_t(0))
    lm._check(lm.lib().malt_block_layer_size(m, n, k, transposed, *types, need_x, need_w, *map(byref, sizes)))
    return tuple(s.value for s in sizes)


def _layer_forward(x, weight, transposed, out_dtype, need_x, need_w, stream):
    """The layer's output, what its backward pass needs, and the bytes of the buffers."""
    dev = x.device
    n, k = weight.shape[::-1] if transposed else weight.shape
    xt, wt, yt = _DTYPES[x.dtype], _DTYPES[weight.dtype], _DTYPES[out_dtype]
    m = x.numel() // k
    sizes = _layer_sizes(m, n, k, transposed, (yt, xt, wt), need_x, need_w) if m else (0, 0, 0)

    def work(s):
        y = torch.empty((*x.shape[:-1], n), dtype=out_dtype, device=dev)
        kept = torch.empty(sizes[0], dtype=torch.uint8, device=dev)
        if m:
            flat, ldx = _rows(_flat(x) if x.dim() > 1 else x.reshape(1, -1))
            w, ldw = _rows(weight)
            ws = torch.empty(sizes[1], dtype=torch.uint8, device=dev)
            lm._check(lm.lib().malt_block_layer_forward(
                flat.data_ptr(), xt, m, k, ldx, w.data_ptr(), wt, n, ldw, transposed, y.data_ptr(), yt, n, need_x, need_w,
                kept.data_ptr(), sizes[0], ws.data_ptr(), sizes[1], s))
        return y, kept

    return (*_on(dev, stream, (x, weight), work), (m, n, k, sizes))


class _Fp8Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, transposed, out_dtype):
        need_x, need_w = ctx.needs_input_grad[:2]
        y, kept, sizes = _layer_forward(x, weight, transposed, out_dtype, need_x, need_w, None)
        ctx.save_for_backward(kept)
        ctx.args = (x.shape, x.dtype, weight.shape, weight.dtype, transposed, *sizes)
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        (kept,) = ctx.saved_tensors
        x_shape, x_dtype, w_shape, w_dtype, transposed, m, n, k, sizes = ctx.args
        need_x, need_w = ctx.needs_input_grad[:2]
        dev = dy.device
        if dy.dtype not in _DTYPES:
            dy = dy.float()
        if m == 0:
            return (torch.zeros(x_shape, dtype=x_dtype, device=dev) if need_x else None,
                    torch.zeros(w_shape, dtype=w_dtype, device=dev) if need_w else None, None, None)

        def work(s):
            g, ld = _rows(dy if dy.dim() == 2 else dy.reshape(-1, n))
            dx = torch.empty(x_shape, dtype=x_dtype, device=dev) if need_x else None
            dw = torch.empty(w_shape, dtype=w_dtype, device=dev) if need_w else None
            ws = torch.empty(sizes[2], dtype=torch.uint8, device=dev)
            lm._check(lm.lib().malt_block_layer_backward(
                g.data_ptr(), _DTYPES[g.dtype], m, n, ld, k, transposed, kept.data_ptr(), sizes[0],
                dx.data_ptr() if need_x else None, _DTYPES[x_dtype], k, dw.data_ptr() if need_w else None,
                _DTYPES[w_dtype], w_shape[1], 0, ws.data_ptr(), sizes[2], s))
            return dx, dw, None, None

        return _on(dev, None, (), work)


def _kept(x, values: int, scales: int, n: int, out, s) -> None:
    """out = x W^T on a weight's values and block scales."""
    flat, ld = _rows(_flat(x) if x.dim() > 1 else x.reshape(1, -1))
    m, k = flat.shape
    out_type = _DTYPES[out.dtype]
    size = _linear_size(m, n, k, out_type)
    ws = torch.empty(size, dtype=torch.uint8, device=out.device) if size else None
    lm._check(lm.lib().malt_block_linear(flat.data_ptr(), _DTYPES[flat.dtype], m, k, ld, values, scales, n,
                                         out.data_ptr(), out_type, n, ws.data_ptr() if size else None, size, s))


def _linear(x, weight, out_dtype, stream):
    """The layer without gradients."""
    dev = x.device
    n = weight.shape[0]

    def work(s):
        y = torch.empty((*x.shape[:-1], n), dtype=out_dtype, device=dev)
        if x.numel():
            values, scales = _quantize_weight(weight, s)
            _kept(x, values.data_ptr(), scales.data_ptr(), n, y, s)
        return y

    return _on(dev, stream, (x, weight), work)


def _linear_args(x, k: int, out_dtype):
    if x.dim() < 1 or x.shape[-1] != k:
        raise ValueError(f"x must be (..., {k}) (got {tuple(x.shape)})")
    out_dtype = x.dtype if out_dtype is None else out_dtype
    _type("out_dtype", out_dtype)
    return out_dtype


def _weight(weight, device=None) -> None:
    _tensor("weight", weight, _DTYPES, device)
    if weight.dim() != 2 or weight.numel() < 1:
        raise ValueError(f"weight must be (outer, inner) (got {tuple(weight.shape)})")


def fp8_linear(x: torch.Tensor, weight: torch.Tensor, out_dtype: Optional[torch.dtype] = None,
               transposed: bool = False, stream=None) -> torch.Tensor:
    """x weight^T with both brought to 8 bits: x with a scale for each row and
    128 values, weight (outer, inner) with one for each 128 x 128 block.
    out_dtype: x's unless given.  transposed: weight is (inner, outer), as GPT-2's
    layers store it, and the result x weight.

    float32 results are float32 sums.  bfloat16 results are summed with fewer bits:
    products of 8 neighbouring values with 14 bits below the largest, these sums in
    float32, off by up to 2^-11 sum |x||w| before they are rounded (1e-5 to 6e-5 of
    their norm on random values; more than bfloat16's rounding where large products
    cancel).  For bfloat16 results of float32 sums take out_dtype=torch.float32 and
    round.  The gradients are as precise as their types, x's and weight's.

    The backward pass runs in 8 bits too: the output's gradient by rows times
    the same 8-bit weight, and the transposes of gradient and x, with a scale for
    each column and 128 tokens, for the weight's gradient (of weight's type).
    Rounding to 8 bits passes gradients through unchanged."""
    _tensor("x", x, _DTYPES)
    _weight(weight, x.device)
    _no_tangent("x", x)
    _no_tangent("weight", weight)
    transposed = bool(transposed)
    out_dtype = _linear_args(x, weight.shape[0 if transposed else 1], out_dtype)
    if torch.is_grad_enabled() and (x.requires_grad or weight.requires_grad):
        _no_stream(stream)
        return _Fp8Linear.apply(x, weight, transposed, out_dtype)
    if transposed:
        return _layer_forward(x, weight, True, out_dtype, False, False, stream)[0]
    return _linear(x, weight, out_dtype, stream)


def fp8_quantize_weight(weight: torch.Tensor, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """A weight (outer, inner) in 8 bits, to be kept for fp8_forward: values
    float8_e4m3fn (outer, inner padded with zeros to whole blocks), and the
    exponent (plus 127) of each 128 x 128 block's power-of-two scale, uint8
    (outer blocks, inner blocks).  value * 2^(scale - 127) is what it stands for."""
    _weight(weight)
    weight = weight.detach()
    values, scales = _on(weight.device, stream, (weight,), lambda s: _quantize_weight(weight, s))
    return values.view(torch.float8_e4m3fn), scales


class Fp8Rows(NamedTuple):
    """Activations (shape[:-1] + (inner,)) in 8 bits, as rms_norm_fp8 makes them for fp8_forward."""
    values: torch.Tensor   # float8_e4m3fn (rows, inner padded with zeros to whole blocks)
    scales: torch.Tensor   # uint8 (blocks, rows padded to 256), in the matrix instructions' order
    shape: torch.Size


def _fp8_rows(x: Fp8Rows, dev, k: int, kb: int) -> int:
    """Checks activations in 8 bits; their number of rows."""
    _tensor("x.values", x.values, (torch.float8_e4m3fn,), dev)
    _tensor("x.scales", x.scales, (torch.uint8,), dev)
    m = torch.Size(x.shape[:-1]).numel()
    if tuple(x.values.shape) != (m, kb * BLOCK) or not x.values.is_contiguous():
        raise ValueError(f"x.values must be contiguous, ({m}, {kb * BLOCK}) (got {tuple(x.values.shape)}, "
                         f"strides {x.values.stride()})")
    if tuple(x.scales.shape) != (kb, _pad(m, 256)) or not x.scales.is_contiguous():
        raise ValueError(f"x.scales must be contiguous, ({kb}, {_pad(m, 256)}) (got {tuple(x.scales.shape)}, "
                         f"strides {x.scales.stride()})")
    return m


def fp8_forward(x: Union[torch.Tensor, Fp8Rows], values: torch.Tensor, scales: torch.Tensor,
                out_dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
    """fp8_linear on kept weights (fp8_quantize_weight), without gradients:
    x (..., inner), values (outer, inner padded to whole blocks).  x may be in 8 bits
    already (rms_norm_fp8's rows; out_dtype is bfloat16 then unless given).  Precision by
    out_dtype, as there."""
    ready = isinstance(x, Fp8Rows)
    if (ready and all(isinstance(t, torch.Tensor) and t.is_cuda for t in (x.values, x.scales, values, scales))
            and (out_dtype is None or out_dtype in _DTYPES)):
        out_type = _DTYPES[out_dtype or torch.bfloat16]
        y = _on(values.device, stream, (x.values, x.scales, values, scales),
                lambda s: _host().fp8_rows(x.values, x.scales, x.shape, values, scales, out_type, s))
        if y is not None:
            return y   # otherwise the checks below say what is wrong
    _tensor("values", values, (torch.float8_e4m3fn,))
    dev = values.device
    if not ready:
        _tensor("x", x, _DTYPES, dev)
    _tensor("scales", scales, (torch.uint8,), dev)
    k = x.shape[-1] if len(x.shape) else 0
    if k < 1:
        raise ValueError(f"x must be (..., inner) (got {tuple(x.shape)})")
    kb = -(-k // BLOCK)
    if ready:
        m = _fp8_rows(x, dev, k, kb)
        out_dtype = torch.bfloat16 if out_dtype is None else out_dtype
        _type("out_dtype", out_dtype)
    else:
        out_dtype = _linear_args(x, k, out_dtype)
    if values.dim() != 2 or values.shape[0] < 1 or values.shape[1] != kb * BLOCK or not values.is_contiguous():
        raise ValueError(f"values must be contiguous, (outer, {kb * BLOCK}) (got {tuple(values.shape)}, "
                         f"strides {values.stride()})")
    n = values.shape[0]
    if tuple(scales.shape) != (-(-n // BLOCK), kb) or not scales.is_contiguous():
        raise ValueError(f"scales must be contiguous, ({-(-n // BLOCK)}, {kb}) "
                         f"(got {tuple(scales.shape)}, strides {scales.stride()})")
    if ready:
        raise ValueError(f"x, values and scales do not belong together (x of {tuple(x.shape)}, values {tuple(values.shape)})")
    x = x.detach()

    def work(s):
        y = torch.empty((*x.shape[:-1], n), dtype=out_dtype, device=dev)
        if x.numel():
            _kept(x, values.data_ptr(), scales.data_ptr(), n, y, s)
        return y

    return _on(dev, stream, (x, values, scales), work)


# ------------------------------------------------------- cross entropy of a head
def _head(x, weight, labels, grad, want_losses, want_dx, want_dw, out, accumulate, stats, want_stats, stream):
    """losses, dx, dweight and the rows' statistics, as far as they are wanted.  stats: those of an earlier call."""
    _tensor("x", x, _DTYPES)
    dev = x.device
    _weight(weight, dev)
    v, k = weight.shape
    if x.dim() < 1 or x.shape[-1] != k:
        raise ValueError(f"x must be (..., {k}) (got {tuple(x.shape)})")
    lead = x.shape[:-1]
    n = lead.numel()
    _tensor("labels", labels, _INDEX, dev)
    if labels.shape != lead:
        raise ValueError(f"labels must be {tuple(lead)} (got {tuple(labels.shape)})")
    weights, value = None, 1.0
    if isinstance(grad, torch.Tensor):
        _tensor("grad", grad, (torch.float32,), dev)
        if grad.dim() > 0 and grad.shape != lead:
            raise ValueError(f"grad must be a number, a scalar tensor or {tuple(lead)} (got {tuple(grad.shape)})")
        weights = grad
    else:
        value = float(grad)
    if out is not None:
        _tensor("out", out, _DTYPES, dev)
        if tuple(out.shape) != (v, k) or (k > 1 and out.stride(1) != 1) or (v > 1 and out.stride(0) < k):
            raise ValueError(f"out must be ({v}, {k}) with contiguous rows (got {tuple(out.shape)}, strides {out.stride()})")
    elif accumulate:
        raise ValueError("accumulate needs out")

    def work(s):
        losses = torch.empty(lead, dtype=torch.float32, device=dev) if want_losses else None
        dx = torch.empty(x.shape, dtype=x.dtype, device=dev) if want_dx else None
        dw = out if out is not None else torch.empty((v, k), dtype=weight.dtype, device=dev) if want_dw else None
        kept = torch.empty((n, 4), dtype=torch.float32, device=dev) if want_stats else stats
        flat, ldx = _rows(_flat(x) if x.dim() > 1 else x.reshape(1, k))
        w, ldw = _rows(weight)
        y = labels if labels.dim() == 1 else labels.reshape(-1)
        g = weights if weights is None or weights.dim() < 2 else weights.reshape(-1)
        a = lm.malt_linear_loss_t(
            flat.data_ptr(), _DTYPES[x.dtype], n, k, ldx, w.data_ptr(), _DTYPES[weight.dtype], v, ldw, y.data_ptr(),
            _INDEX[y.dtype], y.stride(0) if n > 1 else 0, None if g is None else g.data_ptr(),
            g.stride(0) if g is not None and n > 1 and g.dim() else 0, value, losses.data_ptr() if want_losses else None,
            None if kept is None else kept.data_ptr(), int(stats is not None), dx.data_ptr() if want_dx else None, k,
            None if dw is None else dw.data_ptr(), 0 if dw is None else _DTYPES[dw.dtype],
            k if dw is None or v == 1 else dw.stride(0), int(bool(accumulate)))
        if n or dw is not None:
            size = c_size_t(0)
            lm._check(lm.lib().malt_linear_loss_size(byref(a), byref(size)))
            ws = torch.empty(size.value, dtype=torch.uint8, device=dev)
            lm._check(lm.lib().malt_linear_loss(byref(a), ws.data_ptr(), size.value, s))
        return losses, dx, dw, kept

    result = _on(dev, stream, (x, weight, labels, weights, out, stats), work)
    _written(out)
    return result


class _LinearCrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, labels):
        losses, _, _, stats = _head(x, weight, labels, 1.0, True, False, False, None, False, None, True, None)
        ctx.save_for_backward(x, weight, labels, stats)
        return losses

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        _host().check_captured_backward()
        x, weight, labels, stats = ctx.saved_tensors
        need_x, need_w = ctx.needs_input_grad[:2]
        _, dx, dw, _ = _head(x, weight, labels, grad.float(), False, need_x, need_w, None, False, stats, False, None)
        return dx, dw, None


def linear_cross_entropy(x: torch.Tensor, weight: torch.Tensor, labels: torch.Tensor, stream=None) -> torch.Tensor:
    """Cross entropy of each row of a linear head, logits = x weight^T with
    x (..., inner) and weight (vocab, inner), float32 of labels' shape.  The logits
    are never held: neither here nor in the backward pass.  A label outside the vocabulary
    (-1, -100) is none: the row's loss is 0, whatever x holds there, and it adds no gradient.
    Types may differ (float32, bfloat16); of float32 values the logits take 22 bits (24 for the losses of
    up to 32 rows), the gradients all.  Differentiable in x and weight; gradients are of their types."""
    for name, t in (("x", x), ("weight", weight)):
        if isinstance(t, torch.Tensor):
            _no_tangent(name, t)
    if torch.is_grad_enabled() and (getattr(x, "requires_grad", False) or getattr(weight, "requires_grad", False)):
        _no_stream(stream)
        return _LinearCrossEntropy.apply(x, weight, labels)
    return _head(x, weight, labels, 1.0, True, False, False, None, False, None, False, stream)[0]


def linear_cross_entropy_step(x: torch.Tensor, weight: torch.Tensor, labels: torch.Tensor,
                              grad: Union[float, torch.Tensor] = 1.0, out: Optional[torch.Tensor] = None,
                              accumulate: bool = False, stream=None
                              ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """The losses of linear_cross_entropy and the gradients of sum(grad * losses)
    to x and weight, as (losses, dx, dweight).  grad: a number, a float32 scalar tensor or
    one weight for each row (0: no gradient).  dweight is of weight's type, or goes to `out`
    (vocab, inner; contiguous rows; either type) when given, with accumulate added to it: to autograd,
    `out` is changed in place."""
    x, weight = (t.detach() if isinstance(t, torch.Tensor) and t.requires_grad else t for t in (x, weight))
    return _head(x, weight, labels, grad, True, True, True, out, accumulate, None, False, stream)[:3]


# -------------------------------------------------------------------------- norm
_binding = None


def _host():
    """The module _malt (csrc/binding.cpp): the host side of what follows, in C++."""
    global _binding
    if _binding is None:
        lm.lib()
        _binding = lm.load_binding()
    return _binding


def _grads_wanted(*tensors) -> bool:
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


def rms_norm(x: torch.Tensor, weight: torch.Tensor, residual: Optional[torch.Tensor] = None, eps: float = 1e-6,
             out_dtype: Optional[torch.dtype] = None, stream=None):
    """Root-mean-square norm of the rows of x (..., width) times weight (width,):
    y = h / sqrt(mean(h^2) + eps) * weight, h = x.  With residual (of x's shape and type)
    h = x + residual, rounded to their type, and the result is (y, h).  out_dtype: x's unless
    given.  Computed in float32, the mean of squares in float64.  Differentiable in x, residual
    and weight, through h as well."""
    _tensor("x", x, _DTYPES)
    _tensor("weight", weight, _DTYPES, x.device)
    if residual is not None:
        _tensor("residual", residual, (x.dtype,), x.device)
        _no_tangent("residual", residual)
    _no_tangent("x", x)
    _no_tangent("weight", weight)
    if out_dtype is not None:
        _type("out_dtype", out_dtype)
    grad = _grads_wanted(x, weight, residual)
    if grad:
        _no_stream(stream)
    return _on(x.device, stream, (x, weight, residual),
               lambda s: _host().rms_norm(x, weight, residual, eps, out_dtype, grad, s))


def rms_norm_fp8(x: torch.Tensor, weight: torch.Tensor, residual: Optional[torch.Tensor] = None, eps: float = 1e-6,
                 stream=None):
    """rms_norm with its output in 8 bits (Fp8Rows: a scale for each row and 128
    values), for fp8_forward on kept weights, in one pass and without gradients:
    rows, or (rows, h) with residual.  y is rounded once, from float32."""
    _tensor("x", x, _DTYPES)
    if stream is not None:   # what is recorded on it
        _tensor("weight", weight, _DTYPES, x.device)
        if residual is not None:
            _tensor("residual", residual, (x.dtype,), x.device)
    values, scales, h = _on(x.device, stream, (x, weight, residual),
                            lambda s: _host().rms_norm_fp8(x, weight, residual, eps, s))
    rows = Fp8Rows(values, scales, x.shape)
    return rows if residual is None else (rows, h)


# ------------------------------------------------------------------------- AdamW
_STATES = (torch.float32, torch.uint8)


def _tensors(name: str, tensors, types, dev) -> list:
    for i, t in enumerate(tensors):
        _tensor(f"{name}[{i}]", t, types, dev)
    return tensors


@functools.lru_cache(maxsize=4096)
def _adamw_size(numel: int, bits: int) -> int:
    size = c_size_t(0)
    lm._check(lm.lib().malt_adamw_state_size(numel, bits, byref(size)))
    return size.value


def adamw_state(param: torch.Tensor, bits: int = 32) -> torch.Tensor:
    """The moments of a parameter before its first step, to be kept for adamw_step: float32
    (2, numel), or with bits=8 the bytes of 8-bit moments (8.125 bits each)."""
    _tensor("param", param, _DTYPES)
    if bits not in (8, 32):
        raise ValueError(f"bits must be 8 or 32 (got {bits})")
    if bits == 32:
        return torch.zeros((2, param.numel()), dtype=torch.float32, device=param.device)
    return torch.zeros(_adamw_size(param.numel(), 8), dtype=torch.uint8, device=param.device)


def adamw_step(params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], states: Sequence[torch.Tensor], lr: float,
               betas: Tuple[float, float] = (0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01, *, step: int,
               grad_scale: Union[float, torch.Tensor] = 1.0, seed: int = 0, stream=None) -> None:
    """One AdamW step over many tensors, in place, a launch for each 108 of them:
    m = b1 m + (1 - b1) g, v = b2 v + (1 - b2) g^2 with g = grad_scale * grad, then
    p = p (1 - lr weight_decay) - lr (m / (1 - b1^step)) / (sqrt(v / (1 - b2^step)) + eps).
    params (contiguous) and grads are float32 or bfloat16, states adamw_state's.  eps is at least
    2^-126; step counts from 1; grad_scale: a number or a float32 scalar tensor, read on the device.

    8-bit moments are rounded up or down at random by their distance, so that small changes
    add up; the random numbers follow from `seed`, the tensor's place in the list and the
    element's: give each step another seed.  Equal calls give equal bits.  A captured call replays its
    arguments, step and seed among them.  To autograd, params and states are changed in place."""
    params, grads, states = list(params), list(grads), list(states)
    if not 0 <= int(seed) < 1 << 64:
        raise ValueError(f"seed must be in [0, 2^64) (got {seed})")
    if not params and not grads and not states:
        return
    scale_at = None
    if isinstance(grad_scale, torch.Tensor):
        scale_at, grad_scale = grad_scale, 1.0
    if params:
        _tensor("params[0]", params[0], _DTYPES)
        dev = params[0].device
    else:   # refused below
        dev = torch.device("cuda", torch.cuda.current_device())
    inputs = ()
    if stream is not None:   # what is recorded on it
        inputs = (*_tensors("params", params, _DTYPES, dev), *_tensors("grads", grads, _DTYPES, dev),
                  *_tensors("states", states, _STATES, dev), scale_at)
        if scale_at is not None:
            _tensor("grad_scale", scale_at, (torch.float32,), dev)
    b1, b2 = betas
    _on(dev, stream, inputs, lambda s: _host().adamw_step(params, grads, states, lr, b1, b2, eps, weight_decay, step,
                                                          grad_scale, scale_at, seed, s))


def adamw_moments(params: Sequence[torch.Tensor], states: Sequence[torch.Tensor], stream=None) -> List[torch.Tensor]:
    """What the moments of adamw_step stand for: float32 (2, numel) for each parameter,
    the first moment and the second, in new tensors."""
    params, states = list(params), list(states)
    if not params and not states:
        return []
    if params:
        _tensor("params[0]", params[0], _DTYPES)
        dev = params[0].device
    else:   # refused below
        dev = torch.device("cuda", torch.cuda.current_device())
    inputs = _tensors("states", states, _STATES, dev) if stream is not None else ()
    return _on(dev, stream, inputs, lambda s: _host().adamw_moments(params, states, s))
