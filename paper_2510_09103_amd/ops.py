"""The operators of a model's end on tensors: dropout, root-mean-square norm with the residual's addition, and softmax cross entropy
over the vocabulary, each with its gradient.  All arithmetic happens in libadapm.so; these functions check the tensors, allocate
outputs and scratch from PyTorch on the current stream of the tensors' device, and make one library call (head_loss: the call of
the forward pass).

There is no autograd here: tensors that require gradients (parameters) are taken as data, and what a function returns or writes has no graph.
A training step calls the forward and the backward functions itself, as it calls AdaPM.step, and hands the gradients on in the buffers it
likes (`out` / `dx` / `dweight` arguments).
"""
from __future__ import annotations

from typing import NamedTuple, Optional, Tuple

import torch

from . import binding as B

try:        # the address alone: torch.cuda.current_stream makes an object for 2 us, as much as a small launch
    from torch._C import _cuda_getCurrentRawStream as _raw_stream
except ImportError:
    def _raw_stream(device):
        return torch.cuda.current_stream(device).cuda_stream

_DT = {torch.float32: B.ADAPM_F32, torch.bfloat16: B.ADAPM_BF16, torch.float8_e4m3fn: B.ADAPM_E4M3}
_REDUCTION = {"sum": B.ADAPM_REDUCE_SUM, "mean": B.ADAPM_REDUCE_MEAN}


class Rng(NamedTuple):
    """Counter of the generator that dropout draws from.  The same (seed, offset) gives the same mask: the backward pass takes the Rng
    of the forward pass, and every use of dropout in a step takes another offset.  offset_dev, an int64 tensor of one element, is added
    to offset on the device: in a captured graph that is how replays draw new masks."""
    seed: int
    offset: int = 0
    offset_dev: Optional[torch.Tensor] = None


class Norm(NamedTuple):
    y: torch.Tensor
    h: torch.Tensor                      # residual + dropout(x): the new residual stream (x itself with neither)
    rstd: torch.Tensor                   # fp32, one a row
    scale: Optional[torch.Tensor]        # 8-bit output: fp32, one a row


class Loss(NamedTuple):
    loss: torch.Tensor                   # fp32, no dimensions
    row_loss: torch.Tensor               # fp32, one a row, not weighted; 0 where the row does not count
    lse: torch.Tensor                    # fp32, one a row


def _first(name, t):
    """The tensor that gives a call its device, type and shape: (its matrix, rows, columns)."""
    if not isinstance(t, torch.Tensor) or t.dim() < 1:
        raise ValueError(f"{name}: a tensor with at least one dimension is wanted")
    if t.device.type != "cuda":
        raise ValueError(f"{name}: on {t.device}, a GPU tensor is wanted")
    cols = t.shape[-1]
    if cols == 0:
        raise ValueError(f"{name}: rows of no elements")
    return B.adapm_rows_t(t.data_ptr(), cols if t.is_contiguous() else _stride(name, t)), t.numel() // cols, cols


def _rows(name, t, like, dtype, shape):
    if t.get_device() != like.get_device():
        raise ValueError(f"{name}: on {t.device}, the other tensors are on {like.device}")
    if t.dtype != dtype:
        raise TypeError(f"{name}: {t.dtype}, {dtype} is wanted")
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, {tuple(shape)} is wanted")
    return B.adapm_rows_t(t.data_ptr(), t.shape[-1] if t.is_contiguous() else _stride(name, t))


def _new(t):
    """An output of the call's own making, whose elements are adjacent."""
    return B.adapm_rows_t(t.data_ptr(), t.shape[-1])


def _empty(like, dtype=None):
    """A tensor of like's shape whose elements are adjacent."""
    if like.is_contiguous():
        return torch.empty_like(like, dtype=dtype)
    return like.new_empty(like.shape, dtype=dtype)


def _stride(name, t):
    """Elements from one row to the next of a matrix with any number of leading dimensions, whose rows have to be evenly spaced."""
    cols = t.shape[-1]
    if cols > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: the elements of a row have to be adjacent (stride {t.stride(-1)})")
    stride = None
    for n, s in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if n == 1 or t.numel() == 0:
            continue
        if stride is None:
            stride, width = s, n * s
        elif s != width:
            raise ValueError(f"{name}: rows are not evenly spaced (shape {tuple(t.shape)}, strides {tuple(t.stride())})")
        else:
            width = n * s
    if stride is None:
        stride = cols
    if stride < cols:
        raise ValueError(f"{name}: rows overlap (stride {stride}, {cols} elements)")
    return stride


def _vector(name, t, n, like, dtype):
    if t.get_device() != like.get_device():
        raise ValueError(f"{name}: on {t.device}, the other tensors are on {like.device}")
    if t.dtype != dtype:
        raise TypeError(f"{name}: {t.dtype}, {dtype} is wanted")
    if t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name}: {tuple(t.shape)} with strides {tuple(t.stride())}, {n} adjacent elements are wanted")
    return t.data_ptr()


def _float_type(name, t):
    if t.dtype is torch.bfloat16:
        return B.ADAPM_BF16
    if t.dtype is torch.float32:
        return B.ADAPM_F32
    raise TypeError(f"{name}: {t.dtype}, float32 or bfloat16 is wanted")


def _dropout(p, rng, like):
    if not 0.0 <= p < 1.0:
        raise ValueError(f"p = {p}: a probability in [0, 1) is wanted")
    if p == 0.0:
        return None
    if rng is None:
        raise ValueError("dropout needs rng")
    at = 0
    if rng.offset_dev is not None:
        at = _vector("rng.offset_dev", rng.offset_dev, 1, like, torch.int64)
    mask = (1 << 64) - 1
    return B.adapm_dropout_t(rng.seed & mask, rng.offset & mask, at or None, p, 0)


def _call(f, t, *args):
    """One library call on t's device and the current stream of that device."""
    at = t.get_device()
    if at == torch.cuda.current_device():
        f(*args, _raw_stream(at))
    else:
        with torch.cuda.device(at):
            f(*args, _raw_stream(at))


_NO_ROWS = B.rows()


def _scratch(nbytes, like):
    # from the current stream's pool: PyTorch hands it to no other stream before the work queued here is done
    return like.new_empty(max(nbytes, 1), dtype=torch.uint8)


def dropout(x: torch.Tensor, p: float, rng: Rng, residual: Optional[torch.Tensor] = None,
            out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """residual + dropout(x), rounded once.  The gradient of x is dropout(gradient of the result, p, rng), which the
    caller calls: the result has no autograd graph.  out may be x or residual."""
    dt = _float_type("x", x)
    xr, n, cols = _first("x", x)
    res = _NO_ROWS if residual is None else _rows("residual", residual, x, x.dtype, x.shape)
    drop = _dropout(p, rng, x) or B.adapm_dropout_t(0, 0, None, 0.0, 0)
    if out is None:
        out = _empty(x)
        y = _new(out)
    else:
        y = _rows("out", out, x, x.dtype, x.shape)
    _call(B.adapm_dropout, x, y, xr, res, n, cols, dt, drop)
    return out


def rms_norm(x: torch.Tensor, weight: torch.Tensor, eps: float = 1e-5, residual: Optional[torch.Tensor] = None, p: float = 0.0,
             rng: Optional[Rng] = None, out_dtype: Optional[torch.dtype] = None) -> Norm:
    """h = residual + dropout(x), y = h / sqrt(mean(h^2) + eps) * weight over the last dimension.  out_dtype: that of x, or
    torch.float8_e4m3fn with a scale for each row (y stands for y * scale).  The results have no autograd graph: the gradients are
    rms_norm_backward's."""
    dt, wt = _float_type("x", x), _float_type("weight", weight)
    xr, n, cols = _first("x", x)
    w = _vector("weight", weight, cols, x, weight.dtype)
    out_dtype = x.dtype if out_dtype is None else out_dtype
    if out_dtype not in (x.dtype, torch.float8_e4m3fn):
        raise TypeError(f"out_dtype {out_dtype}: {x.dtype} or torch.float8_e4m3fn is wanted")
    drop = _dropout(p, rng, x)
    res = _NO_ROWS if residual is None else _rows("residual", residual, x, x.dtype, x.shape)
    y = _empty(x, out_dtype)
    rstd = x.new_empty(x.shape[:-1], dtype=torch.float32)
    scale = torch.empty_like(rstd) if out_dtype == torch.float8_e4m3fn else None
    h, hr = x, _NO_ROWS
    if residual is not None or drop is not None:
        h = _empty(x)
        hr = _new(h)
    _call(B.adapm_norm_forward, x, B.adapm_norm_t(n, cols, dt, wt, _DT[out_dtype], wt, eps, 0), xr, res, hr, w, _new(y),
          0 if scale is None else scale.data_ptr(), rstd.data_ptr(), drop)
    return Norm(y, h, rstd, scale)


def rms_norm_backward(dy: torch.Tensor, h: torch.Tensor, weight: torch.Tensor, rstd: torch.Tensor, dh: Optional[torch.Tensor] = None,
                      p: float = 0.0, rng: Optional[Rng] = None, dweight: Optional[torch.Tensor] = None,
                      grad_dtype: Optional[torch.dtype] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(dx, dresidual, dweight) from the gradient of y and, where the residual stream goes on, that of h (dh).  h and rstd are rms_norm's.
    Without dropout dx and dresidual are one tensor.  dweight is written where it is given (any shape of cols elements, such as a norm
    vector's gradient in a block table); else it is new, in grad_dtype or the type of weight."""
    dt, wt = _float_type("dy", dy), _float_type("weight", weight)
    dyr, n, cols = _first("dy", dy)
    w = _vector("weight", weight, cols, dy, weight.dtype)
    r = _vector("rstd", rstd, n, dy, torch.float32)
    drop = _dropout(p, rng, dy)
    up = _NO_ROWS if dh is None else _rows("dh", dh, dy, dy.dtype, dy.shape)
    hr = _rows("h", h, dy, dy.dtype, dy.shape)
    if dweight is None:
        dweight = _empty(weight, grad_dtype)
    elif grad_dtype is not None and dweight.dtype != grad_dtype:
        raise TypeError(f"dweight: {dweight.dtype}, grad_dtype is {grad_dtype}")
    g = _vector("dweight", dweight, cols, dy, dweight.dtype)
    desc = B.adapm_norm_t(n, cols, dt, wt, dt, _float_type("dweight", dweight), 0.0, 0)
    dx = _empty(dy)
    dres = dx if drop is None else torch.empty_like(dx)
    ws = _scratch(B.adapm_norm_workspace_bytes(desc), dy)
    _call(B.adapm_norm_backward, dy, desc, dyr, up, hr, w, r, _new(dx), _NO_ROWS if drop is None else _new(dres), g, drop, ws.data_ptr())
    return dx, dres, dweight


def _head(x, weight, targets, row_weight, reduction, scale):
    dt = _float_type("x", x)
    xr, n, cols = _first("x", x)
    if weight.dim() != 2 or weight.shape[1] != cols:
        raise ValueError(f"weight: shape {tuple(weight.shape)}, (vocabulary, {cols}) is wanted")
    if weight.shape[0] == 0:
        raise ValueError("weight: a vocabulary of no entries")
    if reduction not in _REDUCTION:
        raise ValueError(f"reduction {reduction!r}: 'mean' or 'sum' is wanted")
    w = _rows("weight", weight, x, x.dtype, weight.shape)
    t = _vector("targets", targets, n, x, torch.int64)
    rw = 0 if row_weight is None else _vector("row_weight", row_weight, n, x, torch.float32)
    return B.adapm_head_t(n, weight.shape[0], cols, dt, _REDUCTION[reduction], scale, 0), xr, w, t, rw


def head_loss(x: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, row_weight: Optional[torch.Tensor] = None,
              reduction: str = "mean", scale: float = 1.0) -> Loss:
    """Softmax cross entropy of x @ weight.T against targets (int64, one a row); rows whose target is outside the vocabulary (-100, say)
    do not count.  loss = scale * sum(row_weight * row_loss), divided by the number of rows that count where reduction is "mean".  The
    results have no autograd graph: the gradients are head_backward's."""
    h, xr, w, t, rw = _head(x, weight, targets, row_weight, reduction, scale)
    loss = x.new_empty((), dtype=torch.float32)
    row_loss = _empty(targets, torch.float32)
    lse = torch.empty_like(row_loss)
    size = B.adapm_head_workspace_bytes(h, w, False)
    ws = _scratch(size, x)
    _call(B.adapm_head_loss, x, h, xr, w, t, rw, loss.data_ptr(), row_loss.data_ptr(), lse.data_ptr(), ws.data_ptr(), size)
    return Loss(loss, row_loss, lse)


def head_backward(x: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor,
                  row_weight: Optional[torch.Tensor] = None, reduction: str = "mean", scale: float = 1.0,
                  upstream: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None, dweight: Optional[torch.Tensor] = None,
                  need_dx: bool = True, need_dweight: bool = True) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
    """(dx, dweight), the gradients of upstream * loss (upstream: one fp32 element on the device, 1 if absent) for the arguments and the lse
    of head_loss.  They are written where dx and dweight are given (the gradient buffer of a table's output head, say)."""
    h, xr, w, t, rw = _head(x, weight, targets, row_weight, reduction, scale)
    at = _vector("lse", lse, targets.numel(), x, torch.float32)
    up = 0 if upstream is None else _vector("upstream", upstream, 1, x, torch.float32)
    if not need_dx and not need_dweight:
        raise ValueError("need_dx and need_dweight are both false")
    if need_dx and dx is None:
        dx = _empty(x)
    if need_dweight and dweight is None:
        dweight = _empty(weight)
    gx = _rows("dx", dx, x, x.dtype, x.shape) if need_dx else _NO_ROWS
    gw = _rows("dweight", dweight, x, x.dtype, weight.shape) if need_dweight else _NO_ROWS
    size = B.adapm_head_workspace_bytes(h, w, True)
    ws = _scratch(size, x)
    _call(B.adapm_head_backward, x, h, xr, w, t, rw, at, up, gx, gw, ws.data_ptr(), size)
    return dx if need_dx else None, dweight if need_dweight else None
