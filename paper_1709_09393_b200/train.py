"""Binding of a worker's local step: layer norm, matrix product with its epilogue, distillation loss.

Argument marshalling only, as in binding.py.  Matrices are 2-D CUDA tensors of float32, bfloat16 or float16
(one type per call) whose columns are adjacent; rows may be padded.  gamma, beta, bias and all parameter
gradients are float32, so that they can be slices of the flat model and of the flat update.  Outputs and
workspaces are the caller's.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as B

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}

_lib, _check, _stream = B.lib, B._check, B._stream


def _type(t: torch.Tensor, name: str) -> int:
    code = _TYPES.get(t.dtype)
    if code is None or not t.is_cuda or t.dim() != 2:
        raise TypeError(f"{name}: expected a 2-D CUDA tensor of float32, bfloat16 or float16")
    return code


def _matrix(t: Optional[torch.Tensor], rows: int, cols: int, dtype: torch.dtype, name: str):
    """(address, row stride) of a matrix; (NULL, cols) for a missing one."""
    if t is None:
        return None, cols
    if t.dtype != dtype or not t.is_cuda or t.dim() != 2:
        raise TypeError(f"{name}: expected a 2-D CUDA tensor of {dtype}")
    if t.shape[0] != rows or t.shape[1] != cols:
        raise ValueError(f"{name}: expected {rows} x {cols}, got {t.shape[0]} x {t.shape[1]}")
    ld, step = t.stride()
    if cols > 1 and step != 1:
        raise ValueError(f"{name}: columns are not adjacent")
    if rows <= 1:
        ld = cols
    elif ld < cols:
        raise ValueError(f"{name}: rows overlap")
    return t.data_ptr() or None, ld


def _vector(t: Optional[torch.Tensor], n: int, name: str, dtype: torch.dtype = torch.float32) -> Optional[int]:
    if t is None:
        return None
    if t.dtype != dtype or not t.is_cuda or not t.is_contiguous():
        raise TypeError(f"{name}: expected a contiguous CUDA tensor of {dtype}")
    if t.numel() != n:
        raise ValueError(f"{name}: expected {n} elements, got {t.numel()}")
    return t.data_ptr() or None


def _ws(ws: Optional[torch.Tensor]):
    if ws is None:
        return None, 0
    if not ws.is_cuda or not ws.is_contiguous():
        raise TypeError("ws: expected a contiguous CUDA tensor")
    return ws.data_ptr(), ws.numel() * ws.element_size()


def _act(activation: str) -> int:
    if activation not in ACTIVATIONS:
        raise ValueError(f"activation: expected one of {', '.join(ACTIVATIONS)}")
    return ACTIVATIONS[activation]


def layernorm_workspace_bytes(rows: int, dim: int) -> int:
    return _lib.slimdp_layernorm_workspace_bytes(rows, dim)


def linear_workspace_bytes(m: int, n: int, k: int, dtype: torch.dtype) -> int:
    """Scratch that serves the forward product and both gradients of an [m, k] x [n, k] layer."""
    if dtype not in _TYPES:
        raise TypeError("dtype: expected float32, bfloat16 or float16")
    return _lib.slimdp_linear_workspace_bytes(m, n, k, _TYPES[dtype])


def slimdp_layernorm_forward(x: torch.Tensor, gamma: Optional[torch.Tensor], beta: Optional[torch.Tensor], eps: float,
                             y: torch.Tensor, mean: Optional[torch.Tensor] = None,
                             rstd: Optional[torch.Tensor] = None, stream=None):
    code = _type(x, "x")
    rows, dim = x.shape
    px, ldx = _matrix(x, rows, dim, x.dtype, "x")
    py, ldy = _matrix(y, rows, dim, x.dtype, "y")
    _check("slimdp_layernorm_forward",
           _lib.slimdp_layernorm_forward(px, ldx, rows, dim, code, _vector(gamma, dim, "gamma"),
                                         _vector(beta, dim, "beta"), eps, py, ldy, _vector(mean, rows, "mean"),
                                         _vector(rstd, rows, "rstd"), _stream(stream)))


def slimdp_layernorm_backward(dy: torch.Tensor, x: torch.Tensor, gamma: Optional[torch.Tensor], mean: torch.Tensor,
                              rstd: torch.Tensor, dx: torch.Tensor, dgamma: Optional[torch.Tensor],
                              dbeta: Optional[torch.Tensor], ws: Optional[torch.Tensor], accumulate: bool = False,
                              stream=None):
    code = _type(x, "x")
    rows, dim = x.shape
    pdy, lddy = _matrix(dy, rows, dim, x.dtype, "dy")
    px, ldx = _matrix(x, rows, dim, x.dtype, "x")
    pdx, lddx = _matrix(dx, rows, dim, x.dtype, "dx")
    pws, nws = _ws(ws)
    _check("slimdp_layernorm_backward",
           _lib.slimdp_layernorm_backward(pdy, lddy, px, ldx, rows, dim, code, _vector(gamma, dim, "gamma"),
                                          _vector(mean, rows, "mean"), _vector(rstd, rows, "rstd"), pdx, lddx,
                                          _vector(dgamma, dim, "dgamma"), _vector(dbeta, dim, "dbeta"),
                                          bool(accumulate), pws, nws, _stream(stream)))


def slimdp_linear_forward(x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor], y: torch.Tensor,
                          ws: torch.Tensor, activation: str = "none", residual: Optional[torch.Tensor] = None,
                          z: Optional[torch.Tensor] = None, stream=None):
    """y = act(x w^T + bias) + residual; z, if given, receives x w^T + bias."""
    code, act = _type(x, "x"), _act(activation)
    _type(w, "w")
    m, k = x.shape
    n = w.shape[0]
    px, ldx = _matrix(x, m, k, x.dtype, "x")
    pw, ldw = _matrix(w, n, k, x.dtype, "w")
    pr, ldr = _matrix(residual, m, n, x.dtype, "residual")
    py, ldy = _matrix(y, m, n, x.dtype, "y")
    pz, ldz = _matrix(z, m, n, x.dtype, "z")
    pws, nws = _ws(ws)
    _check("slimdp_linear_forward",
           _lib.slimdp_linear_forward(px, ldx, pw, ldw, _vector(bias, n, "bias"), pr, ldr, m, n, k, code, act, py, ldy,
                                      pz, ldz, pws, nws, _stream(stream)))


def slimdp_linear_backward_input(dy: torch.Tensor, w: torch.Tensor, dx: torch.Tensor, ws: torch.Tensor,
                                 activation: str = "none", z: Optional[torch.Tensor] = None,
                                 add: Optional[torch.Tensor] = None, stream=None):
    """dx = (dy w) * act'(z) + add, with z the pre-activation of the layer that made this one's input."""
    code, act = _type(dy, "dy"), _act(activation)
    _type(w, "w")
    m, n = dy.shape
    k = w.shape[1]
    pdy, lddy = _matrix(dy, m, n, dy.dtype, "dy")
    pw, ldw = _matrix(w, n, k, dy.dtype, "w")
    pz, ldz = _matrix(z, m, k, dy.dtype, "z")
    pa, lda = _matrix(add, m, k, dy.dtype, "add")
    pdx, lddx = _matrix(dx, m, k, dy.dtype, "dx")
    pws, nws = _ws(ws)
    _check("slimdp_linear_backward_input",
           _lib.slimdp_linear_backward_input(pdy, lddy, pw, ldw, pz, ldz, pa, lda, m, n, k, code, act, pdx, lddx, pws,
                                             nws, _stream(stream)))


def slimdp_linear_backward_weight(dy: torch.Tensor, x: torch.Tensor, dw: torch.Tensor, db: Optional[torch.Tensor],
                                  ws: torch.Tensor, accumulate: bool = False, stream=None):
    """dw (+)= dy^T x in float32, db (+)= column sums of dy."""
    code = _type(dy, "dy")
    _type(x, "x")
    m, n = dy.shape
    k = x.shape[1]
    pdy, lddy = _matrix(dy, m, n, dy.dtype, "dy")
    px, ldx = _matrix(x, m, k, dy.dtype, "x")
    pdw, lddw = _matrix(dw, n, k, torch.float32, "dw")
    pws, nws = _ws(ws)
    _check("slimdp_linear_backward_weight",
           _lib.slimdp_linear_backward_weight(pdy, lddy, px, ldx, m, n, k, code, pdw, lddw, _vector(db, n, "db"),
                                              bool(accumulate), pws, nws, _stream(stream)))


def train_read_status(stream=None) -> None:
    """Synchronises, and raises if a bounded wait of one of these kernels ever ran out on this device."""
    _check("slimdp_train_read_status", _lib.slimdp_train_read_status(_stream(stream)))


def slimdp_activation_backward(dy: torch.Tensor, z: torch.Tensor, dz: torch.Tensor, activation: str, stream=None):
    """dz = dy * act'(z)."""
    code, act = _type(dy, "dy"), _act(activation)
    m, n = dy.shape
    pdy, lddy = _matrix(dy, m, n, dy.dtype, "dy")
    pz, ldz = _matrix(z, m, n, dy.dtype, "z")
    pdz, lddz = _matrix(dz, m, n, dy.dtype, "dz")
    _check("slimdp_activation_backward",
           _lib.slimdp_activation_backward(pdy, lddy, pz, ldz, m, n, code, act, pdz, lddz, _stream(stream)))


def slimdp_distill(logits: torch.Tensor, teacher_idx: Optional[torch.Tensor], teacher_logit: Optional[torch.Tensor],
                   loss: torch.Tensor, dlogits: Optional[torch.Tensor] = None, label: Optional[torch.Tensor] = None,
                   row_weight: Optional[torch.Tensor] = None, temperature: float = 1.0, kd_weight: float = 1.0,
                   ce_weight: float = 0.0, stream=None):
    """Loss of each row and its gradient; dlogits may be logits (replaced) or None (the loss alone)."""
    code = _type(logits, "logits")
    rows, vocab = logits.shape
    pl, ldl = _matrix(logits, rows, vocab, logits.dtype, "logits")
    pd, ldd = _matrix(dlogits, rows, vocab, logits.dtype, "dlogits")
    if (teacher_idx is None) != (teacher_logit is None):
        raise ValueError("teacher_idx and teacher_logit come together")
    top, pi, pt, tcode = 0, None, None, 0
    if teacher_idx is not None:
        if teacher_idx.dim() != 2:
            raise ValueError("teacher_idx: expected rows x top")
        top = teacher_idx.shape[1]
        tcode = _TYPES.get(teacher_logit.dtype)
        if tcode is None:
            raise TypeError("teacher_logit: expected float32, bfloat16 or float16")
        pi = _vector(teacher_idx, rows * top, "teacher_idx", torch.int32)
        pt = _vector(teacher_logit, rows * top, "teacher_logit", teacher_logit.dtype)
        if teacher_idx.shape != teacher_logit.shape or teacher_idx.shape[0] != rows:
            raise ValueError("teacher_idx, teacher_logit: expected rows x top")
    _check("slimdp_distill",
           _lib.slimdp_distill(pl, ldl, rows, vocab, code, pi, pt, tcode, top,
                               _vector(label, rows, "label", torch.int32), _vector(row_weight, rows, "row_weight"),
                               temperature, kd_weight, ce_weight, _vector(loss, rows, "loss"), pd, ldd,
                               _stream(stream)))
