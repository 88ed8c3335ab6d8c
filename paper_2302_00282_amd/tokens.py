"""The operators of a token model's serving step on torch tensors: 8-bit linear layers.

Each function checks its tensors, allocates what it returns, and makes one or two calls of the C ABI (include/xenos.h) on torch's current
stream of the tensors' device; nothing synchronises.  The kernels are the library's own: there is no CPU path.  Forward passes only: what
they return carries no gradient, and an input that asks for one is refused.
"""
from __future__ import annotations

from contextlib import nullcontext
from typing import Optional, Tuple

import torch

from . import xenos as X

_DTYPE = {torch.float32: X.XENOS_F32, torch.bfloat16: X.XENOS_BF16}


def _need(ok: bool, status: int, message: str):
    if not ok:
        raise X.XenosError(status, message)


def _tensor(t: torch.Tensor, name: str, like: Optional[torch.Tensor] = None, dtype=None, shape=None):
    """What every operator asks of a tensor: on the GPU (that of `like`), no gradient, of this type and shape."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise X.XenosError(X.XENOS_EINVAL, f"{name} is no tensor on the GPU")
    if like is not None and t.device != like.device:
        raise X.XenosError(X.XENOS_EINVAL, f"{name} is on {t.device}, not on {like.device}")
    if dtype is not None and t.dtype != dtype:
        raise X.XenosError(X.XENOS_EINVAL, f"{name} is {t.dtype}, not {dtype}")
    if shape is not None and t.shape != shape:
        raise X.XenosError(X.XENOS_ESHAPE, f"{name} is {tuple(t.shape)}, not {tuple(shape)}")
    if t.requires_grad and torch.is_grad_enabled():
        raise X.XenosError(X.XENOS_EUNSUPPORTED, f"{name} requires a gradient: these operators have no backward pass")


def _float(t: torch.Tensor, name: str):
    _tensor(t, name)
    if t.dtype not in _DTYPE:
        raise X.XenosError(X.XENOS_EUNSUPPORTED, f"{name} is {t.dtype}: float32 and bfloat16 are supported")


def _on(t: torch.Tensor):
    """The tensor's device as the current one, for the launches."""
    return nullcontext() if t.device.index == torch.cuda.current_device() else torch.cuda.device(t.device)


def _stream(t: torch.Tensor) -> int:
    return torch.cuda.current_stream(t.device).cuda_stream


def _packed(t: Optional[torch.Tensor], name: str, like: torch.Tensor, shape, dtype=torch.float32) -> Optional[torch.Tensor]:
    """A contiguous tensor of this shape and type, or None."""
    if t is None:
        return None
    _tensor(t, name, like, dtype, shape)
    return t.contiguous()


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def quant_pitch(cols: int) -> int:
    """Bytes from one quantised row to the next (XENOS_QUANT_PITCH)."""
    return -(-cols // 128) * 128


def quantize_rows(x: torch.Tensor, gamma: Optional[torch.Tensor] = None, eps: float = 1e-5) -> Tuple[torch.Tensor, torch.Tensor]:
    """x [rows][cols] (float32 or bfloat16, any row stride) in 8 bits: (int8 [rows][quant_pitch(cols)] with zeros behind the columns, float32 scale [rows]).

    `gamma` [cols] (float32): the weights of an RMS norm in front, whose factor becomes part of the scale.  Weights of a layer [out][in] take
    the same form, a scale for each output channel."""
    _float(x, "x")
    _need(x.dim() == 2 and x.shape[1] > 0, X.XENOS_ESHAPE, f"x is {tuple(x.shape)}, not rows x columns")
    rows, cols = x.shape
    if x.stride(1) != 1 or (rows > 1 and x.stride(0) < cols):
        x = x.contiguous()
    gamma = _packed(gamma, "gamma", x, (cols,))
    q = torch.empty((rows, quant_pitch(cols)), dtype=torch.int8, device=x.device)
    scale = torch.empty(rows, dtype=torch.float32, device=x.device)
    with _on(x):
        X.xenos_quant_rows(x.data_ptr(), _DTYPE[x.dtype], rows, cols, x.stride(0), _ptr(gamma), eps, q.data_ptr(), scale.data_ptr(), _stream(x))
    return q, scale


def quant_matmul(q: torch.Tensor, scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, cols: int, *, bias: Optional[torch.Tensor] = None,
                 residual: Optional[torch.Tensor] = None, relu: bool = False, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """act(q w^T * scale * w_scale + bias + residual) [rows][out] of two quantised matrices of `cols` columns (quantize_rows)."""
    _tensor(q, "q", None, torch.int8)
    _need(q.dim() == 2 and cols > 0 and q.shape[1] == quant_pitch(cols), X.XENOS_ESHAPE, f"q is {tuple(q.shape)}, not rows of {quant_pitch(cols)} bytes for {cols} columns")
    _need(dtype in _DTYPE, X.XENOS_EUNSUPPORTED, f"{dtype}: float32 and bfloat16 are supported")
    _tensor(w, "w", q, torch.int8)
    _need(w.dim() == 2 and w.shape[1] == q.shape[1], X.XENOS_ESHAPE, f"w is {tuple(w.shape)}, not rows of {q.shape[1]} bytes")
    rows, out_c = q.shape[0], w.shape[0]
    q, w = q.contiguous(), w.contiguous()
    scale, w_scale, bias = _packed(scale, "scale", q, (rows,)), _packed(w_scale, "w_scale", q, (out_c,)), _packed(bias, "bias", q, (out_c,))
    if residual is not None:
        _tensor(residual, "residual", q, dtype, (rows, out_c))
        if residual.stride(1) != 1 or (rows > 1 and residual.stride(0) < out_c):
            residual = residual.contiguous()
    out = torch.empty((rows, out_c), dtype=dtype, device=q.device)
    args = X.QuantMatmulArgs(rows, cols, out_c, q.data_ptr(), scale.data_ptr(), w.data_ptr(), w_scale.data_ptr(), _ptr(bias), _ptr(residual),
                             0 if residual is None else residual.stride(0), int(relu), _DTYPE[dtype], out.data_ptr(), out_c)
    with _on(q):
        X.xenos_quant_matmul(args, _stream(q))
    return out


def linear(x: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, *, bias: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None,
           relu: bool = False, gamma: Optional[torch.Tensor] = None, eps: float = 1e-5) -> torch.Tensor:
    """A linear layer in 8-bit integers: x [..., in] (float32 or bfloat16) quantised row by row as it comes, times w (int8 [out][quant_pitch(in)], w_scale [out]: the
    layer's weights through quantize_rows, once).  `gamma`: an RMS norm in front; bias [out], then residual [..., out], then ReLU behind it."""
    _float(x, "x")
    _need(x.dim() >= 1, X.XENOS_ESHAPE, "x has no columns")
    _need(isinstance(w, torch.Tensor) and w.dim() == 2, X.XENOS_ESHAPE, "w is not a matrix")
    cols, lead = x.shape[-1], x.shape[:-1]
    flat = x.reshape(-1, cols) if x.dim() != 2 else x
    if residual is not None and x.dim() != 2:
        _tensor(residual, "residual", x, x.dtype, (*lead, w.shape[0]))
        residual = residual.reshape(-1, w.shape[0])
    q, scale = quantize_rows(flat, gamma, eps)
    y = quant_matmul(q, scale, w, w_scale, cols, bias=bias, residual=residual, relu=relu, dtype=x.dtype)
    return y if x.dim() == 2 else y.view(*lead, w.shape[0])
