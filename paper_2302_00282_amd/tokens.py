"""The operators of a token model's serving step on torch tensors: 8-bit linear layers, the quantised cache of keys and values, the
attention that reads it, and what is read from the logits.

Each function checks its tensors, allocates what it returns, and makes one call of the C ABI (include/xenos.h) on torch's current
stream of the tensors' device; nothing synchronises.  The kernels are the library's own: there is no CPU path.  Forward passes only: what
they return carries no gradient, and an input that asks for one, or has a tangent, is refused.
"""
from __future__ import annotations

import math
from typing import Optional, Tuple

import torch
import torch.autograd.forward_ad as _forward

from . import xenos as X

# A call of few rows takes the GPU a few microseconds, so the host's part is kept as short: tensors are looked at once, messages are made only for what is refused, and the
# stream's handle is asked for without making a Stream object of it (0.1 us in place of 2 us).
_raw_stream = torch._C._cuda_getCurrentRawStream
_DTYPE = {torch.float32: X.XENOS_F32, torch.bfloat16: X.XENOS_BF16}
_INT_MAX = (1 << 31) - 1      # (sizes are ints of the C ABI, and ctypes keeps the lower bits of a larger one)


def _refuse(status: int, message: str):
    raise X.XenosError(status, message)


def _check(t: torch.Tensor, name: str, device: Optional[int], dtype=None, shape=None) -> torch.Tensor:
    """What every operator asks of a tensor: on the GPU `device`, of this type (None: float32 or bfloat16) and shape, without a gradient."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _refuse(X.XENOS_EINVAL, f"{name} is no tensor on the GPU")
    if device is not None and t.get_device() != device:
        _refuse(X.XENOS_EINVAL, f"{name} is on {t.device}, not on cuda:{device}")
    if dtype is None:
        if t.dtype not in _DTYPE:
            _refuse(X.XENOS_EUNSUPPORTED, f"{name} is {t.dtype}: float32 and bfloat16 are supported")
    elif t.dtype != dtype:
        _refuse(X.XENOS_EINVAL, f"{name} is {t.dtype}, not {dtype}")
    if shape is not None and t.shape != shape:
        _refuse(X.XENOS_ESHAPE, f"{name} is {tuple(t.shape)}, not {tuple(shape)}")
    if t.requires_grad and torch.is_grad_enabled():
        _refuse(X.XENOS_EUNSUPPORTED, f"{name} requires a gradient: these operators have no backward pass")
    return t


def _no_tangents(*tensors: Optional[torch.Tensor]):
    """Inside a level of forward-mode differentiation (asked once a call): no input has a tangent."""
    for t in tensors:
        if isinstance(t, torch.Tensor) and t.is_floating_point() and _forward.unpack_dual(t).tangent is not None:
            _refuse(X.XENOS_EUNSUPPORTED, f"an input {tuple(t.shape)} has a tangent: these operators have no derivatives")


def _too_many(what: str):
    _refuse(X.XENOS_EUNSUPPORTED, f"{what}: sizes of at most {_INT_MAX}")


def _needed(t: torch.Tensor, name: str, device: int, shape, dtype=torch.float32) -> torch.Tensor:
    """A contiguous tensor of this shape and type."""
    return _check(t, name, device, dtype, shape).contiguous()


def _given(t: Optional[torch.Tensor], name: str, device: int, shape, dtype=torch.float32) -> Optional[torch.Tensor]:
    """The same, or None."""
    return None if t is None else _check(t, name, device, dtype, shape).contiguous()


def _address(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _launch(device: int, call, *args):
    """call(*args, stream) with `device` as the current one."""
    if device == torch.cuda.current_device():
        call(*args, _raw_stream(device))
    else:
        with torch.cuda.device(device):
            call(*args, _raw_stream(device))


def _rows(t: torch.Tensor) -> torch.Tensor:
    """A matrix whose rows are contiguous and do not overlap."""
    stride = t.stride()
    return t if stride[1] == 1 and (stride[0] >= t.shape[1] or t.shape[0] <= 1) else t.contiguous()


def quant_pitch(cols: int) -> int:
    """Bytes from one quantised row to the next (XENOS_QUANT_PITCH)."""
    return -(-cols // 128) * 128


def quantize_rows(x: torch.Tensor, gamma: Optional[torch.Tensor] = None, eps: float = 1e-5) -> Tuple[torch.Tensor, torch.Tensor]:
    """x [rows][cols] (float32 or bfloat16, any row stride) in 8 bits: (int8 [rows][quant_pitch(cols)] with zeros behind the columns, float32 scale [rows]).

    `gamma` [cols] (float32): the weights of an RMS norm in front, whose factor becomes part of the scale.  Weights of a layer [out][in] take
    the same form, a scale for each output channel."""
    device = _check(x, "x", None).get_device()
    if x.dim() != 2 or x.shape[1] == 0:
        _refuse(X.XENOS_ESHAPE, f"x is {tuple(x.shape)}, not rows x columns")
    rows, cols = x.shape
    if rows > _INT_MAX or cols > _INT_MAX:
        _too_many(f"x is {rows} x {cols}")
    x, gamma = _rows(x), _given(gamma, "gamma", device, (cols,))
    if _forward._current_level >= 0:
        _no_tangents(x, gamma)
    q, scale = x.new_empty((rows, quant_pitch(cols)), dtype=torch.int8), x.new_empty(rows, dtype=torch.float32)
    _launch(device, X.xenos_quant_rows, x.data_ptr(), _DTYPE[x.dtype], rows, cols, x.stride(0), _address(gamma), eps, q.data_ptr(), scale.data_ptr())
    return q, scale


def _weights(w: torch.Tensor, device: int, cols: int) -> torch.Tensor:
    _check(w, "w", device, torch.int8)
    if w.dim() != 2 or w.shape[1] != quant_pitch(cols):
        _refuse(X.XENOS_ESHAPE, f"w is {tuple(w.shape)}, not rows of {quant_pitch(cols)} bytes for {cols} columns")
    if w.shape[0] > _INT_MAX:
        _too_many(f"w is {tuple(w.shape)}")
    return w.contiguous()


def quant_matmul(q: torch.Tensor, scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, cols: int, *, bias: Optional[torch.Tensor] = None,
                 residual: Optional[torch.Tensor] = None, relu: bool = False, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """act(q w^T * scale * w_scale + bias + residual) [rows][out] of two quantised matrices of `cols` columns (quantize_rows)."""
    device = _check(q, "q", None, torch.int8).get_device()
    if q.dim() != 2 or cols <= 0 or q.shape[1] != quant_pitch(cols):
        _refuse(X.XENOS_ESHAPE, f"q is {tuple(q.shape)}, not rows of {quant_pitch(cols)} bytes for {cols} columns")
    if dtype not in _DTYPE:
        _refuse(X.XENOS_EUNSUPPORTED, f"{dtype}: float32 and bfloat16 are supported")
    if q.shape[0] > _INT_MAX or cols > _INT_MAX:
        _too_many(f"q is {tuple(q.shape)}")
    q, w = q.contiguous(), _weights(w, device, cols)
    rows, out_c = q.shape[0], w.shape[0]
    scale, w_scale, bias = _needed(scale, "scale", device, (rows,)), _needed(w_scale, "w_scale", device, (out_c,)), _given(bias, "bias", device, (out_c,))
    if residual is not None:
        residual = _rows(_check(residual, "residual", device, dtype, (rows, out_c)))
    if _forward._current_level >= 0:
        _no_tangents(scale, w_scale, bias, residual)
    out = q.new_empty((rows, out_c), dtype=dtype)
    args = X.QuantMatmulArgs(rows, cols, out_c, q.data_ptr(), scale.data_ptr(), w.data_ptr(), w_scale.data_ptr(), _address(bias), _address(residual),
                             0 if residual is None else residual.stride(0), relu, _DTYPE[dtype], out.data_ptr(), out_c)
    _launch(device, X.xenos_quant_matmul, args)
    return out


def linear(x: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, *, bias: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None,
           relu: bool = False, gamma: Optional[torch.Tensor] = None, eps: float = 1e-5) -> torch.Tensor:
    """A linear layer in 8-bit integers: x [..., in] (float32 or bfloat16) quantised row by row as it comes, times w (int8 [out][quant_pitch(in)], w_scale [out]: the
    layer's weights through quantize_rows, once).  `gamma`: an RMS norm in front; bias [out], then residual [..., out], then ReLU behind it."""
    device = _check(x, "x", None).get_device()
    shape = x.shape
    if len(shape) == 0 or shape[-1] == 0:
        _refuse(X.XENOS_ESHAPE, f"x is {tuple(shape)}, without columns")
    cols = shape[-1]
    if cols > _INT_MAX or x.numel() // cols > _INT_MAX:
        _too_many(f"x is {tuple(shape)}")
    w = _weights(w, device, cols)
    out_c = w.shape[0]
    if residual is not None:
        _check(residual, "residual", device, x.dtype, (*shape[:-1], out_c))
    if len(shape) != 2:
        x = x.reshape(-1, cols)
        residual = None if residual is None else residual.reshape(x.shape[0], out_c)
    x, residual, rows = _rows(x), None if residual is None else _rows(residual), x.shape[0]
    w_scale, bias, gamma = _needed(w_scale, "w_scale", device, (out_c,)), _given(bias, "bias", device, (out_c,)), _given(gamma, "gamma", device, (cols,))
    if _forward._current_level >= 0:
        _no_tangents(x, w_scale, bias, residual, gamma)
    out = x.new_empty((rows, out_c))
    need = X.xenos_linear_workspace(rows, cols, out_c) if cols <= X.XENOS_QUANT_MAX_COLS else 0
    workspace = x.new_empty(need, dtype=torch.uint8) if need else None
    args = X.LinearArgs(rows, cols, out_c, _DTYPE[x.dtype], x.data_ptr(), x.stride(0), _address(gamma), eps, w.data_ptr(), w_scale.data_ptr(), _address(bias),
                        _address(residual), 0 if residual is None else residual.stride(0), relu, out.data_ptr(), out_c)
    _launch(device, X.xenos_linear, args, _address(workspace), need)
    return out if len(shape) == 2 else out.view(*shape[:-1], out_c)


class KVCache:
    """Keys and values of tokens in 8-bit integers with a scale for each token and head, in pages (the layout: xenos_cache in include/xenos.h).

    The tensors are the caller's: k int8 [pages][heads][page][dim], v int8 [pages][heads][page / 16][dim][16], scales float32 [pages][heads][page].
    Which page holds which tokens is the caller's too; a token's slot is page * page_tokens + its place in the page."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor):
        device = _check(k, "k", None, torch.int8).get_device()
        if k.dim() != 4:
            _refuse(X.XENOS_ESHAPE, f"k is {tuple(k.shape)}, not pages x heads x tokens x dimensions")
        n, heads, page, dim = k.shape
        if n > _INT_MAX or heads > _INT_MAX or page > _INT_MAX:
            _too_many(f"k is {tuple(k.shape)}")
        _check(v, "v", device, torch.int8, (n, heads, page // 16, dim, 16))
        _check(k_scale, "k_scale", device, torch.float32, (n, heads, page))
        _check(v_scale, "v_scale", device, torch.float32, (n, heads, page))
        if page % 16 or dim % 16 or not 0 < dim <= 256:
            _refuse(X.XENOS_EUNSUPPORTED, f"pages of {page} tokens, heads of {dim} values (multiples of 16, at most 256 values)")
        if not (k.is_contiguous() and v.is_contiguous() and k_scale.is_contiguous() and v_scale.is_contiguous()):
            _refuse(X.XENOS_ESHAPE, "the cache's tensors are not contiguous")
        if _forward._current_level >= 0:
            _no_tangents(k_scale, v_scale)
        self.k, self.v, self.k_scale, self.v_scale, self.device = k, v, k_scale, v_scale, device
        self.n_pages, self.heads, self.page_tokens, self.head_dim = n, heads, page, dim
        self.desc = X.Cache(n, page, heads, dim, k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr())

    @classmethod
    def empty(cls, n_pages: int, page_tokens: int, heads: int, head_dim: int, device="cuda") -> "KVCache":
        """A cache of that many pages; nothing in it is read before it is written."""
        if page_tokens <= 0 or page_tokens % 16:
            _refuse(X.XENOS_EUNSUPPORTED, f"pages of {page_tokens} tokens (a multiple of 16)")
        ints, floats = dict(dtype=torch.int8, device=device), dict(dtype=torch.float32, device=device)
        return cls(torch.empty((n_pages, heads, page_tokens, head_dim), **ints), torch.empty((n_pages, heads, page_tokens // 16, head_dim, 16), **ints),
                   torch.empty((n_pages, heads, page_tokens), **floats), torch.empty((n_pages, heads, page_tokens), **floats))

    def write(self, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor):
        """Quantises the keys and values [tokens][heads][dim] (float32 or bfloat16, any strides of tokens and heads) into the slots (int64 [tokens], each once;
        one below 0 or beyond the cache: that token is not stored)."""
        _check(k, "k", self.device)
        shape = k.shape
        if len(shape) != 3 or shape[1] != self.heads or shape[2] != self.head_dim:
            _refuse(X.XENOS_ESHAPE, f"k is {tuple(shape)}, not tokens x {self.heads} x {self.head_dim}")
        if shape[0] > _INT_MAX:
            _too_many(f"k is {tuple(shape)}")
        _check(v, "v", self.device, k.dtype, shape)
        slots = _needed(slots, "slots", self.device, shape[:1], torch.int64)
        if _forward._current_level >= 0:
            _no_tangents(k, v)
        if k.stride(2) != 1:
            k = k.contiguous()
        if v.stride(2) != 1:
            v = v.contiguous()
        ks, vs = k.stride(), v.stride()
        _launch(self.device, X.xenos_cache_write, self.desc, shape[0], k.data_ptr(), ks[0], ks[1], v.data_ptr(), vs[0], vs[1], _DTYPE[k.dtype], slots.data_ptr())

    def read(self, slots: torch.Tensor, dtype: torch.dtype = torch.bfloat16) -> Tuple[torch.Tensor, torch.Tensor]:
        """The keys and values of the slots (int64 [tokens]) as the numbers they stand for, [tokens][heads][dim] each; zeros for a slot that is none."""
        _check(slots, "slots", self.device, torch.int64)
        if slots.dim() != 1:
            _refuse(X.XENOS_ESHAPE, f"slots is {tuple(slots.shape)}, not a list")
        if slots.shape[0] > _INT_MAX:
            _too_many(f"slots is {tuple(slots.shape)}")
        if dtype not in _DTYPE:
            _refuse(X.XENOS_EUNSUPPORTED, f"{dtype}: float32 and bfloat16 are supported")
        slots = slots.contiguous()
        shape = (slots.shape[0], self.heads, self.head_dim)
        k, v = slots.new_empty(shape, dtype=dtype), slots.new_empty(shape, dtype=dtype)
        _launch(self.device, X.xenos_cache_read, self.desc, shape[0], slots.data_ptr(), k.data_ptr(), v.data_ptr(), _DTYPE[dtype])
        return k, v


def attention(q: torch.Tensor, cache: KVCache, tables: torch.Tensor, lengths: torch.Tensor, *, starts: Optional[torch.Tensor] = None, max_queries: int = 1,
              max_length: Optional[int] = None, prefix_table: Optional[torch.Tensor] = None, prefix_length: int = 0, scale: Optional[float] = None,
              out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of q bfloat16 [queries][heads][dim] (any strides of tokens and heads) to the cache; heads: a multiple of the cache's. Returns [queries][heads][dim].

    Sequence b has lengths[b] (int32 [sequences]) tokens in the pages tables[b] (int32 [sequences][pages], entries behind its last page are not looked at) behind `prefix_length`
    tokens in the pages `prefix_table` (int32) that all sequences share.  Its queries, rows starts[b] .. starts[b + 1] of q (int32 [sequences + 1]; None: row b alone), are the last of
    its tokens, already in the cache, and each sees the prefix and the tokens up to itself; rows of q that no sequence has see the prefix alone.  max_queries, max_length: what no sequence exceeds
    (max_length None: what its table holds); they decide how the work is shared out and cost no look at the lengths.  scale: None is 1 / sqrt(dim)."""
    device, dim = cache.device, cache.head_dim
    _check(q, "q", device)
    shape, ts = q.shape, tables.shape if isinstance(tables, torch.Tensor) else ()
    if q.dtype != torch.bfloat16:
        _refuse(X.XENOS_EUNSUPPORTED, f"q is {q.dtype}: bfloat16 is supported")
    if len(shape) != 3 or shape[2] != dim or shape[1] == 0 or shape[1] % cache.heads:
        _refuse(X.XENOS_ESHAPE, f"q is {tuple(shape)}, not queries x a multiple of {cache.heads} heads x {dim}")
    n_queries, heads, _ = shape
    if len(ts) != 2:
        _refuse(X.XENOS_ESHAPE, f"tables is {tuple(ts)}, not sequences x pages")
    n_seqs, pages = ts
    if max_length is None:
        max_length = pages * cache.page_tokens
    if n_queries > _INT_MAX or heads > _INT_MAX or n_seqs > _INT_MAX or pages > _INT_MAX or max_length > _INT_MAX or prefix_length > _INT_MAX:
        _too_many(f"{n_queries} queries of {heads} heads, tables of {tuple(ts)}, up to {max_length} tokens behind {prefix_length}")
    tables = _needed(tables, "tables", device, None, torch.int32)
    lengths, starts = _needed(lengths, "lengths", device, (n_seqs,), torch.int32), _given(starts, "starts", device, (n_seqs + 1,), torch.int32)
    if starts is None and n_queries != n_seqs:
        _refuse(X.XENOS_ESHAPE, f"{n_queries} queries of {n_seqs} sequences, and no starts")
    prefix_table = _given(prefix_table, "prefix_table", device, None, torch.int32)
    if prefix_length and not 0 < prefix_length <= (0 if prefix_table is None else prefix_table.numel() * cache.page_tokens):
        _refuse(X.XENOS_ESHAPE, f"a prefix of {prefix_length} tokens in {0 if prefix_table is None else prefix_table.numel()} pages of {cache.page_tokens}")
    if _forward._current_level >= 0:
        _no_tangents(q)
    if q.stride(2) != 1:
        q = q.contiguous()
    if out is None:
        out = q.new_empty(shape)
    elif _check(out, "out", device, q.dtype, shape).stride(2) != 1:
        _refuse(X.XENOS_ESHAPE, "the rows of out are not contiguous")
    qs, os = q.stride(), out.stride()
    args = X.AttentionArgs(n_seqs, n_queries, heads, X.XENOS_BF16, q.data_ptr(), qs[0], qs[1], out.data_ptr(), os[0], os[1], _address(starts), lengths.data_ptr(),
                           tables.data_ptr(), pages, max_queries if max_queries < n_queries else n_queries, max_length, _address(prefix_table), prefix_length,
                           1.0 / math.sqrt(dim) if scale is None else scale)
    need = X.xenos_attention_workspace(cache.desc, args)
    workspace = q.new_empty(need, dtype=torch.uint8) if need else None
    _launch(device, X.xenos_attention, cache.desc, args, _address(workspace), need)
    return out


def logprobs(logits: torch.Tensor, targets: Optional[torch.Tensor] = None, top: int = 0):
    """Log probabilities of given tokens, entropy, and the likeliest tokens of each position: logits [positions][vocab] (float32 or bfloat16, any row stride),
    targets int64 [positions] or None.

    Returns (logprob float32 [positions] or None, entropy float32 [positions], top_logprob float32 [positions][top], top_token int32 [positions][top]): the tokens
    from the likeliest on, equal ones by the lowest index.  A target outside 0 .. vocab - 1 is none, and its logprob 0."""
    device = _check(logits, "logits", None).get_device()
    if logits.dim() != 2 or logits.shape[1] == 0:
        _refuse(X.XENOS_ESHAPE, f"logits is {tuple(logits.shape)}, not positions x tokens")
    rows, vocab = logits.shape
    if rows > _INT_MAX or vocab > _INT_MAX:
        _too_many(f"logits is {rows} x {vocab}")
    if not 0 <= top <= X.XENOS_TOP_MAX:
        _refuse(X.XENOS_EUNSUPPORTED, f"the best {top} tokens (at most {X.XENOS_TOP_MAX})")
    if top > vocab:
        _refuse(X.XENOS_ESHAPE, f"the best {top} of {vocab} tokens")
    targets, logits = _given(targets, "targets", device, (rows,), torch.int64), _rows(logits)
    if _forward._current_level >= 0:
        _no_tangents(logits)
    given = None if targets is None else logits.new_empty(rows, dtype=torch.float32)
    entropy, best, token = logits.new_empty(rows, dtype=torch.float32), logits.new_empty((rows, top), dtype=torch.float32), logits.new_empty((rows, top), dtype=torch.int32)
    need = X.xenos_logprobs_workspace(rows, vocab, top)
    workspace = logits.new_empty(need, dtype=torch.uint8) if need else None
    _launch(device, X.xenos_logprobs, logits.data_ptr(), _DTYPE[logits.dtype], rows, vocab, logits.stride(0), _address(targets), top, _address(given), entropy.data_ptr(),
            best.data_ptr(), token.data_ptr(), _address(workspace), need)
    return given, entropy, best, token
