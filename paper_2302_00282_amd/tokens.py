"""The operators of a token model's serving step on torch tensors: 8-bit linear layers, the quantised cache of keys and values, the
attention that reads it, and what is read from the logits.

Each function checks its tensors, allocates what it returns, and makes one or two calls of the C ABI (include/xenos.h) on torch's current
stream of the tensors' device; nothing synchronises.  The kernels are the library's own: there is no CPU path.  Forward passes only: what
they return carries no gradient, and an input that asks for one is refused.
"""
from __future__ import annotations

import math
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


class KVCache:
    """Keys and values of tokens in 8-bit integers with a scale for each token and head, in pages (the layout: xenos_cache in include/xenos.h).

    The tensors are the caller's: k int8 [pages][heads][page][dim], v int8 [pages][heads][page / 16][dim][16], scales float32 [pages][heads][page].
    Which page holds which tokens is the caller's too; a token's slot is page * page_tokens + its place in the page."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor):
        _tensor(k, "k", None, torch.int8)
        _need(k.dim() == 4, X.XENOS_ESHAPE, f"k is {tuple(k.shape)}, not pages x heads x tokens x dimensions")
        n, heads, page, dim = k.shape
        _tensor(v, "v", k, torch.int8, (n, heads, page // 16, dim, 16))
        _tensor(k_scale, "k_scale", k, torch.float32, (n, heads, page))
        _tensor(v_scale, "v_scale", k, torch.float32, (n, heads, page))
        _need(page % 16 == 0 and dim % 16 == 0 and 0 < dim <= 256, X.XENOS_EUNSUPPORTED, f"pages of {page} tokens, heads of {dim} values (multiples of 16, at most 256 values)")
        _need(k.is_contiguous() and v.is_contiguous() and k_scale.is_contiguous() and v_scale.is_contiguous(), X.XENOS_ESHAPE, "the cache's tensors are not contiguous")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_pages, self.heads, self.page_tokens, self.head_dim = n, heads, page, dim
        self.desc = X.Cache(n, page, heads, dim, k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr())

    @classmethod
    def empty(cls, n_pages: int, page_tokens: int, heads: int, head_dim: int, device="cuda") -> "KVCache":
        """A cache of that many pages; nothing in it is read before it is written."""
        _need(page_tokens > 0 and page_tokens % 16 == 0, X.XENOS_EUNSUPPORTED, f"pages of {page_tokens} tokens (a multiple of 16)")
        ints, floats = dict(dtype=torch.int8, device=device), dict(dtype=torch.float32, device=device)
        return cls(torch.empty((n_pages, heads, page_tokens, head_dim), **ints), torch.empty((n_pages, heads, page_tokens // 16, head_dim, 16), **ints),
                   torch.empty((n_pages, heads, page_tokens), **floats), torch.empty((n_pages, heads, page_tokens), **floats))

    def write(self, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor):
        """Quantises the keys and values [tokens][heads][dim] (float32 or bfloat16, any strides of tokens and heads) into the slots (int64 [tokens], each once;
        one below 0 or beyond the cache: that token is not stored)."""
        _float(k, "k")
        _need(k.dim() == 3 and k.shape[1] == self.heads and k.shape[2] == self.head_dim, X.XENOS_ESHAPE, f"k is {tuple(k.shape)}, not tokens x {self.heads} x {self.head_dim}")
        _tensor(k, "k", self.k)
        _tensor(v, "v", self.k, k.dtype, k.shape)
        _tensor(slots, "slots", self.k, torch.int64, k.shape[:1])
        k, v, slots = k if k.stride(2) == 1 else k.contiguous(), v if v.stride(2) == 1 else v.contiguous(), slots.contiguous()
        with _on(k):
            X.xenos_cache_write(self.desc, k.shape[0], k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(), v.stride(0), v.stride(1), _DTYPE[k.dtype],
                                slots.data_ptr(), _stream(k))

    def read(self, slots: torch.Tensor, dtype: torch.dtype = torch.bfloat16) -> Tuple[torch.Tensor, torch.Tensor]:
        """The keys and values of the slots (int64 [tokens]) as the numbers they stand for, [tokens][heads][dim] each; zeros for a slot that is none."""
        _tensor(slots, "slots", self.k, torch.int64)
        _need(slots.dim() == 1, X.XENOS_ESHAPE, f"slots is {tuple(slots.shape)}, not a list")
        _need(dtype in _DTYPE, X.XENOS_EUNSUPPORTED, f"{dtype}: float32 and bfloat16 are supported")
        slots = slots.contiguous()
        k, v = (torch.empty((slots.shape[0], self.heads, self.head_dim), dtype=dtype, device=slots.device) for _ in range(2))
        with _on(slots):
            X.xenos_cache_read(self.desc, slots.shape[0], slots.data_ptr(), k.data_ptr(), v.data_ptr(), _DTYPE[dtype], _stream(slots))
        return k, v


def attention(q: torch.Tensor, cache: KVCache, tables: torch.Tensor, lengths: torch.Tensor, *, starts: Optional[torch.Tensor] = None, max_queries: int = 1,
              max_length: Optional[int] = None, prefix_table: Optional[torch.Tensor] = None, prefix_length: int = 0, scale: Optional[float] = None,
              out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of q bfloat16 [queries][heads][dim] (any strides of tokens and heads) to the cache; heads: a multiple of the cache's. Returns [queries][heads][dim].

    Sequence b has lengths[b] (int32 [sequences]) tokens in the pages tables[b] (int32 [sequences][pages], entries behind its last page are not looked at) behind `prefix_length`
    tokens in the pages `prefix_table` (int32) that all sequences share.  Its queries, rows starts[b] .. starts[b + 1] of q (int32 [sequences + 1]; None: row b alone), are the last of
    its tokens, already in the cache, and each sees the prefix and the tokens up to itself.  max_queries, max_length: what no sequence exceeds
    (max_length None: what its table holds); they decide how the work is shared out and cost no look at the lengths.  scale: None is 1 / sqrt(dim)."""
    _tensor(q, "q", cache.k)
    _need(q.dtype == torch.bfloat16, X.XENOS_EUNSUPPORTED, f"q is {q.dtype}: bfloat16 is supported")
    _need(q.dim() == 3 and q.shape[2] == cache.head_dim and q.shape[1] > 0 and q.shape[1] % cache.heads == 0, X.XENOS_ESHAPE,
          f"q is {tuple(q.shape)}, not queries x a multiple of {cache.heads} heads x {cache.head_dim}")
    _tensor(lengths, "lengths", q, torch.int32)
    _tensor(tables, "tables", q, torch.int32)
    _need(lengths.dim() == 1 and tables.dim() == 2 and tables.shape[0] == lengths.shape[0], X.XENOS_ESHAPE, f"{tuple(tables.shape)} tables of {tuple(lengths.shape)} sequences")
    n_seqs, n_queries = lengths.shape[0], q.shape[0]
    starts = _packed(starts, "starts", q, (n_seqs + 1,), torch.int32)
    _need(starts is not None or n_queries == n_seqs, X.XENOS_ESHAPE, f"{n_queries} queries of {n_seqs} sequences, and no starts")
    if prefix_table is not None:
        _tensor(prefix_table, "prefix_table", q, torch.int32)
        prefix_table = prefix_table.contiguous()
    held = 0 if prefix_table is None else prefix_table.numel() * cache.page_tokens
    _need(0 <= prefix_length <= held, X.XENOS_ESHAPE, f"a prefix of {prefix_length} tokens in pages of {held}")
    q = q if q.stride(2) == 1 else q.contiguous()
    tables, lengths = tables.contiguous(), lengths.contiguous()
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    else:
        _tensor(out, "out", q, q.dtype, q.shape)
        _need(out.stride(2) == 1, X.XENOS_ESHAPE, "the rows of out are not contiguous")
    args = X.AttentionArgs(n_seqs, n_queries, q.shape[1], X.XENOS_BF16, q.data_ptr(), q.stride(0), q.stride(1), out.data_ptr(), out.stride(0), out.stride(1),
                           _ptr(starts), lengths.data_ptr(), tables.data_ptr(), tables.shape[1], max_queries, tables.shape[1] * cache.page_tokens if max_length is None else max_length,
                           _ptr(prefix_table), prefix_length, 1.0 / math.sqrt(cache.head_dim) if scale is None else scale)
    need = X.xenos_attention_workspace(cache.desc, args)
    workspace = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    with _on(q):
        X.xenos_attention(cache.desc, args, _ptr(workspace), need, _stream(q))
    return out


def logprobs(logits: torch.Tensor, targets: Optional[torch.Tensor] = None, top: int = 0):
    """Log probabilities of given tokens, entropy, and the likeliest tokens of each position: logits [positions][vocab] (float32 or bfloat16, any row stride),
    targets int64 [positions] or None.

    Returns (logprob float32 [positions] or None, entropy float32 [positions], top_logprob float32 [positions][top], top_token int32 [positions][top]): the tokens
    from the likeliest on, equal ones by the lowest index.  A target outside 0 .. vocab - 1 is none, and its logprob 0."""
    _float(logits, "logits")
    _need(logits.dim() == 2 and logits.shape[1] > 0, X.XENOS_ESHAPE, f"logits is {tuple(logits.shape)}, not positions x tokens")
    rows, vocab = logits.shape
    _need(0 <= top <= X.XENOS_TOP_MAX, X.XENOS_EUNSUPPORTED, f"the best {top} tokens (at most {X.XENOS_TOP_MAX})")
    _need(top <= vocab, X.XENOS_ESHAPE, f"the best {top} of {vocab} tokens")
    if targets is not None:
        _tensor(targets, "targets", logits, torch.int64, (rows,))
        targets = targets.contiguous()
    if logits.stride(1) != 1 or (rows > 1 and logits.stride(0) < vocab):
        logits = logits.contiguous()
    floats = dict(dtype=torch.float32, device=logits.device)
    given = None if targets is None else torch.empty(rows, **floats)
    entropy, best = torch.empty(rows, **floats), torch.empty((rows, top), **floats)
    token = torch.empty((rows, top), dtype=torch.int32, device=logits.device)
    need = X.xenos_logprobs_workspace(rows, vocab, top)
    workspace = torch.empty(need, dtype=torch.uint8, device=logits.device) if need else None
    with _on(logits):
        X.xenos_logprobs(logits.data_ptr(), _DTYPE[logits.dtype], rows, vocab, logits.stride(0), _ptr(targets), top, _ptr(given), entropy.data_ptr(),
                         best.data_ptr(), token.data_ptr(), _ptr(workspace), need, _stream(logits))
    return given, entropy, best, token
