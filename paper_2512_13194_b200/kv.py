"""A key/value cache held in 4 bits beside the verification step (include/ears.h, "A key/value cache held in 4 bits"):
writing tokens into its pages, reading them back as values, and attention of the newest positions over it, full or with a
sliding window and first tokens that stay visible.  Argument marshalling only; every computation runs in the CUDA library.

A pass over K + 1 tokens per sequence calls ``kv_write`` and ``kv_attention`` in each layer with the same ``pages``, ``start`` and
``counts``; of those tokens the verification step keeps ``accept_len + 1``, and ``kv_advance`` (or ``EarsSampler`` with ``kv_start``)
moves ``start`` there without a word to the host.  What was written behind is overwritten by the next pass.

``pages`` [B, W], ``start`` [B] and ``counts`` [B] (optional) are integer CUDA tensors, int32 where nothing is to be converted (integers
that 32 bits cannot hold stay unusable); keys, values and queries are used where they lie as long as the elements of a head
are contiguous.  Serving only: inputs that require a gradient, a cache's ``params`` among them, are refused.
``status``: optional int32 CUDA tensor of one element that gets EARS_DEV_INVALID_INPUT OR-ed in where a position lies outside the
page table or a page outside the pool.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch
from torch.autograd import forward_ad

from . import rows
from .binding import KvCacheStruct, _check, load_library

GROUP = 64
HEAD_DIMS = (64, 128, 256)
_DTYPES = rows._DTYPES
_ptr = rows._ptr


class KVCache(NamedTuple):
    """The pool: ``codes`` uint8 [pages, 2, heads, page_size, head_dim / 2], ``params`` bfloat16 [pages, 2, heads, page_size,
    head_dim / 64, 2] (scale, minimum), contiguous CUDA tensors."""
    codes: torch.Tensor
    params: torch.Tensor

    @property
    def page_size(self) -> int:
        return self.codes.shape[3]

    @property
    def heads(self) -> int:
        return self.codes.shape[2]

    @property
    def head_dim(self) -> int:
        return self.codes.shape[4] * 2


def kv_cache(pages: int, heads: int, head_dim: int, page_size: int = 64, *, device="cuda") -> KVCache:
    """An empty pool of ``pages`` pages of ``page_size`` tokens (a multiple of 16); head_dim 64, 128 or 256.  4.5 bits a value."""
    if head_dim not in HEAD_DIMS:
        raise ValueError(f"head_dim must be one of {HEAD_DIMS}")
    if pages < 1 or heads < 1 or page_size < 16 or page_size % 16:
        raise ValueError("a pool has at least one page and one head, and pages of a multiple of 16 tokens")
    lead = (pages, 2, heads, page_size)
    return KVCache(torch.zeros(lead + (head_dim // 2,), dtype=torch.uint8, device=device),
                   torch.zeros(lead + (head_dim // GROUP, 2), dtype=torch.bfloat16, device=device))


def _refuse_gradients(*tensors) -> None:
    for t in tensors:
        if isinstance(t, torch.Tensor) and (t.requires_grad and torch.is_grad_enabled()
                                            or forward_ad._current_level >= 0 and forward_ad.unpack_dual(t).tangent is not None):
            raise NotImplementedError("the cache's operators have no gradient")


def _plain():
    """The extension module's calls, which leave everything that is not in its plain form (a gradient asked for, too) to the ones
    here; nothing is plain while forward-mode derivatives are taken."""
    return rows._plain_calls() if forward_ad._current_level < 0 else rows._Ctypes


def _on_stream(stream, cache, fn, *args, **kwargs):
    """``stream=``: the whole call, its conversions and outputs included, belongs to that stream as under torch.cuda.stream."""
    if stream.device_index != cache.codes.get_device():
        raise ValueError("the stream must belong to the cache's device")
    with torch.cuda.stream(stream):
        return fn(*args, **kwargs)


class _Call:
    """The common part of a call: cache, page table, positions, status."""

    __slots__ = ("index", "cache", "held", "table", "status", "B", "heads", "head_dim")

    def __init__(self, cache, pages, start, counts, status):
        codes, params = cache
        self.index = index = codes.get_device()
        if index < 0 or params.get_device() != index:
            raise ValueError("the cache must consist of CUDA tensors of one device")
        if codes.dtype != torch.uint8 or params.dtype != torch.bfloat16:
            raise TypeError("a cache has uint8 codes and bfloat16 params")
        if codes.dim() != 5 or codes.shape[1] != 2 or codes.shape[4] * 2 not in HEAD_DIMS \
                or params.shape != codes.shape[:4] + (codes.shape[4] * 2 // GROUP, 2):
            raise ValueError("expected codes [pages, 2, heads, page_size, head_dim / 2] and params [pages, 2, heads, page_size, head_dim / 64, 2]")
        if not codes.is_contiguous() or not params.is_contiguous():
            raise ValueError("the cache must be contiguous")
        self.heads, self.head_dim = codes.shape[2], codes.shape[4] * 2
        self.cache = KvCacheStruct(codes.data_ptr(), params.data_ptr(), codes.shape[0], self.heads, codes.shape[3], self.head_dim)
        if pages.dim() != 2:
            raise ValueError("expected pages [B, W]")
        self.B = pages.shape[0]
        table = self.ints(pages, tuple(pages.shape), "pages")
        start = self.ints(start, (self.B,), "start").contiguous()
        counts = None if counts is None else self.ints(counts, (self.B,), "counts").contiguous()
        if table.shape[1] > 1 and table.stride(1) != 1 or table.stride(0) < 0:
            table = table.contiguous()
        if status is not None and (status.get_device() != index or status.dtype != torch.int32 or status.numel() != 1):
            raise ValueError("status must be an int32 CUDA tensor of one element on the cache's device")
        self.held = (table, start, counts)         # alive until the call is enqueued
        self.status = status
        self.table = (table.data_ptr(), table.shape[1], table.stride(0), start.data_ptr(), _ptr(counts))

    def ints(self, t, shape, name):
        if t.get_device() != self.index:
            raise ValueError(f"{name} must live on the cache's device")
        if tuple(t.shape) != shape:
            raise ValueError(f"{name} must have shape {list(shape)}, got {list(t.shape)}")
        if t.dtype is not torch.int32:
            if t.dtype.is_floating_point or t.dtype.is_complex or t.dtype is torch.bool:
                raise TypeError(f"{name} must hold integers")
            t = rows._within_int32(t).to(torch.int32)
        return t

    def heads_of(self, t, name, heads=None):
        """[B, Q, heads, head_dim] where it lies -> (tensor, its strides)"""
        if t.get_device() != self.index:
            raise ValueError(f"{name} must live on the cache's device")
        if t.dim() != 4 or t.shape[0] != self.B or t.shape[3] != self.head_dim or heads is not None and t.shape[2] != heads:
            raise ValueError(f"expected {name} [{self.B}, Q, {heads or 'heads'}, {self.head_dim}], got {list(t.shape)}")
        if 0 in t.shape:
            raise ValueError(f"{name} must not be empty")
        st = t.stride()
        if st[3] != 1 or min(st) < 0:
            t = t.contiguous()
            st = t.stride()
        return t, st[:3]

    def run(self, fn, *args):
        with torch.cuda.device(self.index):
            _check(fn(*args, _ptr(self.status), rows._raw_stream(self.index)))


def kv_write(cache: KVCache, k: torch.Tensor, v: torch.Tensor, pages: torch.Tensor, start: torch.Tensor,
             counts: Optional[torch.Tensor] = None, *, status: Optional[torch.Tensor] = None, stream=None) -> None:
    """Quantises keys and values [B, Q, heads, head_dim] (float32, bfloat16, float16) into the cache, as tokens ``start[b]`` to
    ``start[b] + Q - 1`` of each sequence, or the first ``counts[b]`` of them (ears_kv_write).  One token or a prompt: Q is any."""
    if stream is not None:
        return _on_stream(stream, cache, kv_write, cache, k, v, pages, start, counts, status=status)
    if _plain().kv_write(cache[0], cache[1], k, v, pages, start, counts, status):
        return
    _refuse_gradients(k, v, *cache)
    c = _Call(cache, pages, start, counts, status)
    code = _DTYPES.get(k.dtype)
    if code is None or v.dtype != k.dtype:
        raise TypeError(f"keys and values must both be float32, bfloat16 or float16, got {k.dtype} and {v.dtype}")
    if k.shape != v.shape:
        raise ValueError("keys and values must have the same shape")
    k, ks = c.heads_of(k, "k", c.heads)
    v, vs = c.heads_of(v, "v", c.heads)
    c.run(load_library().ears_kv_write, code, ctypes.byref(c.cache), k.data_ptr(), v.data_ptr(), c.B, k.shape[1], *ks, *vs, *c.table)


def kv_read(cache: KVCache, pages: torch.Tensor, start: torch.Tensor, tokens: int, counts: Optional[torch.Tensor] = None, *,
            dtype: torch.dtype = torch.bfloat16, status: Optional[torch.Tensor] = None, stream=None):
    """The values of ``tokens`` tokens of each sequence from ``start[b]`` on: (keys, values), each [B, tokens, heads, head_dim] of ``dtype``
    (ears_kv_read).  Positions from ``counts[b]`` on are zeros."""
    if stream is not None:
        return _on_stream(stream, cache, kv_read, cache, pages, start, tokens, counts, dtype=dtype, status=status)
    out = _plain().kv_read(cache[0], cache[1], pages, start, tokens, counts, _DTYPES.get(dtype), status)
    if out is not None:
        return out
    _refuse_gradients(*cache)
    c = _Call(cache, pages, start, counts, status)
    if dtype not in _DTYPES:
        raise TypeError(f"values can be read as float32, bfloat16 or float16, not {dtype}")
    tokens = int(tokens)
    if tokens < 1:
        raise ValueError("at least one token is read")
    k = torch.empty(c.B, tokens, c.heads, c.head_dim, dtype=dtype, device=cache.codes.device)
    v = torch.empty_like(k)
    c.run(load_library().ears_kv_read, _DTYPES[dtype], ctypes.byref(c.cache), c.B, tokens, *c.table, k.data_ptr(), v.data_ptr())
    return k, v


def kv_attention(q: torch.Tensor, cache: KVCache, pages: torch.Tensor, start: torch.Tensor, counts: Optional[torch.Tensor] = None, *,
                 scale: Optional[float] = None, window: int = 0, sinks: int = 0, lse: bool = False,
                 status: Optional[torch.Tensor] = None, stream=None):
    """Attention of the positions ``start[b]`` to ``start[b] + Q - 1``, whose tokens ``kv_write`` has written, over each sequence's
    tokens up to and including their own (ears_kv_attention): with ``window`` > 0 the last ``window`` of them and the first
    ``sinks``.  q [B, Q, heads_q, head_dim] (bfloat16, float16), heads_q a multiple of the cache's heads, consecutive query heads on
    one of them; ``scale`` is 1 / sqrt(head_dim) unless given.  A sequence with a position outside its table is NaN in all its rows
    (``counts`` leaves positions out).  Small calls are faster with a table no wider than they need.  Returns [B, Q, heads_q, head_dim] of q's type, zeros from position
    ``counts[b]`` on; with ``lse=True`` also the scores' log-sum-exp, float32 [B, Q, heads_q]."""
    if stream is not None:
        return _on_stream(stream, cache, kv_attention, q, cache, pages, start, counts, scale=scale, window=window, sinks=sinks, lse=lse, status=status)
    out = _plain().kv_attention(cache[0], cache[1], q, pages, start, counts, scale, window, sinks, bool(lse), status)
    if out is not None:
        return out if lse else out[0]
    _refuse_gradients(q, *cache)
    if scale is None:
        scale = q.shape[-1] ** -0.5 if q.dim() and q.shape[-1] else 1.0
    c = _Call(cache, pages, start, counts, status)
    if q.dtype not in (torch.bfloat16, torch.float16):
        raise TypeError(f"queries must be bfloat16 or float16, got {q.dtype}")
    q, st = c.heads_of(q, "q")
    B, Q, heads = q.shape[:3]
    if heads % c.heads:
        raise ValueError(f"{heads} query heads do not divide among {c.heads} heads of the cache")
    window, sinks = int(window), int(sinks)
    if not 0 <= window < 2**31 or not 0 <= sinks < 2**31:
        raise ValueError("window and sinks must not be negative")
    lib, code, ref = load_library(), _DTYPES[q.dtype], ctypes.byref(c.cache)
    out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    sums = torch.empty(B, Q, heads, dtype=torch.float32, device=q.device) if lse else None
    with torch.cuda.device(c.index):
        need = lib.ears_kv_attention_workspace_bytes(code, ref, B, Q, heads, c.table[1], window, sinks)
    work = torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)
    c.run(lib.ears_kv_attention, code, ref, q.data_ptr(), B, Q, heads, *st, *c.table, float(scale), window, sinks, out.data_ptr(),
          _ptr(sums), work.data_ptr(), work.numel())
    return (out, sums) if lse else out


def _check_start(start, shape, index) -> None:
    """What kv_advance can move in place."""
    if start.dtype not in (torch.int32, torch.int64) or tuple(start.shape) != tuple(shape) or start.get_device() != index:
        raise ValueError("start must be an integer tensor of accept_len's shape and device")
    if any(n > 1 and s == 0 for n, s in zip(start.shape, start.stride())):
        raise ValueError("start must have an element of its own for every sequence")
    if start.is_inference() and not torch.is_inference_mode_enabled():
        raise ValueError("start was made in inference mode and cannot be moved outside of it")


def kv_advance(start: torch.Tensor, accept_len: torch.Tensor, *, stream=None) -> torch.Tensor:
    """``start`` [B], in place, behind the tokens that a verification step keeps: the one before the drafts and ``accept_len`` drafts; the
    token it emits last has not been through the model yet.  An unusable sequence (-1) stays where it is."""
    _check_start(start, accept_len.shape, accept_len.get_device())
    if accept_len.dtype.is_floating_point or accept_len.dtype.is_complex or accept_len.dtype is torch.bool:
        raise TypeError("accept_len must hold integers")
    if stream is None:
        return start.add_(accept_len).add_(1)
    with torch.cuda.stream(stream):
        return start.add_(accept_len).add_(1)
