"""Operators on rows of logits beside the verification step (include/ears.h, "Operators on rows of
logits"): a teacher's top logits, token log probabilities, distillation from top logits and the clipped
policy loss.  Argument marshalling only; every computation runs in the CUDA library.

Logits are CUDA tensors [B, R, V] or [R, V] (float32, bfloat16, float16); rows are used where they
lie as long as the entries of a row are contiguous (a slice ``target[:, :K]`` is not copied).  Per-row tensors
have the logits' shape without V and are converted to contiguous float32 / int32 where they are not (integers that 32 bits
cannot hold stay unusable).
A gradient is allocated contiguous where the logits are not.  With V x element size no multiple of 16 (``logits[:, :-1]`` of a
vocabulary of 50257) its rows then start elsewhere within 16 bytes than the logits' and are stored entry by entry, at a
half to a quarter of the speed; a step is spared that by an ``out_grad`` with the logits' strides.
``*_loss`` and ``token_logprobs`` can be differentiated by autograd, in the logits alone (every other input counts as a
constant; forward mode is refused); ``*_step`` return the gradient at once, reading the logits from memory a single
time, and are what a step recorded into a CUDA graph uses.
Calls whose tensors are in their plain form already go through csrc/ears_torch.cpp, which makes the same C-ABI call
with less work on the host; everything else is converted, checked and refused here.
``status``: optional int32 CUDA tensor of one element that gets EARS_DEV_INVALID_INPUT OR-ed in.
"""
from __future__ import annotations

import ctypes
import functools
import warnings
from typing import NamedTuple, Optional

import torch
from torch.autograd import forward_ad

from . import binding
from . import build as _build
from .binding import _check, load_library

MAX_TOP = 128
DISTILL_KINDS = {"forward_kl": 0, "reverse_kl": 1, "jsd": 2}
_INT32_MAX = 2**31 - 1
_DTYPES = {torch.float32: binding.EARS_DTYPE_F32, torch.bfloat16: binding.EARS_DTYPE_BF16, torch.float16: binding.EARS_DTYPE_F16}


class TopLogits(NamedTuple):
    values: torch.Tensor                 # [..., k] float32, descending; -inf where absent
    ids: torch.Tensor                    # [..., k] int32, -1 where absent
    lse: Optional[torch.Tensor]          # [...] float32 log normaliser at the call's temperature, or None


class PolicyTerms(NamedTuple):
    loss: torch.Tensor
    logp: torch.Tensor
    kl: Optional[torch.Tensor]
    entropy: Optional[torch.Tensor]


_plain = None          # the ears_torch module, bound to the library in use, or _Ctypes
_plain_for = None


class _Ctypes:
    """In the module's place where it cannot be had: no call is in its plain form."""
    top_logits = token_logprobs = token_logprobs_step = policy = distill = staticmethod(lambda *args: None)


def _plain_calls():
    """csrc/ears_torch.cpp, calling the library that load_library() returns."""
    global _plain, _plain_for
    lib = binding._lib
    if lib is not None and lib is _plain_for:
        return _plain
    lib = load_library()
    try:
        _plain = _bind_module(lib)
    except Exception as e:
        warnings.warn(f"ears: the row operators' calls go through ctypes, which takes the host some 10 us more each: {e}", RuntimeWarning)
        _plain = _Ctypes
    _plain_for = lib
    return _plain


def _bind_module(lib):
    _build.build_torch()       # nothing to do when what is there was built from these sources for this torch
    from . import ears_torch
    if ears_torch.version != lib.ears_version():
        raise RuntimeError(f"ears_torch is for version {ears_torch.version} of the library, which has {lib.ears_version()}")
    names = ("ears_top_logits", "ears_token_logprobs", "ears_token_logprobs_step", "ears_policy_loss", "ears_policy_step",
             "ears_distill_loss", "ears_distill_step")
    ears_torch.bind({n: ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in names})
    return ears_torch


def _refuse_tangents(values) -> None:
    # a dual tensor does not say requires_grad: its tangent would be dropped without a word
    for v in values:
        if isinstance(v, (tuple, list)):
            _refuse_tangents(v)
        elif isinstance(v, torch.Tensor) and forward_ad.unpack_dual(v).tangent is not None:
            raise NotImplementedError("the row operators have no forward-mode derivatives")


def _on_stream(fn):
    """``stream=``: the whole call, its conversions and outputs included, belongs to that stream as under torch.cuda.stream."""
    @functools.wraps(fn)
    def call(*args, stream=None, **kwargs):
        if forward_ad._current_level >= 0:
            _refuse_tangents(args)
            _refuse_tangents(kwargs.values())
        if stream is None:
            return fn(*args, **kwargs)
        logits = args[0] if args else kwargs["logits"]
        if stream.device_index != logits.get_device():
            raise ValueError("the stream must belong to the logits' device")
        with torch.cuda.stream(stream):
            return fn(*args, **kwargs)
    return call


def _overwritten(out_grad) -> None:
    """A gradient has been written over a tensor of the caller's (the logits, say): an autograd graph that saved
    it notices in its backward pass."""
    if out_grad is not None:
        torch.autograd.graph.increment_version(out_grad)


def _within_int32(t):
    """Integers beyond 32 bits go to the nearest that 32 bits hold, which is an index of no row either."""
    if t.dtype is torch.uint64:
        t = t.to(torch.int64)
        t = torch.where(t < 0, _INT32_MAX, t)       # 2^63 and more
    elif t.dtype is torch.uint32:
        t = t.to(torch.int64)
    return t.clamp(-_INT32_MAX - 1, _INT32_MAX) if t.dtype is torch.int64 else t


class _Rows:
    """The common head of a call: dtype, pointer, sizes, strides, temperature.  Small calls are bound by the host, so
    nothing is converted, viewed or looked up that is as it should be already."""

    __slots__ = ("logits", "lead", "index", "B", "R", "V", "seq_T", "status", "args")

    def __init__(self, logits: torch.Tensor, temperature, seq_temperature, status):
        code = _DTYPES.get(logits.dtype)
        if code is None:
            raise TypeError(f"logits must be float32, bfloat16 or float16, got {logits.dtype}")
        shape = logits.shape
        dims = len(shape)
        if dims != 3 and dims != 2:
            raise ValueError("expected logits [B,R,V] or [R,V]")
        self.index = index = logits.get_device()
        if index < 0:
            raise ValueError("logits must be a CUDA tensor")
        if 0 in shape:
            raise ValueError("logits must not be empty")
        strides = logits.stride()
        if strides[-1] != 1 and shape[-1] > 1 or min(strides) < 0:
            logits = logits.contiguous()
            strides = logits.stride()
        self.logits, self.lead, self.V = logits, shape[:-1], shape[-1]
        if dims == 3:
            self.B, self.R = shape[0], shape[1]
            sb, sr = strides[0], strides[1]
        else:
            self.B, self.R = 1, shape[0]
            sb, sr = 0, strides[0]
        self.seq_T = None if seq_temperature is None else self.per(seq_temperature, torch.float32, (self.B,), "seq_temperature")
        if status is not None and (status.get_device() != index or status.dtype != torch.int32 or status.numel() != 1):
            raise ValueError("status must be an int32 CUDA tensor of one element on the logits' device")
        self.status = status           # held, not its address: a backward call writes to it again
        self.args = (code, logits.data_ptr(), self.B, self.R, self.V, sb, sr, float(temperature),
                     None if self.seq_T is None else self.seq_T.data_ptr())

    def per(self, t, dtype, shape, name):
        if t is None:
            return None
        if t.get_device() != self.index:
            raise ValueError(f"{name} must live on the logits' device")
        if t.shape != shape:
            raise ValueError(f"{name} must have shape {list(shape)}, got {list(t.shape)}")
        if t.dtype is not dtype:
            if dtype is torch.int32 and (t.dtype.is_floating_point or t.dtype is torch.bool):
                raise TypeError(f"{name} must hold integers")
            t = t.detach()
            if dtype is torch.int32:
                t = _within_int32(t)
            t = t.to(dtype)
        return t if t.is_contiguous() else t.contiguous()

    def row(self, t, name, dtype=torch.float32):
        return None if t is None else self.per(t, dtype, self.lead, name)

    def grad(self, out_grad):
        x = self.logits
        if out_grad is None:
            out_grad = torch.empty_like(x) if x.is_contiguous() else torch.empty(x.shape, dtype=x.dtype, device=x.device)
        elif out_grad.shape != x.shape or out_grad.dtype != x.dtype or out_grad.get_device() != self.index:
            raise ValueError("out_grad must have the logits' shape, type and device")
        elif out_grad.shape[-1] > 1 and out_grad.stride(-1) != 1:
            raise ValueError("the entries of out_grad's rows must be contiguous")
        st = out_grad.stride()
        return out_grad, (out_grad.data_ptr(), st[0] if len(st) == 3 else 0, st[-2])

    def call(self, fn, *tail):
        """fn(*head, *tail, status, stream) with the logits' device current, on its current stream."""
        if _current_device() == self.index:
            rc = fn(*self.args, *tail, _ptr(self.status), _raw_stream(self.index))
        else:
            with torch.cuda.device(self.index):
                rc = fn(*self.args, *tail, _ptr(self.status), _raw_stream(self.index))
        if rc:
            _check(rc)


_current_device = torch._C._cuda_getDevice
_raw_stream = torch._C._cuda_getCurrentRawStream
_F32 = torch.float32


def _ptr(t):
    return None if t is None else t.data_ptr()


def _addresses(ts):
    return tuple(_ptr(t) for t in ts)


def _saved(rows):
    return torch.empty(rows.lead + (4,), dtype=_F32, device=rows.logits.device)


def _keep(ctx, rows, logits, status, saved, *held):
    """What the backward call reads goes through autograd, which notices changes, frees it and may move it meanwhile: the logits
    (or the copy made of them), the temperatures, the statistics, the per-row inputs.  The status word is written to."""
    ctx.temperature, ctx.status = rows.args[7], status
    ctx.save_for_backward(logits if rows.logits.data_ptr() == logits.data_ptr() else rows.logits, rows.seq_T, saved, *held)


def _kept(ctx):
    """-> the rows again, the statistics, the per-row inputs"""
    logits, seq_T, saved, *held = ctx.saved_tensors
    return _Rows(logits, ctx.temperature, seq_T, ctx.status), saved, held


def _refuse_capture():
    # a backward pass recorded into a CUDA graph meets the gradient accumulators of whatever eager graph
    # of the same leaves is alive; the step calls need no autograd graph
    if torch.cuda.is_current_stream_capturing():
        raise RuntimeError("autograd through this operator cannot be recorded into a CUDA graph; record the *_step call")


def _wants_grad(logits) -> bool:
    return logits.requires_grad and torch.is_grad_enabled()


# ---- top logits ------------------------------------------------------------------------------

@_on_stream
def top_logits(logits: torch.Tensor, k: int, temperature: float = 1.0, *, accept_len: Optional[torch.Tensor] = None,
               seq_temperature: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None) -> TopLogits:
    """The k largest logits of every row (1 <= k <= 128), equal values by ascending index, and the row's log
    normaliser at ``temperature`` (ears_top_logits).  Entries of -inf are not listed (id -1, value -inf).
    ``accept_len`` [B] int32, as a verification call returns it: rows behind a sequence's first rejection
    are left out."""
    out = _plain_calls().top_logits(logits, accept_len, k, temperature, seq_temperature, status)
    if out is not None:
        return TopLogits(*out)
    rows = _Rows(logits, temperature, seq_temperature, status)
    acc = rows.per(accept_len, torch.int32, (rows.B,), "accept_len")
    k = int(k)
    if not 1 <= k <= MAX_TOP:
        raise ValueError(f"k must lie in 1..{MAX_TOP}")
    values = torch.empty(rows.lead + (k,), dtype=_F32, device=rows.logits.device)
    ids = torch.empty_like(values, dtype=torch.int32)
    lse = torch.empty(rows.lead, dtype=_F32, device=rows.logits.device)
    rows.call(load_library().ears_top_logits, _ptr(acc), k, values.data_ptr(), ids.data_ptr(), lse.data_ptr())
    return TopLogits(values, ids, lse)


# ---- token log probabilities --------------------------------------------------------------------

def _token_forward(rows, tokens, entropy, saved):
    logp = torch.empty_like(tokens, dtype=_F32)
    H = torch.empty_like(logp) if entropy else None
    rows.call(load_library().ears_token_logprobs, tokens.data_ptr(), logp.data_ptr(), _ptr(H), _ptr(saved))
    return logp, H


class _TokenLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, temperature, seq_temperature, entropy, status):
        _refuse_capture()
        rows = _Rows(logits.detach(), temperature, seq_temperature, status)
        saved, tokens = _saved(rows), rows.row(tokens, "tokens", torch.int32)
        _keep(ctx, rows, logits, status, saved, tokens)
        logp, H = _token_forward(rows, tokens, entropy, saved)
        return (logp, H) if entropy else logp

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_logp, d_entropy=None):
        _refuse_capture()
        rows, saved, (tokens,) = _kept(ctx)
        g, place = rows.grad(None)
        dl = rows.row(d_logp, "d_logp")
        dh = rows.row(d_entropy, "d_entropy")
        rows.call(load_library().ears_token_logprobs_backward, tokens.data_ptr(), saved.data_ptr(), dl.data_ptr(), _ptr(dh), *place)
        return (g,) + (None,) * 5


@_on_stream
def token_logprobs(logits: torch.Tensor, tokens: torch.Tensor, temperature: float = 1.0, *, entropy: bool = False,
                   seq_temperature: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
    """Log probability of ``tokens`` (one per row, int; -1 leaves the row out: 0) at ``temperature``; with
    ``entropy=True`` the pair (logp, entropy in nats).  Differentiable (ears_token_logprobs, _backward)."""
    if _wants_grad(logits):
        return _TokenLogprobs.apply(logits, tokens, temperature, seq_temperature, bool(entropy), status)
    out = _plain_calls().token_logprobs(logits, tokens, bool(entropy), temperature, seq_temperature, status)
    if out is not None:
        return out if entropy else out[0]
    rows = _Rows(logits, temperature, seq_temperature, status)
    logp, H = _token_forward(rows, rows.row(tokens, "tokens", torch.int32), entropy, None)
    return (logp, H) if entropy else logp


@_on_stream
def token_logprobs_step(logits: torch.Tensor, tokens: torch.Tensor, d_logp: torch.Tensor, d_entropy: Optional[torch.Tensor] = None,
                        temperature: float = 1.0, *, out_grad: Optional[torch.Tensor] = None,
                        seq_temperature: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
    """(logp, entropy or None, gradient) for upstream gradients known beforehand (ears_token_logprobs_step):
    ``d_logp`` and, optionally, ``d_entropy`` per row.  ``out_grad=logits`` writes the gradient over them."""
    out = _plain_calls().token_logprobs_step(logits, tokens, d_logp, d_entropy, out_grad, temperature, seq_temperature, status)
    if out is not None:
        _overwritten(out_grad)
        return out
    rows = _Rows(logits, temperature, seq_temperature, status)
    tok, dl, dh = rows.row(tokens, "tokens", torch.int32), rows.row(d_logp, "d_logp"), rows.row(d_entropy, "d_entropy")
    logp = torch.empty_like(dl)
    H = None if dh is None else torch.empty_like(dl)
    g, place = rows.grad(out_grad)
    rows.call(load_library().ears_token_logprobs_step, tok.data_ptr(), dl.data_ptr(), _ptr(dh), logp.data_ptr(), _ptr(H),
              *place)
    _overwritten(out_grad)
    return logp, H, g


# ---- clipped policy loss ---------------------------------------------------------------------------

def _policy_inputs(rows, tokens, old_logp, advantage, ref_logp, clip_low, clip_high, kl_coef, entropy_coef):
    held = (rows.row(tokens, "tokens", torch.int32), rows.row(old_logp, "old_logp"), rows.row(ref_logp, "ref_logp"),
            rows.row(advantage, "advantage"))
    return held, _addresses(held) + (float(clip_low), float(clip_high), float(kl_coef), float(entropy_coef))


def _policy_outputs(rows, held, entropy):
    _, old, ref, _ = held
    new = torch.empty_like
    return PolicyTerms(new(old), new(old), None if ref is None else new(old), new(old) if entropy else None)


class _PolicyLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, old_logp, advantage, ref_logp, temperature, coefs, seq_temperature, entropy, status):
        _refuse_capture()
        rows = _Rows(logits.detach(), temperature, seq_temperature, status)
        held, args = _policy_inputs(rows, tokens, old_logp, advantage, ref_logp, *coefs)
        saved, ctx.coefs = _saved(rows), args[len(held):]
        _keep(ctx, rows, logits, status, saved, *held)
        t = _policy_outputs(rows, held, entropy)
        rows.call(load_library().ears_policy_loss, *args, *_addresses(t), saved.data_ptr())
        ctx.mark_non_differentiable(*(o for o in t[1:] if o is not None))
        return tuple(t)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_loss, *_):
        _refuse_capture()
        rows, saved, held = _kept(ctx)
        g, place = rows.grad(None)
        dl = rows.row(d_loss, "d_loss")
        rows.call(load_library().ears_policy_backward, *_addresses(held), *ctx.coefs, saved.data_ptr(), dl.data_ptr(), *place)
        return (g,) + (None,) * 9


@_on_stream
def policy_loss(logits: torch.Tensor, tokens: torch.Tensor, old_logp: torch.Tensor, advantage: torch.Tensor,
                temperature: float = 1.0, *, ref_logp: Optional[torch.Tensor] = None, clip_low: float = 0.2,
                clip_high: float = 0.2, kl_coef: float = 0.0, entropy_coef: float = 0.0, entropy: bool = False,
                seq_temperature: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None) -> PolicyTerms:
    """Clipped policy loss per row with a KL term and an entropy bonus (ears_policy_loss), differentiable in the
    logits through ``loss``; the other terms (kl with ``ref_logp``, entropy when its coefficient is not 0 or
    ``entropy=True``) come without gradients.  Token -1 leaves a row out."""
    with_entropy = bool(entropy) or entropy_coef != 0.0
    coefs = (clip_low, clip_high, kl_coef, entropy_coef)
    if _wants_grad(logits):
        return PolicyTerms(*_PolicyLoss.apply(logits, tokens, old_logp, advantage, ref_logp, temperature, coefs, seq_temperature,
                                              with_entropy, status))
    out = _plain_calls().policy(logits, tokens, old_logp, ref_logp, advantage, *coefs, with_entropy, False, None, None, temperature,
                                seq_temperature, status)
    if out is not None:
        return PolicyTerms(*out[:4])
    rows = _Rows(logits, temperature, seq_temperature, status)
    held, args = _policy_inputs(rows, tokens, old_logp, advantage, ref_logp, *coefs)
    t = _policy_outputs(rows, held, with_entropy)
    rows.call(load_library().ears_policy_loss, *args, *_addresses(t), None)
    return t


@_on_stream
def policy_step(logits: torch.Tensor, tokens: torch.Tensor, old_logp: torch.Tensor, advantage: torch.Tensor,
                temperature: float = 1.0, *, ref_logp: Optional[torch.Tensor] = None, clip_low: float = 0.2,
                clip_high: float = 0.2, kl_coef: float = 0.0, entropy_coef: float = 0.0, entropy: bool = False,
                row_weight: Optional[torch.Tensor] = None, out_grad: Optional[torch.Tensor] = None,
                seq_temperature: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
    """(PolicyTerms, gradient of sum row_weight * loss) in one call (ears_policy_step)."""
    with_entropy = bool(entropy) or entropy_coef != 0.0
    out = _plain_calls().policy(logits, tokens, old_logp, ref_logp, advantage, clip_low, clip_high, kl_coef, entropy_coef, with_entropy,
                                True, row_weight, out_grad, temperature, seq_temperature, status)
    if out is not None:
        _overwritten(out_grad)
        return PolicyTerms(*out[:4]), out[4]
    rows = _Rows(logits, temperature, seq_temperature, status)
    held, args = _policy_inputs(rows, tokens, old_logp, advantage, ref_logp, clip_low, clip_high, kl_coef, entropy_coef)
    w = rows.row(row_weight, "row_weight")
    t = _policy_outputs(rows, held, with_entropy)
    g, place = rows.grad(out_grad)
    rows.call(load_library().ears_policy_step, *args, _ptr(w), *_addresses(t), *place)
    _overwritten(out_grad)
    return t, g


# ---- distillation from top logits ----------------------------------------------------------------------

def _distill_inputs(rows, teacher, kind, mix):
    if kind not in DISTILL_KINDS:
        raise ValueError(f"kind must be one of {sorted(DISTILL_KINDS)}")
    values, ids, lse = teacher
    k = int(ids.shape[-1]) if ids.dim() else 0
    if not 1 <= k <= MAX_TOP:
        raise ValueError(f"the teacher's lists must have 1..{MAX_TOP} entries")
    held = (rows.per(values, torch.float32, rows.lead + (k,), "teacher values"),
            rows.per(ids, torch.int32, rows.lead + (k,), "teacher ids"), rows.row(lse, "teacher lse"))
    return held, (k,) + _addresses(held) + (DISTILL_KINDS[kind], float(mix))


def _loss_like(rows, t):
    return torch.empty(rows.lead, dtype=_F32, device=rows.logits.device) if t is None else torch.empty_like(t)


class _DistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, teacher, temperature, kind, mix, seq_temperature, status):
        _refuse_capture()
        rows = _Rows(logits.detach(), temperature, seq_temperature, status)
        held, args = _distill_inputs(rows, teacher, kind, mix)
        saved, ctx.kind = _saved(rows), args[1 + len(held):]
        _keep(ctx, rows, logits, status, saved, *held)
        loss = _loss_like(rows, held[2])
        rows.call(load_library().ears_distill_loss, *args, loss.data_ptr(), saved.data_ptr())
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_loss):
        _refuse_capture()
        rows, saved, held = _kept(ctx)
        g, place = rows.grad(None)
        dl = rows.row(d_loss, "d_loss")
        rows.call(load_library().ears_distill_backward, held[1].shape[-1], *_addresses(held), *ctx.kind, saved.data_ptr(), dl.data_ptr(), *place)
        return (g,) + (None,) * 6


@_on_stream
def distill_loss(logits: torch.Tensor, teacher: TopLogits, temperature: float = 1.0, *, kind: str = "forward_kl",
                 mix: float = 0.5, seq_temperature: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Divergence of the draft rows from a teacher's top logits, per row (ears_distill_loss), differentiable in
    the draft's logits.  ``teacher``: what ``top_logits`` returned for the matching rows at the same temperature;
    with ``lse=None`` its entries are renormalised, else the rest of the vocabulary is one more outcome.
    kind: "forward_kl", "reverse_kl" (needs lse) or "jsd" with weight ``mix``.  Rows without entries are left out."""
    if _wants_grad(logits):
        return _DistillLoss.apply(logits, teacher, temperature, kind, mix, seq_temperature, status)
    out = _plain_calls().distill(logits, *teacher, DISTILL_KINDS.get(kind), mix, False, None, None, temperature, seq_temperature, status)
    if out is not None:
        return out[0]
    rows = _Rows(logits, temperature, seq_temperature, status)
    held, args = _distill_inputs(rows, teacher, kind, mix)
    loss = _loss_like(rows, held[2])
    rows.call(load_library().ears_distill_loss, *args, loss.data_ptr(), None)
    return loss


@_on_stream
def distill_step(logits: torch.Tensor, teacher: TopLogits, temperature: float = 1.0, *, kind: str = "forward_kl",
                 mix: float = 0.5, row_weight: Optional[torch.Tensor] = None, out_grad: Optional[torch.Tensor] = None,
                 seq_temperature: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
    """(loss per row, gradient of sum row_weight * loss) in one call (ears_distill_step)."""
    out = _plain_calls().distill(logits, *teacher, DISTILL_KINDS.get(kind), mix, True, row_weight, out_grad, temperature, seq_temperature,
                                 status)
    if out is not None:
        _overwritten(out_grad)
        return out
    rows = _Rows(logits, temperature, seq_temperature, status)
    held, args = _distill_inputs(rows, teacher, kind, mix)
    w = rows.row(row_weight, "row_weight")
    loss = _loss_like(rows, w)
    g, place = rows.grad(out_grad)
    rows.call(load_library().ears_distill_step, *args, _ptr(w), loss.data_ptr(), *place)
    _overwritten(out_grad)
    return loss, g


def set_row_cluster(cluster: int = 0) -> None:
    """CTAs per row of these operators (1, 2, 4, 8, 16; 0 = automatic), for tests and measurements."""
    _check(load_library().ears_set_row_cluster(int(cluster)))
