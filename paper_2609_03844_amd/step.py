"""The operators beside the watermark in a decode or training step (``include/sbw_step.h``).

    head_logits(hidden, codes, scales) -> logits [B, V]      a head with 4-bit weights
    top_candidates(logits, k) -> (ids int32 [B, k], values float32 [B, k])
    token_logprobs(logits, tokens, inv_temperature=1.0, top=0) -> TokenLogprobs
    token_logprobs_grad(logits, tokens, stats, ...) -> the gradient, like logits
    sample_tokens(logits, seeds, inv_temperature=1.0, top_k=0, top_p=1.0, min_p=0.0) -> (tokens, logprobs)

Ordinary calls are marshalled in native code (``_binding.so``), the others here.  Same conventions
as the watermark's calls: tensors on the current HIP device, unit stride
along the vocabulary, rows padded or not, the current stream unless one is given, every step
in the HIP kernels of ``libsbw.so``.  token_logprobs carries a gradient; inputs with a forward-mode
tangent and lazily negated views are refused.

With ``stream`` the work is on that stream: what the caller passes must be ready there, and stay unchanged and
alive until it has been read (``Tensor.record_stream``); what the call allocates does by itself, and its outputs are
ready when that stream is.
"""
from __future__ import annotations

import ctypes
import functools
from typing import NamedTuple, Optional

import torch
from torch.autograd.forward_ad import unpack_dual
from torch.autograd.function import once_differentiable

from . import BF16, F32, _check, _empty, _native, _on_device, _side, _stream, raw

MAX_STEP_TOKENS = 1024   # SBW_STEP_MAX_TOKENS
HEAD_GROUPS = (32, 64, 128)
MAX_HIDDEN = 8192

#: C entry points of include/sbw_step.h.
EXPORTED_STEP = ("sbw_token_logprobs", "sbw_token_logprobs_workspace", "sbw_token_logprobs_grad",
                 "sbw_top_candidates", "sbw_top_candidates_workspace", "sbw_head_logits",
                 "sbw_quantize_fp8", "sbw_matmul_fp8", "sbw_matmul_fp8_workspace",
                 "sbw_sample_tokens", "sbw_sample_tokens_workspace")


def _declare(lib: ctypes.CDLL) -> ctypes.CDLL:
    P, i64, f32, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_float, ctypes.c_int
    lib.sbw_token_logprobs.restype = i32
    lib.sbw_token_logprobs.argtypes = [P, i32, i64, i64, i64, P, i64, f32, i64, P, P, P, P, P, P, P, P]
    lib.sbw_token_logprobs_workspace.restype = i64
    lib.sbw_token_logprobs_workspace.argtypes = [i64, i64, i64]
    lib.sbw_token_logprobs_grad.restype = i32
    lib.sbw_token_logprobs_grad.argtypes = [P, i32, i64, i64, i64, P, i64, P, P, P, P, P, f32, P, i64, P]
    lib.sbw_top_candidates.restype = i32
    lib.sbw_top_candidates.argtypes = [P, i32, i64, i64, i64, i64, i64, P, P, P, P]
    lib.sbw_top_candidates_workspace.restype = i64
    lib.sbw_top_candidates_workspace.argtypes = [i64, i64, i64]
    lib.sbw_sample_tokens.restype = i32
    lib.sbw_sample_tokens.argtypes = [P, i32, i64, i64, i64, P, P, f32, P, i64, P, f32, P, f32, P, P, P, P]
    lib.sbw_sample_tokens_workspace.restype = i64
    lib.sbw_sample_tokens_workspace.argtypes = [i64, i64]
    lib.sbw_head_logits.restype = i32
    lib.sbw_head_logits.argtypes = [P, i64, i64, i64, P, P, i32, i64, i64, P, i32, i64, P]
    return lib


_lib = _declare(raw())


class TokenLogprobs(NamedTuple):
    """What token_logprobs() returns; fields that were not asked for are None."""
    logprobs: Optional[torch.Tensor]      # float32, shaped as tokens
    lse: torch.Tensor                     # float32 [B]
    entropy: torch.Tensor                 # float32 [B], in nats
    stats: torch.Tensor                   # float32 [B, 2], what token_logprobs_grad needs
    top_ids: Optional[torch.Tensor]       # int32 [B, top]
    top_logprobs: Optional[torch.Tensor]  # float32 [B, top]


def _dtype(t: torch.Tensor, name: str) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"{name} must be float32 or bfloat16")


def _plain(t: torch.Tensor, name: str) -> None:
    """Refuses what a tensor's memory does not show."""
    if t.is_neg():
        raise ValueError(f"{name} is a lazily negated view: give {name}.resolve_neg()")
    if unpack_dual(t).tangent is not None:
        raise ValueError(f"{name} has a forward-mode tangent, which these operators do not carry")


def _matrix(t: torch.Tensor, name: str):
    """(dtype, rows, columns, row stride) of a matrix with unit stride along its rows."""
    _plain(t, name)
    if t.dim() != 2:
        raise ValueError(f"{name} must be two-dimensional")
    dtype = _dtype(t, name)
    B, V = t.shape
    if B > 0 and V > 1 and t.stride(1) != 1:
        raise ValueError(f"{name} must have unit stride along its rows")
    if B > 1 and t.stride(0) < V:
        raise ValueError(f"the rows of {name} must not overlap")
    return dtype, B, V, t.stride(0) if B > 1 else max(V, t.stride(0))


def _tokens(tokens: Optional[torch.Tensor], B: int) -> int:
    """Tokens per row of int32 [B] or [B, n]."""
    if tokens is None:
        return 0
    if tokens.dtype != torch.int32 or tokens.dim() not in (1, 2) or tokens.shape[0] != B:
        raise ValueError("tokens must be int32 [B] or [B, n]")
    if not tokens.is_contiguous():
        raise ValueError("tokens must be contiguous")
    return 1 if tokens.dim() == 1 else tokens.shape[1]


def _vector(t: Optional[torch.Tensor], shape, dtype, name: str) -> Optional[int]:
    """The address of a contiguous tensor of this shape and type (None for None)."""
    if t is None:
        return None
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous {dtype} {list(shape)}")
    _plain(t, name)
    return t.data_ptr()


def _no_gradient(what: str, **tensors) -> None:
    """Refuses inputs whose gradient a call would drop."""
    if torch.is_grad_enabled():
        for name, t in tensors.items():
            if t.requires_grad:
                raise ValueError(f"{what} carry no gradient to {name}: give {name}.detach(), or call under "
                                 "torch.no_grad()")


def _scratch(workspace: Optional[torch.Tensor], need: int, device, side) -> torch.Tensor:
    if workspace is None:
        return _empty(max(need, 1), torch.int64, device, side, kept=False)
    if workspace.dtype != torch.int64 or not workspace.is_contiguous() or workspace.numel() < need:
        raise ValueError(f"workspace must be contiguous int64 with >= {need} elements")
    return workspace


@functools.lru_cache(maxsize=1024)
def token_logprobs_workspace_size(B: int, V: int, top: int = 0) -> int:
    """int64 elements of scratch that token_logprobs needs."""
    return int(_lib.sbw_token_logprobs_workspace(int(B), int(V), int(top)))


@functools.lru_cache(maxsize=1024)
def top_candidates_workspace_size(B: int, V: int, k: int) -> int:
    """int64 elements of scratch that top_candidates needs."""
    return int(_lib.sbw_top_candidates_workspace(int(B), int(V), int(k)))


def _forward(logits, tokens, inv_temperature, top, out, workspace, stream) -> TokenLogprobs:
    dtype, B, V, row_stride = _matrix(logits, "logits")
    n = _tokens(tokens, B)
    top = int(top)
    dev = logits.device
    side = _side(stream, dev)
    if out is None:
        f32 = functools.partial(_empty, dtype=torch.float32, device=dev, side=side)
        k = max(top, 0)
        out = TokenLogprobs(f32(tokens.shape) if tokens is not None else None, f32(B), f32(B), f32((B, 2)),
                            _empty((B, k), torch.int32, dev, side) if top else None,
                            f32((B, k)) if top else None)
    if (tokens is not None) != (out.logprobs is not None) or (top > 0 and out.top_ids is None):
        raise ValueError("out must hold what the call writes")
    workspace = _scratch(workspace, token_logprobs_workspace_size(B, V, top), dev, side)
    pointers = [_vector(out.logprobs, tokens.shape if tokens is not None else (), torch.float32, "logprobs"),
                _vector(out.lse, (B,), torch.float32, "lse"),
                _vector(out.entropy, (B,), torch.float32, "entropy"),
                _vector(out.stats, (B, 2), torch.float32, "stats"),
                _vector(out.top_ids, (B, max(top, 0)), torch.int32, "top_ids"),
                _vector(out.top_logprobs, (B, max(top, 0)), torch.float32, "top_logprobs")]
    _on_device(logits=logits, tokens=tokens, workspace=workspace, **out._asdict())
    _check(_lib.sbw_token_logprobs(logits.data_ptr(), dtype, B, V, row_stride,
                                   tokens.data_ptr() if tokens is not None else None, n,
                                   float(inv_temperature), top, *pointers, workspace.data_ptr(),
                                   _stream(stream)))
    return out


class _Differentiable(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, inv_temperature, top, workspace, stream):
        out = _call(logits.detach(), tokens, inv_temperature, top, None, workspace, stream)
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(logits, tokens, out.stats, out.entropy)
        ctx.inv_temperature = inv_temperature
        side = _side(stream, logits.device)
        ctx.done = side.record_event() if side is not None else None
        ctx.mark_non_differentiable(*(t for t in out[3:] if t is not None))   # stats and alternatives
        return tuple(out)

    @staticmethod
    @once_differentiable
    def backward(ctx, g_logprobs, g_lse, g_entropy, *_):
        logits, tokens, stats, entropy = ctx.saved_tensors
        if g_logprobs is None and g_lse is None and g_entropy is None:
            return (None,) * 6
        g = [t.resolve_neg().contiguous() if t is not None else None for t in (g_logprobs, g_lse, g_entropy)]
        # on autograd's stream, whatever the forward call's: it has waited for these gradients, and waits for the
        # statistics here, as gradients need not come from reading the outputs
        if ctx.done is not None:
            torch.cuda.current_stream().wait_event(ctx.done)
        grad = token_logprobs_grad(logits.detach(), tokens, stats, entropy, *g, ctx.inv_temperature)
        return grad, None, None, None, None, None


def _call(logits, tokens, inv_temperature, top, out, workspace, stream) -> TokenLogprobs:
    if stream is None and out is None and workspace is None:
        got = _native.token_logprobs(logits, tokens, inv_temperature, top)
        if type(got) is tuple:
            return tuple.__new__(TokenLogprobs, got)
        if got is not None:
            _check(got)
    return _forward(logits, tokens, inv_temperature, top, out, workspace, stream)


def token_logprobs(logits: torch.Tensor, tokens: Optional[torch.Tensor],
                   inv_temperature: float = 1.0, top: int = 0,
                   out: Optional[TokenLogprobs] = None, workspace: Optional[torch.Tensor] = None,
                   stream=None) -> TokenLogprobs:
    """Log probabilities of given tokens under softmax(logits * inv_temperature), with the log
    sum, the entropy and the ``top`` most likely alternatives of every row, in one pass.

    logits: [B, V] float32 or bfloat16, for instance as ``watermark()`` left them.  tokens:
    int32 [B] or [B, n], n <= 1024, or None for none; an id outside [0, V) is padding, with
    log probability 0.  top <= 1024; alternatives stand in order, equal ones by their id, places
    beyond V hold -1 and -inf.  ``workspace`` is an int64 scratch tensor of at least
    token_logprobs_workspace_size(B, V, top) elements and ``out`` the tensors to write (both
    allocated here when not given).

    Outputs that are allocated here may share one storage with each other and with a small workspace: clone() what
    is kept for long or saved to a file.

    With logits that require a gradient, logprobs, lse and entropy carry one (through
    ``token_logprobs_grad``; ``out`` must not be given).  The logits must then keep their
    values until the backward pass: the in-place ``watermark`` does not tell torch of its writes.
    """
    if torch.is_grad_enabled() and logits.requires_grad:
        if out is not None:
            raise ValueError("out cannot be given where the logits require a gradient")
        return TokenLogprobs(*_Differentiable.apply(logits, tokens, inv_temperature, top, workspace,
                                                    stream))
    return _call(logits, tokens, inv_temperature, top, out, workspace, stream)


def token_logprobs_grad(logits: torch.Tensor, tokens: Optional[torch.Tensor], stats: torch.Tensor,
                        entropy: Optional[torch.Tensor] = None,
                        grad_logprobs: Optional[torch.Tensor] = None,
                        grad_lse: Optional[torch.Tensor] = None,
                        grad_entropy: Optional[torch.Tensor] = None,
                        inv_temperature: float = 1.0, out: Optional[torch.Tensor] = None,
                        stream=None) -> torch.Tensor:
    """The gradient with respect to the logits, given that of token_logprobs()'s outputs: each
    grad_* is float32, shaped as its output, or None.  stats and entropy are what the forward call
    returned (entropy is needed with grad_entropy only).  ``out`` is like logits; it may be the
    logits themselves.  The result carries no gradient of its own."""
    if stream is None and out is None:
        got = _native.token_logprobs_grad(logits, tokens, stats, entropy, grad_logprobs, grad_lse,
                                          grad_entropy, inv_temperature)
        if type(got) is torch.Tensor:
            return got
        if got is not None:
            _check(got)
    dtype, B, V, row_stride = _matrix(logits, "logits")
    n = _tokens(tokens, B)
    if out is None:
        out = _empty((B, V), logits.dtype, logits.device, _side(stream, logits.device))
    out_dtype, *out_shape, out_stride = _matrix(out, "out")
    if out_dtype != dtype or out_shape != [B, V]:
        raise ValueError("out must be like logits")
    if grad_logprobs is not None and tokens is None:
        raise ValueError("grad_logprobs needs the tokens")
    if grad_entropy is not None and entropy is None:
        raise ValueError("grad_entropy needs the entropy")
    if stats is None:
        raise ValueError("stats is needed")
    pointers = [_vector(stats, (B, 2), torch.float32, "stats"),
                _vector(entropy, (B,), torch.float32, "entropy"),
                _vector(grad_logprobs, tokens.shape if tokens is not None else (), torch.float32,
                        "grad_logprobs"),
                _vector(grad_lse, (B,), torch.float32, "grad_lse"),
                _vector(grad_entropy, (B,), torch.float32, "grad_entropy")]
    _on_device(logits=logits, tokens=tokens, stats=stats, entropy=entropy, grad_logprobs=grad_logprobs,
               grad_lse=grad_lse, grad_entropy=grad_entropy, out=out)
    _check(_lib.sbw_token_logprobs_grad(logits.data_ptr(), dtype, B, V, row_stride,
                                        tokens.data_ptr() if tokens is not None else None, n,
                                        *pointers, float(inv_temperature), out.data_ptr(),
                                        out_stride, _stream(stream)))
    return out


def top_candidates(logits: torch.Tensor, k: int, v_offset: int = 0,
                   ids: Optional[torch.Tensor] = None, values: Optional[torch.Tensor] = None,
                   workspace: Optional[torch.Tensor] = None, with_values: bool = True, stream=None):
    """The k <= 1024 largest logits of every row: (ids int32 [B, k], values float32 [B, k] or
    None), larger first, equal ones by their id, a NaN above every number.  Places beyond V hold
    -1 and -inf.  The ids are what ``watermark_candidates`` takes.  Both may share one storage, as token_logprobs()'s
    outputs do.  v_offset: the token id of
    column 0 when the logits are a vocabulary shard.  The values carry no gradient: logits that require
    one are refused unless it is off (torch.no_grad()) or the ids alone are asked for."""
    if stream is None and ids is None and values is None and workspace is None and with_values:
        got = _native.top_candidates(logits, k, v_offset)
        if type(got) is tuple:
            return got
        if got is not None:
            _check(got)
    if with_values or values is not None:
        _no_gradient("the values of top_candidates", logits=logits)
    dtype, B, V, row_stride = _matrix(logits, "logits")
    k = int(k)
    dev = logits.device
    side = _side(stream, dev)
    if ids is None:
        ids = _empty((B, max(k, 0)), torch.int32, dev, side)
    if values is None and with_values:
        values = _empty((B, max(k, 0)), torch.float32, dev, side)
    workspace = _scratch(workspace, top_candidates_workspace_size(B, V, k), dev, side)
    if k > 0:
        _vector(ids, (B, k), torch.int32, "ids")
        _vector(values, (B, k), torch.float32, "values")
    _on_device(logits=logits, ids=ids, values=values, workspace=workspace)
    _check(_lib.sbw_top_candidates(logits.data_ptr(), dtype, B, V, row_stride, int(v_offset), k,
                                   ids.data_ptr(), values.data_ptr() if values is not None else None,
                                   workspace.data_ptr(), _stream(stream)))
    return ids, values


def head_logits(hidden: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor,
                dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None,
                stream=None) -> torch.Tensor:
    """Logits [B, V] of hidden states by a head with 4-bit weights: weight (v, c) is
    (q - 8) * scales[v, c // group] with q the low half of codes[v, c // 2] for even c, the high
    half for odd c.

    hidden: bfloat16 [B, K], unit stride along K, K <= 8192.  codes: uint8 [V, K / 2] and scales:
    float32 or bfloat16 [V, K / group], contiguous; group is 32, 64 or 128.  V may be a shard
    of the vocabulary.  dtype (of the logits): float32 or bfloat16.  The logits carry no gradient: hidden
    states or scales that require one are refused unless it is off (torch.no_grad()).
    """
    if stream is None and out is None and (dtype is torch.float32 or dtype is torch.bfloat16):
        got = _native.head_logits(hidden, codes, scales, dtype is torch.bfloat16)
        if type(got) is torch.Tensor:
            return got
        if got is not None:
            _check(got)
    _no_gradient("the logits of head_logits", hidden=hidden, scales=scales)
    if hidden.dim() != 2 or hidden.dtype != torch.bfloat16:
        raise ValueError("hidden must be bfloat16 [B, K]")
    _, B, K, hidden_stride = _matrix(hidden, "hidden")
    if codes.dim() != 2 or codes.dtype != torch.uint8 or not codes.is_contiguous() or 2 * codes.shape[1] != K:
        raise ValueError("codes must be contiguous uint8 [V, K / 2]")
    V = codes.shape[0]
    scale_dtype = _dtype(scales, "scales")
    _plain(scales, "scales")
    if scales.dim() != 2 or scales.shape[0] != V or not scales.is_contiguous():
        raise ValueError("scales must be contiguous [V, K / group]")
    groups = scales.shape[1]
    if groups == 0 or K % groups != 0:
        raise ValueError("K must be a multiple of the groups")
    if out is None:
        out = _empty((B, V), dtype, hidden.device, _side(stream, hidden.device))
    out_dtype, *out_shape, row_stride = _matrix(out, "out")
    if out_shape != [B, V] or out.dtype != dtype:
        raise ValueError("out must be [B, V] of dtype")
    _on_device(hidden=hidden, codes=codes, scales=scales, out=out)
    _check(_lib.sbw_head_logits(hidden.data_ptr(), B, K, hidden_stride, codes.data_ptr(),
                                scales.data_ptr(), scale_dtype, K // groups, V, out.data_ptr(),
                                out_dtype, row_stride, _stream(stream)))
    return out


@functools.lru_cache(maxsize=1024)
def sample_tokens_workspace_size(B: int, V: int) -> int:
    """int64 elements of scratch that sample_tokens needs."""
    return int(_lib.sbw_sample_tokens_workspace(int(B), int(V)))


def _of_rows(value, B: int, dtype, name: str):
    """(address of a parameter of every row or None, the one of all rows)."""
    if not isinstance(value, torch.Tensor):
        return None, value
    return _vector(value, (B,), dtype, name), 0


def sample_tokens(logits: torch.Tensor, seeds: torch.Tensor, inv_temperature=1.0, top_k=0, top_p=1.0, min_p=0.0,
                  tokens: Optional[torch.Tensor] = None, logprobs: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None, with_logprobs: bool = True, stream=None):
    """One token of every row, drawn from what the filters keep of softmax(logits * inv_temperature): (tokens int32 [B],
    their log probabilities among the kept, float32 [B], or None).

    In the order of logits (larger first, equal ones by their id) top_k keeps the first k, top_p of those the ones before
    which less than top_p of their probability lies (the first at least), min_p of those the ones with at least min_p times
    the largest probability.  0, 1 and 0 keep all, a top_p of 0 and less the first alone.  Each parameter is a number, or a
    tensor with one for every row: float32 [B], top_k int32 [B].

    logits: [B, V] float32 or bfloat16, for instance as ``watermark()`` left them.  seeds: int64 [B], random; the noise is
    that of ``watermark_sample``, and without filters so is the token (with gamma 0).  A row with a NaN or +inf gives the
    first column of its order with NaN, one of -inf alone column 0 with -inf, and a row whose inv_temperature in a tensor
    is not finite and positive -1 with NaN.  ``workspace`` is an int64 scratch tensor of at least
    sample_tokens_workspace_size(B, V) elements; what is allocated here may share one storage with it.  The log
    probabilities carry no gradient (token_logprobs' do): logits or inv_temperature that require one are refused unless it is
    off (torch.no_grad()) or the tokens alone are asked for."""
    if stream is None and tokens is None and logprobs is None and workspace is None and with_logprobs:
        got = _native.sample_tokens(logits, seeds, inv_temperature, top_k, top_p, min_p)
        if type(got) is tuple:
            return got
        if got is not None:
            _check(got)
    if with_logprobs or logprobs is not None:
        of_temperature = {"inv_temperature": inv_temperature} if isinstance(inv_temperature, torch.Tensor) else {}
        _no_gradient("the log probabilities of sample_tokens", logits=logits, **of_temperature)
    dtype, B, V, row_stride = _matrix(logits, "logits")
    dev = logits.device
    side = _side(stream, dev)
    if seeds.dtype != torch.int64 or tuple(seeds.shape) != (B,) or not seeds.is_contiguous():
        raise ValueError("seeds must be contiguous int64 [B]")
    inv_ts, inv_t = _of_rows(inv_temperature, B, torch.float32, "inv_temperature")
    top_ks, k = _of_rows(top_k, B, torch.int32, "top_k")
    top_ps, p = _of_rows(top_p, B, torch.float32, "top_p")
    min_ps, least = _of_rows(min_p, B, torch.float32, "min_p")
    if tokens is None:
        tokens = _empty(B, torch.int32, dev, side)
    if logprobs is None and with_logprobs:
        logprobs = _empty(B, torch.float32, dev, side)
    _vector(tokens, (B,), torch.int32, "tokens")
    _vector(logprobs, (B,), torch.float32, "logprobs")
    workspace = _scratch(workspace, sample_tokens_workspace_size(B, V), dev, side)
    given = {name: t for name, t in (("inv_temperature", inv_temperature), ("top_k", top_k), ("top_p", top_p),
                                     ("min_p", min_p)) if isinstance(t, torch.Tensor)}
    _on_device(logits=logits, seeds=seeds, tokens=tokens, logprobs=logprobs, workspace=workspace, **given)
    _check(_lib.sbw_sample_tokens(logits.data_ptr(), dtype, B, V, row_stride, seeds.data_ptr(), inv_ts, float(inv_t), top_ks,
                                  int(k), top_ps, float(p), min_ps, float(least), tokens.data_ptr(),
                                  logprobs.data_ptr() if logprobs is not None else None, workspace.data_ptr(),
                                  _stream(stream)))
    return tokens, logprobs
