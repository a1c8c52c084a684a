"""Matrices in 8-bit floating point with a scale for each block of 128, and their products
(``include/sbw_step.h``): what a head or another layer in front of the logits is made of.

    quantize_fp8(x) -> (codes, scales)
    matmul_fp8(a, a_scales, b, b_scales) -> a b^T
    linear_fp8(x, weight) -> x weight^T by such products, with both gradients

Codes are torch.float8_e4m3fn.  Scales are torch.float8_e8m0fnu (powers of two, which the matrix instructions
apply themselves) or float32, one for each 128 columns of a row, or of 128 rows.  Same conventions as the operators
of ``step.py``.
"""
from __future__ import annotations

import ctypes
import functools
from typing import Optional

import torch
from torch.autograd.function import once_differentiable

from . import _check, _empty, _native, _on_device, _side, _stream, raw  # noqa: F401
from .step import _dtype, _matrix, _no_gradient, _plain, _scratch

BLOCK = 128
SCALE_E8M0, SCALE_F32 = 0, 1
_SCALE_TYPES = {torch.float8_e8m0fnu: SCALE_E8M0, torch.float32: SCALE_F32}


def _declare(lib: ctypes.CDLL) -> ctypes.CDLL:
    P, i64, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int
    lib.sbw_quantize_fp8.restype = i32
    lib.sbw_quantize_fp8.argtypes = [P, i32, i64, i64, i64, i64, i32, P, i64, P, P, i64, P, P]
    lib.sbw_matmul_fp8_workspace.restype = i64
    lib.sbw_matmul_fp8_workspace.argtypes = [i64, i64, i64]
    lib.sbw_matmul_fp8.restype = i32
    lib.sbw_matmul_fp8.argtypes = [P, i64, i64, P, i64, P, i64, i64, P, i64, i64, i32, P, i32, i64, P, P]
    return lib


_lib = _declare(raw())


def _blocks(n: int, block: int = BLOCK) -> int:
    return -(-n // block)


def _scale_type(dtype) -> int:
    if dtype not in _SCALE_TYPES:
        raise TypeError("scales must be float8_e8m0fnu or float32")
    return _SCALE_TYPES[dtype]


def _codes(t: torch.Tensor, name: str):
    """(rows, columns, row stride) of a matrix of codes."""
    if t.dtype != torch.float8_e4m3fn or t.dim() != 2:
        raise ValueError(f"{name} must be two-dimensional float8_e4m3fn")
    _plain(t, name)
    rows, columns = t.shape
    if rows > 0 and columns > 1 and t.stride(1) != 1:
        raise ValueError(f"{name} must have unit stride along its rows")
    if rows > 1 and t.stride(0) < columns:
        raise ValueError(f"the rows of {name} must not overlap")
    return rows, columns, t.stride(0) if rows > 1 else max(columns, t.stride(0))


def _new_codes(rows: int, columns: int, device, side) -> torch.Tensor:
    """Rows start at whole lines of 128 bytes, so that a product can fetch them in parts of 16."""
    return _empty((rows, _blocks(columns) * BLOCK), torch.float8_e4m3fn, device, side)[:, :columns]


def _quantized(x, block_rows, scale_dtype, straight, transposed, stream=None):
    """Both orientations, each a pair (codes, scales) to write, True for a new one, or None."""
    if stream is None and scale_dtype in _SCALE_TYPES and (straight is None or straight is True) and \
            (transposed is None or transposed is True):
        got = _native.quantize_fp8(x, block_rows, straight is True, transposed is True, scale_dtype is torch.float8_e8m0fnu)
        if type(got) is tuple:
            return [got[:2] if straight else None, got[2:] if transposed else None]
        if got is not None:
            _check(got)
    dtype, M, K, row_stride = _matrix(x, "x")
    kind = _scale_type(scale_dtype)
    block_rows = int(block_rows)
    if block_rows not in (1, BLOCK):
        raise ValueError("block_rows must be 1 or 128")
    side = _side(stream, x.device)
    pairs, arguments = [], []
    for which, rows, columns in ((straight, M, K), (transposed, K, M)):
        shape = (_blocks(rows, block_rows), _blocks(columns))
        if which is None:
            pairs.append(None)
            arguments += [None, 0, None]
            continue
        codes, scales = which if which is not True else (None, None)
        if codes is None:
            codes = _new_codes(rows, columns, x.device, side)
        if scales is None:
            scales = _empty(shape, scale_dtype, x.device, side)
        *codes_shape, stride = _codes(codes, "codes")
        if codes_shape != [rows, columns]:
            raise ValueError(f"codes must be {[rows, columns]}")
        if tuple(scales.shape) != shape or scales.dtype != scale_dtype or not scales.is_contiguous():
            raise ValueError(f"scales must be contiguous {scale_dtype} {list(shape)}")
        _on_device(x=x, codes=codes, scales=scales)
        pairs.append((codes, scales))
        arguments += [codes.data_ptr(), stride, scales.data_ptr()]
    if M > 0 and K > 0:
        _check(_lib.sbw_quantize_fp8(x.data_ptr(), dtype, M, K, row_stride, block_rows, kind, *arguments, _stream(stream)))
    return pairs


def quantize_fp8(x: torch.Tensor, block_rows: int = 1, transposed: bool = False,
                 scale_dtype: torch.dtype = torch.float8_e8m0fnu, codes: Optional[torch.Tensor] = None,
                 scales: Optional[torch.Tensor] = None, stream=None):
    """(codes, scales) of x, float32 or bfloat16 [M, K] with unit stride along its rows, or with ``transposed`` of its
    transpose: codes float8_e4m3fn [M, K], scales [ceil(M / block_rows), ceil(K / 128)], block_rows 1 or 128.

    A block's largest finite magnitude a gives its scale: the smallest power of two that leaves a / scale at 448 or below
    (float8_e8m0fnu), or a / 448 itself (float32).  Codes are rounded to the nearest, ties to even; infinities and
    NaN become NaN.  Codes that are allocated here have rows padded to whole blocks (a view).  They carry no gradient:
    an x that requires one is refused unless it is off (torch.no_grad())."""
    _no_gradient("the codes of quantize_fp8", x=x)
    given = (codes, scales) if codes is not None or scales is not None else True
    straight, turned = _quantized(x, block_rows, scale_dtype, None if transposed else given, given if transposed else None,
                                  stream)
    return turned if transposed else straight


@functools.lru_cache(maxsize=1024)
def matmul_fp8_workspace_size(M: int, N: int, K: int) -> int:
    """int64 elements of scratch that matmul_fp8 needs."""
    return int(_lib.sbw_matmul_fp8_workspace(int(M), int(N), int(K)))


def _block_rows(scales: torch.Tensor, rows: int, columns: int, name: str) -> int:
    _plain(scales, name)
    if scales.dim() == 2 and scales.is_contiguous() and scales.shape[1] == _blocks(columns):
        if scales.shape[0] == rows:
            return 1
        if scales.shape[0] == _blocks(rows):
            return BLOCK
    raise ValueError(f"{name} must be contiguous, [rows, ceil(K / 128)] or [ceil(rows / 128), ceil(K / 128)]")


def matmul_fp8(a: torch.Tensor, a_scales: torch.Tensor, b: torch.Tensor, b_scales: torch.Tensor,
               dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None,
               workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """a b^T [M, N] of codes a [M, K] and b [N, K] with scales of one type, as quantize_fp8() gives them: for each
    128 columns of a row, or of 128 rows, by their shape.  K >= 1.  Rows of codes have unit stride and may be padded; those
    that start at multiples of 16 bytes are fetched faster.

    dtype (of the product): float32 or bfloat16, rounded once from sums in float32.  A float32 product is of exact terms; for a
    bfloat16 one each term may be cut off 13 bits below the power of two of the largest of its eight neighbours on its way into the
    sum.  The product of two blocks' scales is to lie in float32's range, outside of which results are 0, infinite or NaN where
    the sums need not be.  The product carries no gradient (linear_fp8() does): scales that require one are refused unless it is
    off.  ``workspace`` is an int64 scratch tensor of at least matmul_fp8_workspace_size(M, N, K) elements (allocated here when not
    given)."""
    if stream is None and out is None and workspace is None and (dtype is torch.float32 or dtype is torch.bfloat16):
        got = _native.matmul_fp8(a, a_scales, b, b_scales, dtype is torch.bfloat16)
        if type(got) is torch.Tensor:
            return got
        if got is not None:
            _check(got)
    _no_gradient("the products of matmul_fp8", a=a, a_scales=a_scales, b=b, b_scales=b_scales)
    M, K, a_stride = _codes(a, "a")
    N, b_columns, b_stride = _codes(b, "b")
    if b_columns != K:
        raise ValueError("a and b must have the same columns")
    kind = _scale_type(a_scales.dtype)
    if b_scales.dtype != a_scales.dtype:
        raise TypeError("a_scales and b_scales must be of one type")
    a_rows, b_rows = _block_rows(a_scales, M, K, "a_scales"), _block_rows(b_scales, N, K, "b_scales")
    side = _side(stream, a.device)
    if out is None:
        out = _empty((M, N), dtype, a.device, side)
    out_dtype, *out_shape, out_stride = _matrix(out, "out")
    if out_shape != [M, N] or out.dtype != dtype:
        raise ValueError("out must be [M, N] of dtype")
    need = matmul_fp8_workspace_size(M, N, K)
    if need > 0 or workspace is not None:
        workspace = _scratch(workspace, need, a.device, side)
    _on_device(a=a, a_scales=a_scales, b=b, b_scales=b_scales, out=out, workspace=workspace)
    _check(_lib.sbw_matmul_fp8(a.data_ptr(), M, a_stride, a_scales.data_ptr(), a_rows, b.data_ptr(), N, b_stride,
                               b_scales.data_ptr(), b_rows, K, kind, out.data_ptr(), out_dtype, out_stride,
                               workspace.data_ptr() if workspace is not None else None, _stream(stream)))
    return out


class _Linear(torch.autograd.Function):
    """Both sides are quantised once, in the orientations that this pass and the backward one need."""

    @staticmethod
    def forward(ctx, x, weight, dtype):
        x, weight = x.detach(), weight.detach()
        of_x, of_weight = ctx.needs_input_grad[:2]
        x8, x8_t = _quantized(x, 1, torch.float8_e8m0fnu, True, True if of_weight else None)
        w8, w8_t = _quantized(weight, BLOCK, torch.float8_e8m0fnu, True, True if of_x else None)
        ctx.save_for_backward(*(w8_t or (None, None)), *(x8_t or (None, None)))
        ctx.types = x.dtype, weight.dtype
        return matmul_fp8(*x8, *w8, dtype=dtype)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        w_codes, w_scales, x_codes, x_scales = ctx.saved_tensors
        dy = dy.resolve_neg()
        if dy.stride(-1) != 1 or (dy.shape[0] > 1 and dy.stride(0) < dy.shape[1]):
            dy = dy.contiguous()                       # of a sum, say: one value seen everywhere
        dy8, dy8_t = _quantized(dy, 1, torch.float8_e8m0fnu, True if w_codes is not None else None,
                                True if x_codes is not None else None)
        dx = dw = None
        if dy8 is not None:
            dx = _product_or_zero(dy8, (w_codes, w_scales), ctx.types[0])
        if dy8_t is not None:
            dw = _product_or_zero(dy8_t, (x_codes, x_scales), ctx.types[1])
        return dx, dw, None


def _product_or_zero(a, b, dtype) -> torch.Tensor:
    if a[0].shape[1] == 0:                             # a sum over nothing
        return torch.zeros((a[0].shape[0], b[0].shape[0]), dtype=dtype, device=a[0].device)
    return matmul_fp8(*a, *b, dtype=dtype)


def linear_fp8(x: torch.Tensor, weight: torch.Tensor, dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """x weight^T [M, N] of x [M, K] and weight [N, K], float32 or bfloat16 each, by products in 8 bits: a head in front of
    token_logprobs(), for instance.  With Q1 and Q128 the matrix as quantize_fp8() gives it, scales powers of two, in blocks
    of 1 and 128 rows by 128 columns,

        y = Q1(x) Q128(weight)^T,   dx = Q1(dy) Q128(weight),   dw = Q1(dy^T) Q1(x^T)^T

    (the blocks lie along what is summed over; products as matmul_fp8()'s, so blocks whose largest values multiply to less than
    about 1e-32 or more than about 1e43 are out of range).  ``dtype`` of y: that of x when not given.  The gradients have the
    types of x and weight, which may change after the call: the backward pass has codes of its own.  K >= 1.  On the current
    stream.  A call with a gradient that is captured into a graph is refused while the result of an eager one on the default
    stream, with the same leaf, is alive, and where x or weight itself comes from an eager call there: detach() it."""
    x_dtype, M, K, _ = _matrix(x, "x")
    _, N, columns, _ = _matrix(weight, "weight")
    if columns != K or K == 0:
        raise ValueError("x and weight must have the same columns, one or more")
    if dtype is None:
        dtype = x.dtype
    if dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("dtype must be float32 or bfloat16")
    _on_device(x=x, weight=weight)
    if not (torch.is_grad_enabled() and (x.requires_grad or weight.requires_grad)):
        x8, _ = _quantized(x, 1, torch.float8_e8m0fnu, True, None)
        w8, _ = _quantized(weight, BLOCK, torch.float8_e8m0fnu, True, None)
        return matmul_fp8(*x8, *w8, dtype=dtype)
    if _native.capture_meets_eager(x, weight):
        raise RuntimeError("linear_fp8 cannot be captured while an eager graph of x or weight is alive: delete its results first, "
                           "or detach() what comes from it")
    return _Linear.apply(x, weight, dtype)
