"""Plain 64-bit definitions of the 8-bit matrices of include/sbw_step.h, on the CPU, with the tolerances that the
kernels' 32-bit arithmetic allows.

Tolerances.  u = 2^-24 is the rounding error of one fp32 operation that rounds to nearest, 2 u that of one that
truncates, as additions inside a matrix instruction may.
* Codes and scales are exact: a scale of fp32 is one division, a code one product and one rounding.
* A product of two codes has at most 8 significant bits, exact in fp32.  A sum over K of them meets each at most K - 1
  times in an addition, blocks' sums at most as often as there are blocks, and a scale's product, the scaled sum and
  the product of two scales round three times a block.  Hence 2 u (K + 8) times the sum of magnitudes at most.
* For bf16 results each of eight neighbouring products (in any order of the columns within a block: of any eight) is
  cut off at 2^-13 of the power of two of the largest, so it loses less than 2^-13 of that one.  The sum over a block of
  the largest of eight is taken from the block's products in order, largest first, an eighth of them: no
  choice of eights has a larger sum.  The rounding to bf16 is off by 2^-8 of the result at most.
"""
import numpy as np

U = 2.0 ** -24
LARGEST = 448.0


def _decoded():
    t = np.empty(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        v = (8 + m) * 2.0 ** (e - 10) if e else m * 2.0 ** -9
        t[c] = np.nan if c & 127 == 127 else -v if c & 128 else v
    return t


DECODED = _decoded()                       # value of each e4m3 code
POSITIVE = DECODED[:127]                   # 0 to 448, in order


def encoded(v):
    """The nearest e4m3 value's code of float64 values, ties to the even one; NaN stays."""
    size = np.minimum(np.abs(v), LARGEST)
    at = np.clip(np.searchsorted(POSITIVE, np.nan_to_num(size)), 1, 126)
    low, high = POSITIVE[at - 1], POSITIVE[at]
    below, above = size - low, high - size
    code = np.where(below < above, at - 1, np.where(above < below, at, at - 1 + (at - 1) % 2)).astype(np.uint8)
    code = np.where(np.isnan(v), 127, code)
    return (code | np.where(np.signbit(v) & ~np.isnan(v), 128, 0)).astype(np.uint8)


def quantized(x, block_rows, e8m0):
    """(codes, scales as float64) of float32 values [M, K]."""
    M, K = x.shape
    codes = np.zeros((M, K), np.uint8)
    scales = np.zeros((-(-M // block_rows), -(-K // 128)))
    for i in range(scales.shape[0]):
        for j in range(scales.shape[1]):
            part = x[i * block_rows:(i + 1) * block_rows, j * 128:j * 128 + 128].astype(np.float32)
            finite = np.isfinite(part)
            a = np.float32(np.abs(part[finite]).max()) if finite.any() else np.float32(0)
            if e8m0:
                e = -127
                while float(a) > LARGEST * 2.0 ** e:
                    e += 1
                s = np.float32(2.0 ** e)
            else:
                s = np.maximum(a / np.float32(LARGEST), np.float32(2.0 ** -126))
            with np.errstate(invalid="ignore", over="ignore"):
                v = np.where(finite, part * (np.float32(1) / s if not e8m0 else np.float32(2.0 ** -e)), np.nan)
            codes[i * block_rows:(i + 1) * block_rows, j * 128:j * 128 + 128] = encoded(v.astype(np.float64))
            scales[i, j] = s
    return codes, scales


def spread(scales, rows, columns):
    """Scales as a matrix of the codes' size."""
    s = np.repeat(scales, 128, axis=1)[:, :columns]
    return s if s.shape[0] == rows else np.repeat(s, 128, axis=0)[:rows]


def values(codes, scales):
    return DECODED[codes] * spread(scales, *codes.shape)


def cut_off(x, y):
    """What eights of neighbours can lose of x y^T: 7 of each eight, 2^-13 of the largest."""
    lost = np.zeros((x.shape[0], y.shape[0]))
    for j in range(0, x.shape[1], 128):
        p = np.abs(x[:, None, j:j + 128] * y[None, :, j:j + 128])
        eights = -(-p.shape[2] // 8)
        lost += np.partition(p, p.shape[2] - eights, axis=2)[:, :, -eights:].sum(axis=2)
    return lost * 7 * 2.0 ** -13


def product(a, a_scales, b, b_scales, bf16=False):
    """(a b^T, tolerance) of codes and scales, float64."""
    x, y = values(a, a_scales), values(b, b_scales)
    with np.errstate(invalid="ignore"):
        out = x @ y.T
    x, y = np.nan_to_num(x), np.nan_to_num(y)
    tol = 2 * U * (a.shape[1] + 8) * (np.abs(x) @ np.abs(y).T) + 2.0 ** -126
    if bf16:
        tol = (tol + cut_off(x, y)) * 1.01 + 2.0 ** -8 * np.abs(np.nan_to_num(out))
    return out, tol
