"""The e4m3 form and its products from their definition, in 64 bits, on the CPU (numpy).  Independent of the library."""
from __future__ import annotations

import numpy as np

TOP = 448.0


def e4m3_values() -> np.ndarray:
    """Value of every code (codes 0x7F and 0xFF: NaN)."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e.astype(float) - 10))
    v = np.where((c & 0x7F) == 0x7F, np.nan, v)
    return np.where(c & 0x80, -v, v)


VALUES = e4m3_values()
_ASCENDING = VALUES[:0x7F]                                   # non-negative finite values by code


def e4m3_codes(v: np.ndarray) -> np.ndarray:
    """Nearest code of 64-bit values (ties to the even code; magnitudes past 464 and NaN: NaN), by search over all values."""
    a = np.abs(v)
    hi = np.clip(np.searchsorted(_ASCENDING, a), 1, 0x7E)
    lo = hi - 1
    d = (a - _ASCENDING[lo]) - (_ASCENDING[hi] - a)
    code = np.where(d < 0, lo, np.where(d > 0, hi, np.where(lo % 2 == 0, lo, hi)))
    code = np.where(a == 0, 0, code)
    code = np.where(np.isnan(a) | (a > 464), 0x7F, code)
    return (code | np.where(np.signbit(v), 0x80, 0)).astype(np.uint8)


def _quantize(blocks: np.ndarray, axes):
    """Codes and scales of fp16 blocks: scale, factor and product are fp32, each rounded once."""
    a = blocks.astype(np.float64)
    bits = np.abs(blocks).view(np.uint16).max(axes, keepdims=True)        # magnitudes order like their bits, NaN last
    most = bits.view(np.float16).astype(np.float64)
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        factor = np.where(most > 0, TOP / most, most).astype(np.float32).astype(np.float64)
        scale = (most / TOP).astype(np.float32)
        codes = e4m3_codes((a * factor).astype(np.float32).astype(np.float64))
    return codes, scale


def _pad(w: np.ndarray, rows: int, cols: int) -> np.ndarray:
    return np.pad(w, ((0, -w.shape[0] % rows), (0, -w.shape[1] % cols)))


def quantize_rows(x: np.ndarray):
    """fp16 [n,in] -> codes [n,in], fp32 scales [ceil(in/128), n]."""
    n, inn = x.shape
    b = _pad(x, 1, 128).reshape(n, -1, 128)
    codes, scale = _quantize(b, 2)
    return np.ascontiguousarray(codes.reshape(n, -1)[:, :inn]), np.ascontiguousarray(scale[:, :, 0].T)


def quantize_matrix(w: np.ndarray):
    """fp16 [out,in] -> codes [out,in], fp32 scales [ceil(out/128), ceil(in/128)]."""
    out, inn = w.shape
    p = _pad(w, 128, 128)
    b = p.reshape(p.shape[0] // 128, 128, -1, 128)
    codes, scale = _quantize(b, (1, 3))
    return np.ascontiguousarray(codes.reshape(p.shape)[:out, :inn]), np.ascontiguousarray(scale[:, 0, :, 0])


def row_values(codes, scale):
    return VALUES[codes] * np.repeat(scale.T.astype(np.float64), 128, 1)[:, : codes.shape[1]]


def matrix_values(codes, scale):
    out, inn = codes.shape
    s = np.repeat(np.repeat(scale.astype(np.float64), 128, 0), 128, 1)
    return VALUES[codes] * s[:out, :inn]


def product(xv, wv):
    """(y, sum of magnitudes) in 64 bits."""
    return xv @ wv.T, np.abs(xv) @ np.abs(wv).T


def cut_bound(xv, wv):
    """What the matrix instructions for 8-bit operands may cut off: they bring the eight products of neighbouring columns to the
    exponent of the largest and drop what lies 13 binary places below it, less than that from each of the other seven."""
    n, inn = xv.shape
    total = np.zeros((n, wv.shape[0]))
    for c in range(0, inn, 8):
        p = np.abs(xv[:, None, c:c + 8] * wv[None, :, c:c + 8]).max(2)
        total += 8 * 2.0 ** -13 * p
    return total


def sum_bound(inn: int, mag):
    """Roundings that a product meets on its way through fp32 sums: 128 of its block (each up to a whole step, 2^-23), one per block
    after it, those of the scales and of eight partial sums."""
    return (256 + inn / 128 + 16) * 2.0 ** -24 * mag


def rounded(y, half: bool):
    """Bound of the rounding of y to its type (the smallest step of fp16 included)."""
    return np.abs(y) * 2.0 ** -11 + 2.0 ** -25 if half else np.abs(y) * 2.0 ** -24
