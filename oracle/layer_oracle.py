"""Float64 model of a target layer's steps around its attention: 8-bit rows with a scale per 32 elements, RMS norm
with the residual's addition, matrix products with their epilogue, rotary positions with several axes.

Written from the definitions in include/jakiro.h, one step per function; it shares no code with the library or its
binding.  Codes and scales are kept as the values they stand for; `tiles` gives the stored order of the scales."""
from __future__ import annotations

import math

import numpy as np

_erf = np.vectorize(math.erf, otypes=[np.float64])


# ------------------------------------------------------------------------------------------ 8-bit rows
def e4m3(x):
    """The nearest number of the e4m3 grid (ties to even; 3 fraction bits, smallest step 2^-9, largest 448)."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(x)
    with np.errstate(divide="ignore", invalid="ignore"):
        step = np.exp2(np.maximum(np.floor(np.log2(np.where(a > 0, a, 1.0))), -6.0) - 3.0)
        r = np.minimum(np.rint(np.where(np.isfinite(a), a, 448.0) / step) * step, 448.0)
    r = np.where(np.isinf(a), 448.0, r)
    return np.where(np.isnan(x), np.nan, np.copysign(r, x))


def scale_exponents(y):
    """[rows, n] -> exponents [rows, n / 32]: the smallest e >= -32 with max|finite| <= 448 2^e."""
    y = np.asarray(y, dtype=np.float64)
    b = np.where(np.isfinite(y), np.abs(y), 0.0).reshape(y.shape[0], -1, 32).max(2)
    e = np.full(b.shape, -32, dtype=np.int64)
    while np.any(b > 448.0 * np.exp2(e)):
        e = np.where(b > 448.0 * np.exp2(e), e + 1, e)
    return e


def quantize(y):
    """[rows, n] -> (codes' values [rows, n], exponents [rows, n / 32])."""
    e = scale_exponents(y)
    return e4m3(np.asarray(y, dtype=np.float64) / np.repeat(np.exp2(e), 32, axis=1)), e


def dequantize(codes, e):
    return np.asarray(codes, dtype=np.float64) * np.repeat(np.exp2(np.asarray(e, dtype=np.float64)), 32, axis=1)


def tile_index(rows, n):
    """Byte of the scale of (row, block) in the stored order, [rows, n / 32]."""
    out = np.empty((rows, n // 32), dtype=np.int64)
    kt = -(-n // 128)
    for r in range(rows):
        for k in range(n // 32):
            out[r, k] = (r // 128 * kt + k // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + k % 4
    return out


# ------------------------------------------------------------------------------------------ norm
def add_norm(x, delta, weight, eps):
    """(s, y): s = x + delta, y = s / sqrt(mean(s^2) + eps) * weight, row by row."""
    s = np.asarray(x, dtype=np.float64) + (0.0 if delta is None else np.asarray(delta, dtype=np.float64))
    y = s / np.sqrt(np.mean(s * s, axis=1, keepdims=True) + eps)
    return s, y if weight is None else y * np.asarray(weight, dtype=np.float64)


# ------------------------------------------------------------------------------------------ product
def act(z, kind):
    if kind == "silu":
        return z / (1.0 + np.exp(-z))
    if kind == "gelu":
        return 0.5 * z * (1.0 + _erf(z / math.sqrt(2.0)))
    return z


def linear(x, w, bias=None, kind="none", w_up=None, bias_up=None, residual=None):
    """act(x w^T + bias) [* (x w_up^T + bias_up)] [+ residual]"""
    x = np.asarray(x, dtype=np.float64)
    z = x @ np.asarray(w, dtype=np.float64).T + (0.0 if bias is None else np.asarray(bias, dtype=np.float64))
    y = act(z, kind)
    if w_up is not None:
        y = y * (x @ np.asarray(w_up, dtype=np.float64).T
                 + (0.0 if bias_up is None else np.asarray(bias_up, dtype=np.float64)))
    return y if residual is None else y + np.asarray(residual, dtype=np.float64)


# ------------------------------------------------------------------------------------------ rotary positions
def rope(qkv, pos, sections, theta, Hq, Hkv, d):
    """qkv [B, M, (Hq + 2 Hkv) d], pos [B, M, axes] -> q [B, M, Hq, d], k, v [B, Hkv, M, d]."""
    qkv = np.asarray(qkv, dtype=np.float64)
    B, M = qkv.shape[:2]
    heads = qkv.reshape(B, M, Hq + 2 * Hkv, d)
    out = heads.copy()
    half, axis = d // 2, [a for a, n in enumerate(sections) for _ in range(n)]
    for i in range(half):
        ang = np.asarray(pos, dtype=np.float64)[..., axis[i]] * theta ** (-2.0 * i / d)
        c, s = np.cos(ang)[..., None], np.sin(ang)[..., None]
        a, b = heads[:, :, :Hq + Hkv, i], heads[:, :, :Hq + Hkv, half + i]
        out[:, :, :Hq + Hkv, i] = a * c - b * s
        out[:, :, :Hq + Hkv, half + i] = b * c + a * s
    kv = out[:, :, Hq:].transpose(0, 2, 1, 3)
    return out[:, :, :Hq], kv[:, :Hkv], kv[:, Hkv:]
