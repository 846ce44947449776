"""fp64 oracle of serving in eight bits: rows and products of 8-bit integers, caches of 8-bit floats with block scales, attention over them,
drawing tokens.  Plain loops over requests and heads, one definition a line; every function takes and returns numpy arrays."""
from __future__ import annotations

import math

import numpy as np

ACT_NONE, ACT_GELU_ERF, ACT_GELU_TANH, ACT_SWIGLU = -1, 0, 1, 2


def quant_rows(x):
    """x float32 [rows, cols] -> (int8 codes, float32 scales): both quotients are fp32 divisions."""
    x = np.asarray(x, dtype=np.float32)
    fine = np.isfinite(x).all(axis=1)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        scale = (np.abs(x).max(axis=1) / np.float32(127.0)).astype(np.float32)
        q = np.rint(x / np.where(fine & (scale > 0), scale, np.float32(1.0))[:, None])
    q = np.clip(q, -127.0, 127.0)      # subnormal scales are coarse
    q[~fine | (scale == 0)] = 0.0
    scale[~fine] = np.nan
    return q.astype(np.int8), scale


def contract_quant(A, sa, B, sb, bias=None, act=ACT_NONE):
    """-> (C, slack): slack bounds what the fp32 steps in front of the last rounding may be off by, in units of an fp32 half step (2^-24)."""
    p = (A.astype(np.int64) @ B.astype(np.int64).T).astype(np.float64) * np.asarray(sa, np.float64)[:, None] * np.asarray(sb, np.float64)[None]
    b = np.zeros(B.shape[0]) if bias is None else np.asarray(bias, np.float64)
    y = p + b
    off = 3.0 * np.abs(p) + np.abs(y)      # the sum to fp32, two scales, and the addition, each half a step
    if act == ACT_NONE:
        return y, off
    if act == ACT_SWIGLU:
        g, u, og, ou = y[:, 0::2], y[:, 1::2], off[:, 0::2], off[:, 1::2]
        with np.errstate(over="ignore"):
            s = 1.0 / (1.0 + np.exp(-g))
        # |d silu| <= 1.1; exponential and reciprocal a few steps of their own, the exponential's argument |g| times its rounding
        return g * s * u, 1.1 * og * np.abs(u) + np.abs(g * s) * ou + (16.0 + 4.0 * np.abs(g)) * np.abs(g * s * u)
    if act == ACT_GELU_ERF:
        phi = 0.5 * np.vectorize(math.erfc)(-y / math.sqrt(2.0)) if y.size else y
        return y * phi, 1.13 * off + 8.0 * np.abs(y)       # the tail is good to 3e-7 (5 half steps) of its factor
    t = np.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3))
    return 0.5 * y * (1.0 + t), 1.13 * off + 16.0 * np.abs(y)
