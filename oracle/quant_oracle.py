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


# ---- caches of 8-bit floats ----------------------------------------------------------------------------------------------------------------
def e4m3(x):
    """The nearest e4m3 value (ties to even) of x, |x| <= 448; NaN for what is not finite."""
    x = np.asarray(x, np.float64)
    with np.errstate(invalid="ignore", divide="ignore"):
        e = np.maximum(np.floor(np.log2(np.where(x == 0, 1.0, np.abs(np.where(np.isfinite(x), x, 1.0))))), -6)      # below 2^-6 steps stay 2^-9
        return np.where(np.isfinite(x), np.rint(x / 2.0 ** (e - 3)) * 2.0 ** (e - 3), np.nan)


def block_scale(x):
    """The least power of two from 2^-100 on with |x| <= 448 times it (finite elements only)."""
    x = np.abs(np.asarray(x, np.float64))
    top = float(np.max(x[np.isfinite(x)], initial=0.0))
    e = -100
    while top > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def append(qkv, cache, lens, h, block, pos=None, cos=None, sin=None, rounded=None):
    """qkv [B*L, nqkv]; cache {"k", "v" (values of codes) [B, h_kv, cap, e | f], "k_scale", "v_scale"}; rounded: what rounds a turned key to
    its storage type.  -> (q, the cache after the call).  A token without a row or an angle changes nothing and has a zero query."""
    from .serving_oracle import turn
    B, h_kv, cap, e = cache["k"].shape
    f, L = cache["v"].shape[3], qkv.shape[0] // B
    out = {n: x.copy() for n, x in cache.items()}
    q_out = np.zeros((B * L, h * e))
    rounded = rounded or (lambda x: x)
    for b in range(B):
        first, new = int(lens[b]) - L, {}
        for t in range(L):
            row, slot = qkv[b * L + t], first + t
            at = int(pos[b]) + t if cos is not None else 0
            if slot < 0 or slot >= cap or (cos is not None and not 0 <= at < cos.shape[1]):
                continue
            for i in range(h):
                x, g = row[i * e:(i + 1) * e], i // (h // h_kv)
                q_out[b * L + t, i * e:(i + 1) * e] = x if cos is None else turn(x, cos[g, at], sin[g, at])
            for g in range(h_kv):
                x = row[(h + g) * e:(h + g + 1) * e]
                new["k", g, slot] = x if cos is None else rounded(turn(x, cos[g, at], sin[g, at]))
                new["v", g, slot] = row[(h + h_kv) * e + g * f:(h + h_kv) * e + (g + 1) * f]
        for name in ("k", "v"):
            for g in range(h_kv):
                for i in sorted({s // block for n, gg, s in new if n == name and gg == g}):
                    rows = {s: x for (n, gg, s), x in new.items() if n == name and gg == g and s // block == i}
                    codes, scales = out[name][b, g], out[name + "_scale"][b, g]
                    s = block_scale(np.array(list(rows.values())))
                    lo = max(first, 0)
                    if lo > i * block:
                        s = max(s, scales[i])
                        if s > scales[i]:
                            codes[i * block:lo] = e4m3(codes[i * block:lo] * (scales[i] / s))
                    for at, x in rows.items():
                        codes[at] = e4m3(np.asarray(x, np.float64) / s)
                    scales[i] = s
    return q_out, out


def attn(q, cache, lens, h, scale, block, o_in=None, lse_in=None):
    """q [B*L, h*e] over the rows j < lens - L + 1 + t -> {"o" [B*L, h*f], "lse" [B, h, L], "av": sum p |v| as o, "s_abs": the largest sum
    |scale q k| of a row}."""
    B, h_kv, cap, e = cache["k"].shape
    f, L, g = cache["v"].shape[3], q.shape[0] // B, h // h_kv
    o, av = np.zeros((B * L, h * f)), np.zeros((B * L, h * f))
    lse, s_abs = np.full((B, h, L), -np.inf), np.zeros((B, h, L))
    for b in range(B):
        for i in range(h):
            by = np.arange(cap) // block
            k = cache["k"][b, i // g] * cache["k_scale"][b, i // g][by, None]
            v = cache["v"][b, i // g] * cache["v_scale"][b, i // g][by, None]
            for t in range(L):
                n = max(min(int(lens[b]), cap) - L + 1 + t, 0)
                x = q[b * L + t, i * e:(i + 1) * e]
                s = scale * (k[:n] @ x)
                prior = -np.inf if lse_in is None else lse_in[b, i, t]
                m = max(np.max(s, initial=-np.inf), prior)
                if m == -np.inf:
                    continue
                p, w = np.exp(s - m), np.exp(prior - m)
                tot = p.sum() + w
                cols = slice(i * f, (i + 1) * f)
                o[b * L + t, cols] = p @ v[:n] / tot
                av[b * L + t, cols] = p @ np.abs(v[:n]) / tot
                if w > 0:
                    o[b * L + t, cols] += w * o_in[b * L + t, cols] / tot
                    av[b * L + t, cols] += w * np.abs(o_in[b * L + t, cols]) / tot
                lse[b, i, t] = m + np.log(tot)
                s_abs[b, i, t] = np.max(np.abs(scale) * (np.abs(k[:n]) @ np.abs(x)), initial=0.0)
    return {"o": o, "lse": lse, "av": av, "s_abs": s_abs}


# ---- drawing tokens ------------------------------------------------------------------------------------------------------------------------
def sample(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row of logits -> (token, its probability, clearance): clearance is how near, in weights of the best token, the draw or one of the borders came to
    another answer."""
    x = np.asarray(x, np.float64)
    number = ~np.isnan(x) & (x > -np.inf)
    if not number.any():
        return -1, 0.0, 1.0
    top = x[number].max()
    if not temperature > 0:
        return int(np.flatnonzero(x == top)[0]), 1.0, 1.0
    w = np.zeros(x.size)
    if top == np.inf:
        w[x == np.inf] = 1.0
    else:
        w[number] = np.exp((x[number] - top) / temperature)
    order = np.lexsort((np.arange(x.size), np.where(number, -x, np.inf)))
    order = order[w[order] > 0]
    if 1 <= top_k < order.size:
        order = order[:top_k]
    clear = 1.0
    if top_p < 1.0:
        cum = np.cumsum(w[order])
        goal = max(top_p, 0.0) * cum[-1]
        n = min(int(np.searchsorted(cum, goal)) + 1, order.size)
        near = np.abs(cum - goal)
        # a border that falls on a sum exactly (equal weights) is the oracle's as much as the library's
        clear = min(clear, float(np.min(np.where(near == 0, 1.0, near))))
        order = order[:n]
    if min_p > 0:
        keep = w[order] >= min(min_p, 1.0)
        if top < np.inf:
            near = np.abs(w[order] - min(min_p, 1.0))
            clear = min(clear, float(np.min(np.where(near == 0, 1.0, near))))
        order = order[keep]
    kept = np.sort(order)
    cum = np.cumsum(w[kept])
    u = 0.0 if np.isnan(u) else u
    goal = max(u, 0.0) * cum[-1]
    i = min(int(np.searchsorted(cum, goal, side="right")), kept.size - 1)
    near = np.abs(cum[:-1] - goal)
    if near.size:
        clear = min(clear, float(np.min(np.where(near == 0, 1.0, near))))
    return int(kept[i]), float(w[kept[i]] / cum[-1]), clear
