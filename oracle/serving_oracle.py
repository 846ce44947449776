"""fp64 oracle of serving a compact model token by token: new tokens into the caches, attention over a shared prefix and
own caches, eviction by accumulated attention weight, penalties / biases / masks on logits.  Plain loops over requests and
heads, one definition a line; every function takes and returns numpy arrays."""
from __future__ import annotations

import numpy as np


def turn(x, cos, sin):
    """Adjacent pairs (x0, x1) of the last axis turned: (x0 c - x1 s, x0 s + x1 c)."""
    x = np.asarray(x, dtype=np.float64)
    out = np.empty_like(x)
    out[..., 0::2] = x[..., 0::2] * cos - x[..., 1::2] * sin
    out[..., 1::2] = x[..., 0::2] * sin + x[..., 1::2] * cos
    return out


def append(qkv, k, v, lens, h, pos=None, cos=None, sin=None, w=None):
    """qkv [B*L, nqkv], caches k [B, h_kv, cap, e], v [.., f]; -> (q [B*L, h*e], k, v, w) with the last L rows of every cache set.
    cos/sin [h_kv, L_tab, e/2] or None.  A token without a row or an angle changes nothing and has a zero query."""
    B, h_kv, cap, e = k.shape
    f, L = v.shape[3], qkv.shape[0] // B
    k, v, w = k.copy(), v.copy(), None if w is None else w.copy()
    q_out = np.zeros((B * L, h * e))
    for b in range(B):
        for t in range(L):
            row, slot = qkv[b * L + t], int(lens[b]) - L + t
            at = int(pos[b]) + t if cos is not None else 0
            if slot < 0 or slot >= cap or (cos is not None and not 0 <= at < cos.shape[1]):
                continue
            for i in range(h):
                x = row[i * e:(i + 1) * e]
                g = i // (h // h_kv)
                q_out[b * L + t, i * e:(i + 1) * e] = x if cos is None else turn(x, cos[g, at], sin[g, at])
            for g in range(h_kv):
                x = row[(h + g) * e:(h + g + 1) * e]
                k[b, g, slot] = x if cos is None else turn(x, cos[g, at], sin[g, at])
                v[b, g, slot] = row[(h + h_kv) * e + g * f:(h + h_kv) * e + (g + 1) * f]
                if w is not None:
                    w[b, g, slot] = 0.0
    return q_out, k, v, w


def prefix_attn(q, k, v, lens, h, scale, pk=None, pv=None, w=None):
    """q [B*L, h*e] over prefix pk [h_kv, P, e] / pv and the own rows j < lens - L + 1 + t -> dict with
    o [B*L, h*f], lse [B, h, L], w [B, h_kv, cap], and what error bounds need: av = sum p |v| (as o), s_abs = the largest
    sum |scale q k| of a row (as lse)."""
    B, h_kv, cap, e = k.shape
    f, L, g = v.shape[3], q.shape[0] // B, h // h_kv
    P = 0 if pk is None else pk.shape[1]
    out = {"o": np.zeros((B * L, h * f)), "av": np.zeros((B * L, h * f)), "lse": np.full((B, h, L), -np.inf), "s_abs": np.zeros((B, h, L)),
           "w": np.zeros((B, h_kv, cap)) if w is None else np.array(w, dtype=np.float64)}
    for b in range(B):
        n = min(max(int(lens[b]), 0), cap)
        for i in range(h):
            hk = i // g
            keys, vals = k[b, hk, :n], v[b, hk, :n]
            if P:
                keys, vals = np.concatenate((pk[hk], keys)), np.concatenate((pv[hk], vals))
            for t in range(L):
                seen = P + min(max(n - L + 1 + t, 0), n)
                if seen == 0:
                    continue
                x = q[b * L + t, i * e:(i + 1) * e]
                s = scale * (keys[:seen] @ x)
                m = s.max()
                lse = m + np.log(np.exp(s - m).sum())
                p = np.exp(s - lse)
                out["o"][b * L + t, i * f:(i + 1) * f] = p @ vals[:seen]
                out["av"][b * L + t, i * f:(i + 1) * f] = p @ np.abs(vals[:seen])
                out["lse"][b, i, t] = lse
                out["s_abs"][b, i, t] = scale * (np.abs(keys[:seen]) @ np.abs(x)).max()
                out["w"][b, hk, :seen - P] += p[P:]
    return out


def evict(w, lens, keep, recent):
    """-> (kept [B][h_kv] lists of rows, ascending; new lengths)."""
    B, h_kv, _ = w.shape
    kept = []
    for b in range(B):
        n = int(lens[b])
        rows = []
        for g in range(h_kv):
            if n <= keep:
                rows.append(list(range(n)))
                continue
            old = n - recent
            key = [(np.isnan(x), -x if not np.isnan(x) else 0.0, j) for j, x in enumerate(w[b, g, :old])]      # NaN last, larger first, lower row first
            rows.append(sorted(j for _, _, j in sorted(key)[:keep - recent]) + list(range(old, n)))
        kept.append(rows)
    return kept, [min(int(n), keep) for n in lens]


def logits_process(x, history=None, history_len=None, repetition=None, frequency=None, presence=None, temperature=None, bias_ids=None,
                   bias=None, mask=None, mask_row=None):
    """-> (processed [B, V], pick [B], lse [B])."""
    x = np.array(x, dtype=np.float64)
    B, V = x.shape
    pick, lse = np.full(B, -1, dtype=np.int64), np.full(B, -np.inf)
    get = lambda a, b, d: d if a is None else float(a[b])
    for b in range(B):
        past = [] if history is None else history[b][:min(max(int(history_len[b]), 0), len(history[b])) if history_len is not None else len(history[b])]
        count = np.zeros(V)
        for v in past:
            if 0 <= v < V:
                count[v] += 1
        seen, rep = count > 0, get(repetition, b, 1.0)
        x[b] = np.where(seen, np.where(x[b] > 0, x[b] / rep, x[b] * rep), x[b])
        x[b] -= get(frequency, b, 0.0) * count + get(presence, b, 0.0) * seen
        if bias is not None:
            for v, y in zip(bias_ids[b], bias[b]):
                if 0 <= v < V:
                    x[b, v] += y
        x[b] /= get(temperature, b, 1.0)
        if mask is not None and 0 <= mask_row[b] < len(mask):
            words = np.asarray(mask[mask_row[b]]).astype(np.int64) & 0xffffffff
            v = np.arange(V)
            x[b][((words[v // 32] >> (v % 32)) & 1) == 0] = -np.inf
        ok = ~np.isnan(x[b])
        top = x[b][ok].max() if ok.any() else -np.inf
        if top > -np.inf:
            pick[b] = int(np.flatnonzero(ok & (x[b] == top))[0])
            lse[b] = np.inf if top == np.inf else top + np.log(np.exp(x[b] - top).sum())
        if not ok.all():                                   # a sum with what is not a number in it, whatever else there is
            lse[b] = np.nan
    return x, pick, lse
