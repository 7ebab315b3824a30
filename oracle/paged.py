"""Generation by sampling over a paged cache, as its definitions, in fp64.

Plain numpy, one row, head and token at a time; it shares no code with the GPU
library.  Caches are [P, Hkv, page, D] arrays, bf16 values as their uint16 bits.

* :func:`paged_append` -- new tokens' keys and values to the positions that
  follow those their rows hold.
* :func:`paged_attn` -- softmax attention of one query per head over the
  positions that a row's table names.
* :func:`token_sample` -- the draw of one token per row by temperature, top-k,
  top-p and min-p from a given uniform number.
"""
import math

import numpy as np


def _f64(a: np.ndarray) -> np.ndarray:
    if a.dtype == np.uint16:   # bf16 bits: the upper half of an fp32 value
        return (a.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    return a.astype(np.float64)


def _slot(table, r, pos, page, P):
    """(page, slot) of position pos of row r, or None."""
    if pos < 0 or pos // page >= table.shape[1]:
        return None
    pg = int(table[r, pos // page])
    return (pg, pos % page) if 0 <= pg < P else None


def paged_append(K, V, k, v, table, start, offsets=None):
    """The two caches after the tokens were written (copies)."""
    K, V = K.copy(), V.copy()
    P, page = K.shape[0], K.shape[2]
    R = table.shape[0]
    offsets = np.arange(R + 1) if offsets is None else offsets
    for r in range(R):
        for n in range(max(0, int(offsets[r])), min(int(offsets[r + 1]), k.shape[0])):
            at = _slot(table, r, int(start[r]) + n - int(offsets[r]), page, P)
            if at is not None:
                K[at[0], :, at[1]] = k[n]
                V[at[0], :, at[1]] = v[n]
    return K, V


def paged_attn(q, K, V, table, kv_len, k=None, v=None, scale=None):
    """out [R, Hq, D] fp64, and (with k, v) the caches after the write."""
    R, Hq, D = q.shape
    P, Hkv, page = K.shape[:3]
    scale = D ** -0.5 if scale is None else scale
    if k is not None:
        K, V = K.copy(), V.copy()
    out = np.zeros((R, Hq, D))
    for r in range(R):
        L = min(max(int(kv_len[r]), 0), table.shape[1] * page)
        slots = [_slot(table, r, j, page, P) for j in range(L)]
        if k is not None and L > 0 and int(kv_len[r]) == L and slots[-1] is not None:
            K[slots[-1][0], :, slots[-1][1]] = k[r]
            V[slots[-1][0], :, slots[-1][1]] = v[r]
        slots = [s for s in slots if s is not None]
        if not slots:
            continue
        pg, sl = np.array(slots).T
        for g in range(Hkv):
            kk, vv = _f64(K[pg, g, sl]), _f64(V[pg, g, sl])
            for h in range(g * (Hq // Hkv), (g + 1) * (Hq // Hkv)):
                s = scale * (kk @ _f64(q[r, h]))
                p = np.exp(s - s.max())
                out[r, h] = (p / p.sum()) @ vv
    return (out, K, V) if k is not None else out


def token_sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """(token int32 [R], logprob fp64 [R])."""
    R, V = logits.shape
    tok, lp = np.full(R, -1, np.int32), np.full(R, np.nan)
    for r in range(R):
        x = _f64(logits[r])
        T = 1.0 if temperature is None else float(temperature[r])
        k = 0 if top_k is None else int(top_k[r])
        p = 1.0 if top_p is None else float(top_p[r])
        m = 0.0 if min_p is None else float(min_p[r])
        if np.isnan(x).any() or np.isposinf(x).any() or np.isneginf(x).all() or not T >= 0:
            continue
        if T == 0:
            tok[r], lp[r] = int(np.argmax(x)), 0.0
            continue
        w = np.zeros(V)
        live = x > -np.inf
        w[live] = np.exp((x[live] - x.max()) / T)
        order = np.argsort(-x, kind="stable")
        if 0 < k < V:
            order = order[:k]
        if p < 1:
            mass = np.cumsum(w[order])
            n = int(np.sum(mass - w[order] < p * mass[-1]))
            order = order[:max(n, 1)]
        if m > 0:
            order = order[w[order] >= min(m, 1.0)]
        kept = np.sort(order[w[order] > 0])
        run = np.cumsum(w[kept])
        past = np.flatnonzero(run > float(u[r]) * run[-1])
        i = kept[past[0]] if len(past) else kept[-1]
        tok[r], lp[r] = i, math.log(w[i] / run[-1])
    return tok, lp
