"""Generation by sampling over a paged cache, as its definitions, in fp64.

Plain numpy, one row, head and token at a time; it shares no code with the GPU
library.  Caches are [P, Hkv, page, D] arrays, bf16 values as their uint16 bits.

* :func:`paged_append` -- new tokens' keys and values to the positions that
  follow those their rows hold.
* :func:`paged_attn` -- softmax attention of one query per head over the
  positions that a row's table names.
* :func:`paged_resize` -- rows that grow and shrink: their pages, and the positions
  and slots of new tokens.
* :func:`rotary`, :func:`rotary_frequencies` -- heads turned by their positions.
* :func:`paged_chunk_attn` -- causal attention of several new tokens per row.
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


def paged_resize(table, kv_len, want, free_pages, free_count, page, N=0):
    """The state after the call (copies) and what it says of the tokens, as a dict."""
    table, kv_len, free = table.copy(), kv_len.copy(), free_pages.copy()
    R, cols = table.shape
    P, cap = len(free), cols * page
    count = min(max(int(free_count), 0), P)
    held = [min(max(int(x), 0), cap) for x in kv_len]
    wants = [max(int(x), 0) for x in want]
    pages = lambda n: -(-n // page)
    for r in reversed(range(R)):
        for j in reversed(range(pages(wants[r]), pages(held[r]))):
            if 0 <= table[r, j] < P:
                if count < P:
                    free[count] = table[r, j]
                count += 1
            table[r, j] = -1
    count = min(count, P)
    needed, top, granted = 0, count, []
    for r in range(R):
        more = pages(wants[r]) - pages(held[r])
        ok = wants[r] <= cap
        if ok and more > 0:
            needed += more
            ok = needed <= top
        granted.append(ok)
        if ok:
            for j in range(pages(held[r]), pages(wants[r])):
                count -= 1
                table[r, j] = free[count]
            kv_len[r] = wants[r]
        elif more > 0:
            table[r, pages(held[r]):pages(wants[r])] = -1
    off = [0]
    for r in range(R):
        off.append(off[-1] + max(0, wants[r] - held[r]))
    positions, slots = np.zeros(N, np.int32), np.full(N, -1, np.int64)
    for r in range(R):
        for n in range(off[r], min(off[r + 1], N)):
            pos = positions[n] = held[r] + n - off[r]
            if granted[r] and 0 <= table[r, pos // page] < P:
                slots[n] = int(table[r, pos // page]) * page + pos % page
    return dict(table=table, kv_len=kv_len, free_pages=free, free_count=count, start=np.array(held, np.int32),
                offsets=np.minimum(np.array(off, np.int64), 2**31 - 1).astype(np.int32), positions=positions, slots=slots)


def rotary_frequencies(rot, base=10000.0, factor=1.0, context=0, fast=32.0, slow=1.0):
    out = []
    for i in range(rot // 2):
        f = base ** (-2 * i / rot)
        g = min(1.0, max(0.0, (context * f / (2 * math.pi) - slow) / (fast - slow))) if context else 0.0
        out.append(f / factor * (1 - g) + f * g)
    return np.array(out)


def rotary(x, positions, freq, interleaved=False, magnitude=1.0):
    """x [N, H, D] turned, fp64."""
    x = _f64(x)
    out, half = x.copy(), len(freq)
    for n, p in enumerate(positions):
        for i, f in enumerate(freq):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
            z = (x[n, :, a] + 1j * x[n, :, b]) * magnitude * complex(math.cos(int(p) * f), math.sin(int(p) * f))
            out[n, :, a], out[n, :, b] = z.real, z.imag
    return out


def paged_chunk_attn(q, K, V, table, kv_len, offsets, scale=None):
    """out [N, Hq, D] fp64 (NaN for tokens of no row), and the softmax-weighted mean of the
    values' magnitudes, of the same shape."""
    N, Hq, D = q.shape
    P, Hkv, page = K.shape[:3]
    scale = D ** -0.5 if scale is None else scale
    out, mean = np.full((N, Hq, D), np.nan), np.zeros((N, Hq, D))
    cap = table.shape[1] * page
    for r in range(table.shape[0]):
        lo, hi = int(offsets[r]), int(offsets[r + 1])
        for n in range(max(lo, 0), min(hi, N)):
            p = max(int(kv_len[r]), 0) - hi + n
            out[n] = 0
            slots = [s for s in (_slot(table, r, j, page, P) for j in range(min(p + 1, cap))) if s is not None]
            if not slots:
                continue
            pg, sl = np.array(slots).T
            for g in range(Hkv):
                kk, vv = _f64(K[pg, g, sl]), _f64(V[pg, g, sl])
                hs = slice(g * (Hq // Hkv), (g + 1) * (Hq // Hkv))
                s = scale * (_f64(q[n, hs]) @ kk.T)
                w = np.exp(s - s.max(1, keepdims=True))
                w /= w.sum(1, keepdims=True)
                out[n, hs], mean[n, hs] = w @ vv, w @ np.abs(vv)
    return out, mean


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
