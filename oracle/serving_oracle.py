"""float64 definition of the operators of serving word by word (include/kv_cache.h, vocab_verify in include/vocab_ops.h): codes of
a cache in 8 bits, attention of the newest tokens over a paged cache, verification of drafted words.  One row, one sequence at a
time, no blocking; shares no code with the library."""
from __future__ import annotations

import math

import numpy as np

LARGEST = {"int8": 127.0, "e4m3": 448.0}


def encode(x, cache):
    """(the values that the codes are, the scale) of a row of float32, every step rounded to float32 as the format says."""
    x = np.asarray(x, dtype=np.float32)
    if not np.isfinite(x).all():
        return np.zeros(x.shape), np.float32(np.nan)
    scale = np.maximum(np.abs(x).max() * (np.float32(1.0) / np.float32(LARGEST[cache])), np.float32(2.0 ** -120))
    y = (x * (np.float32(1.0) / scale)).astype(np.float64)
    if cache == "int8":
        return np.rint(y) + 0.0, scale      # (no zero below zero)
    code = y.copy()                         # (zeros keep their sign)
    for i, v in np.ndenumerate(y):
        if v != 0:
            step = 2.0 ** (max(math.frexp(abs(v))[1] - 1, -6) - 3)      # 3 bits behind the leading one; 2^-9 below 2^-6
            code[i] = np.rint(v / step) * step
    return code, scale


def place(seq, pos, table, page, pages):
    """(page, place in it) of a token, or None."""
    if not (0 <= seq < len(table) and 0 <= pos < len(table[seq]) * page):
        return None
    p = table[seq][pos // page]
    return (p, pos % page) if 0 <= p < pages else None


def attn(q, k, v, there, scale, window=0):
    """q [T,q_heads,D]; k, v [n,heads,D] of one sequence, float64; there [n]: tokens whose page is one.  -> out, lse."""
    T, q_heads, D = q.shape
    n, heads = k.shape[0], k.shape[1]
    out, lse = np.zeros((T, q_heads, D)), np.full((T, q_heads), -np.inf)
    for t in range(T):
        pos = n - T + t
        seen = [i for i in range(max(0, pos - window + 1) if window else 0, pos + 1) if there[i]]
        if not seen:
            continue
        for h in range(q_heads):
            a = scale * (k[seen, h * heads // q_heads] @ q[t, h])
            m = a.max()
            w = np.exp(a - m)
            lse[t, h] = m + np.log(w.sum())
            out[t, h] = (w / w.sum()) @ v[seen, h * heads // q_heads]
    return out, lse


def softmax(l, tau):
    """None where it is no distribution."""
    l = np.asarray(l, dtype=np.float64) / tau
    m = l.max()
    if not m < np.inf or m == -np.inf:
        return None
    e = np.exp(l - m)
    return e / e.sum()


def verify(target, draft, drafted, u_accept, u_next, tau):
    """One sequence: (accepted, words [T+1])."""
    T, V = draft.shape
    words = np.full(T + 1, -1, dtype=np.int64)
    n = 0
    while True:
        p = softmax(target[n], tau)
        given = n < T and 0 <= drafted[n] < V
        q = softmax(draft[n], tau) if given else np.zeros(V)
        if p is None or q is None:
            return n, words
        if given and float(u_accept[n]) * q[drafted[n]] < p[drafted[n]]:
            words[n] = drafted[n]
            n += 1
            continue
        rest = np.maximum(p - q, 0.0)
        if not rest.sum() > 0:
            rest = p
        total = np.cumsum(rest)
        above = np.nonzero(total > max(float(u_next), 0.0) * total[-1])[0]
        words[n] = above[0] if len(above) else np.nonzero(rest)[0][-1]
        return n, words
