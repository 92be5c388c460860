"""CPU oracle of the paged prompt cache and of eviction by accumulated attention weight (TEST INFRASTRUCTURE ONLY).

Plain numpy in float64, one sequence and one query after the other in the order of the definitions; nothing here is shared with the HIP path.

  * a token at position p sees the pairs j <= p, with a window W > 0 those with j > p - W or j < n_sink; a pair in a hole of the page
    table is seen by nobody;
  * with s_j = scale * <q, k_j> / ln 2 over the pairs seen: M = max s_j, L = sum 2^(s_j - M), out = sum 2^(s_j - M) v_j / L, and the weight
    that pair j receives is 2^(s_j - M) / L;
  * accumulated weight: the sum of the weights a pair has received from all queries of all heads of its group since it entered.
"""
from __future__ import annotations

import numpy as np


def visible(p: int, n: int, window: int, n_sink: int, present: np.ndarray) -> np.ndarray:
    """bool [n]: the pairs that a query at position p sees."""
    out = np.zeros(n, bool)
    for j in range(min(n, p + 1)):
        out[j] = present[j] and (window == 0 or j > p - window or j < n_sink)
    return out


def pairs(pool: np.ndarray, table: np.ndarray, n: int):
    """The first n pairs of a sequence, float64 [Hkv, n, D], and which of them lie in a page; pool [pages, Hkv, page, D]."""
    P, H, ps, D = pool.shape
    x, present = np.zeros((H, n, D)), np.zeros(n, bool)
    for j in range(n):
        page = int(table[j // ps])
        if 0 <= page < P:
            x[:, j] = pool[page, :, j % ps]
            present[j] = True
    return x, present


def attend(q, K, V, present, first, window, n_sink, scale):
    """q float64 [c, Hq, D] at positions first .. first + c - 1, K, V [Hkv, n, D] -> out [c, Hq, D], M, L [c, Hq], weights [c, Hq, n]."""
    c, Hq, D = q.shape
    H, n, _ = K.shape
    g = Hq // H
    out, M, L, W = np.zeros((c, Hq, D)), np.full((c, Hq), -np.inf), np.zeros((c, Hq)), np.zeros((c, Hq, n))
    for t in range(c):
        seen = np.flatnonzero(visible(first + t, n, window, n_sink, present))
        if seen.size == 0:
            continue
        for h in range(H):
            s = q[t, h * g:(h + 1) * g] @ K[h, seen].T * (scale / np.log(2.0))      # [g, seen]
            m = s.max(axis=1)
            e = np.exp2(s - m[:, None])
            l = e.sum(axis=1)
            heads = slice(h * g, (h + 1) * g)
            M[t, heads], L[t, heads] = m, l
            W[t, heads][:, seen] = e / l[:, None]
            out[t, heads] = (e / l[:, None]) @ V[h, seen]
    return out, M, L, W


def received(W, H):
    """Weights [c, Hq, n] -> what every pair of every KV head received, [H, n]."""
    c, Hq, n = W.shape
    return W.reshape(c, H, Hq // H, n).sum(axis=(0, 2))


def accumulate(acc, W, H, first):
    """acc float64 [H, n] before the chunk at positions first ..; its own pairs start from zero."""
    out = acc.copy()
    out[:, first:] = 0
    return out + received(W, H)
