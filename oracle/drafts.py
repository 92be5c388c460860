"""CPU oracle of drafted tokens over a cache (TEST INFRASTRUCTURE ONLY): rotary positions, attention of trees, verification, commit.

Plain numpy in float64, one sequence, node and head after the other in the order of the definitions; nothing here is shared with the HIP path.
"""
from __future__ import annotations

import numpy as np

MOST_NODES = 256


def ancestors(parent, i):
    """Node i and its ancestors, itself first; a parent that does not come before its child stands for none."""
    way = []
    while True:
        way.append(i)
        p = int(parent[i])
        if p < 0 or p >= i:
            return way
        i = p


def visible(parent, i, n, window, n_sink, present):
    """What node i sees: bool [n] of the cache's pairs, and which nodes of its tree."""
    way = ancestors(parent, i)
    p = n + len(way) - 1
    old = np.array([present[j] and (window == 0 or j > p - window or j < n_sink) for j in range(n)], bool)
    new = [a for up, a in enumerate(way) if window == 0 or up < window or p - up < n_sink]
    return old, new


def attend(q, K, V, present, k_tree, v_tree, parent, window, n_sink, scale):
    """q [T, Hq, D], K, V [H][n_h, D] (rows may differ in length), present [H][n_h] bool, k_tree, v_tree [T, H, D] -> out, M, L and the sum of weight * |V|."""
    T, Hq, D = q.shape
    H = len(K)
    g = Hq // H
    out, M, L, mag = np.zeros((T, Hq, D)), np.full((T, Hq), -np.inf), np.zeros((T, Hq)), np.zeros((T, Hq, D))
    for i in range(T):
        for h in range(H):
            old, new = visible(parent, i, K[h].shape[0], window, n_sink, present[h])
            kk = np.concatenate([K[h][old], k_tree[new, h]])
            vv = np.concatenate([V[h][old], v_tree[new, h]])
            if kk.shape[0] == 0:
                continue
            for hq in range(h * g, (h + 1) * g):
                s = kk @ q[i, hq] * (scale / np.log(2.0))
                m = s.max()
                if m == -np.inf:
                    continue
                w = np.exp2(s - m)
                M[i, hq], L[i, hq] = m, w.sum()
                out[i, hq] = (w / w.sum()) @ vv
                mag[i, hq] = (w / w.sum()) @ np.nan_to_num(np.abs(vv), posinf=0)
    return out, M, L, mag


def rotate(x, pos, freq, layout, rotary_dim, magnitude=1.0, inverse=False):
    """x [tokens, heads, D]; angles in extended precision."""
    y = x.copy()
    a = pos.astype(np.longdouble)[:, None] * freq.astype(np.longdouble)[None]
    if inverse:
        a = -a
    c, s = magnitude * np.cos(a).astype(np.float64), magnitude * np.sin(a).astype(np.float64)
    for i in range(rotary_dim // 2):
        u, w = (i, i + rotary_dim // 2) if layout == "half" else (2 * i, 2 * i + 1)
        y[:, :, u] = x[:, :, u] * c[:, i, None] - x[:, :, w] * s[:, i, None]
        y[:, :, w] = x[:, :, u] * s[:, i, None] + x[:, :, w] * c[:, i, None]
    return y


def verify(target, draft, tokens, parent, uniform):
    """One tree: target, draft [T, vocab] float64 (draft None: tokens that were not drawn) -> path, next token."""
    T, vocab = target.shape
    if T == 0 or T > MOST_NODES:
        return [], -1
    path = [0]
    while True:
        at = path[-1]
        p = np.where(target[at] > 0, target[at], 0.0)
        r, m, found = p.copy(), 1.0, None
        for i in range(at + 1, T):
            if int(parent[i]) != at:
                continue
            x = int(tokens[i])
            there = 0 <= x < vocab
            rx = r[x] if there else 0.0
            if draft is not None:
                q = draft[at]
                if uniform[i] * (q[x] if there else 0.0) < rx:
                    found = i
                    break
                left = r - q
                r = np.where(left > 0, left, 0.0)
                total = r.sum()
                r = r / total if total > 0 else np.zeros_like(r)
            else:
                if uniform[i] * m < rx:
                    found = i
                    break
                m = max(m - rx, 0.0)
                if there:
                    r[x] = 0.0
        if found is None:
            break
        path.append(found)
    if not (r > 0).any():
        r = p
    if not (r > 0).any():
        return path, -1
    below = np.cumsum(r)
    hit = np.flatnonzero((below > uniform[0] * below[-1]) & (r > 0))
    return path, int(hit[0]) if hit.size else int(np.flatnonzero(r > 0)[-1])


def path_of(path, count, nodes):
    """The nodes that join: the first `count` entries, up to the first that is none."""
    out = []
    for x in path[:max(0, min(int(count), nodes))]:
        if not 0 <= x < nodes:
            break
        out.append(int(x))
    return out
