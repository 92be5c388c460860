"""Cases of drafted trees over a cache: seeded inputs, the oracle's results and the error that the arithmetic allows."""
from __future__ import annotations

import numpy as np
import torch

from oracle import drafts as od

U = 2.0 ** -24       # half a step of fp32, relative
UB = 2.0 ** -8       # half a step of bf16, relative


def tree(n, seed=0, depth=None, fan=8):
    """A random tree of n nodes, parents first; depth 0: a chain."""
    r = np.random.default_rng(seed)
    parent, level = [-1], [0]
    for i in range(1, n):
        if depth == 0:
            p = i - 1
        else:
            c = [j for j in range(max(0, i - fan), i) if depth is None or level[j] < depth] or [0]
            p = int(r.choice(c))
        parent.append(p)
        level.append(level[p] + 1)
    return parent


class TreeCase:
    """seqs: [(length or lengths of the KV heads, parents), ...], one per sequence.  page 0: rows.  Host tensors, bf16 values exact in float64."""

    def __init__(self, dtype, D, g, hkv, seqs, page=0, window=0, n_sink=0, scale=None, seed=0, before=0, behind=0, room=5, key_scale=1.0, max_tree=None, max_len=None):
        gen = torch.Generator().manual_seed(seed)
        self.dtype, self.D, self.g, self.H, self.page, self.seqs = dtype, D, g, hkv, page, seqs
        self.window, self.n_sink, self.scale = window, n_sink, D ** -0.5 if scale is None else scale
        self.dt = torch.float32 if dtype == "f32" else torch.bfloat16
        self.B = len(seqs)
        self.lens = np.array([[n] * hkv if np.isscalar(n) else n for n, _ in seqs], np.int32)   # [B, H]
        sizes = [len(p) for _, p in seqs]
        starts = before + np.concatenate([[0], np.cumsum(sizes)])
        self.q_start = torch.tensor(starts, dtype=torch.int32)
        self.n_tokens = int(starts[-1]) + behind
        parent = np.full(self.n_tokens, 10 ** 6, np.int32)   # (of nobody's tokens: nonsense)
        for (_, p), s in zip(seqs, starts):
            parent[s:s + len(p)] = p
        self.parent = torch.tensor(parent)
        top = max(1, int(self.lens.max(initial=0)))
        self.max_tree = max_tree or max(1, min(256, max(sizes)))
        self.max_len = max_len or top
        if page:
            used = [-(-max(int(n[0]), 1) // page) for n in self.lens]
            self.max_pages, self.n_pages = max(used) + 1, sum(used) + 2
            self.table = torch.full((self.B, self.max_pages), -1, dtype=torch.int32)
            order, at = torch.randperm(self.n_pages, generator=gen), 0
            for b, u in enumerate(used):
                self.table[b, :u] = order[at:at + u].int()
                at += u
            shape = (self.n_pages, hkv, page, D)
        else:
            self.cap = top + room
            shape = (self.B, hkv, self.cap, D)
        self.K, self.V = torch.randn(shape, generator=gen).mul_(key_scale).to(self.dt), torch.randn(shape, generator=gen).to(self.dt)
        n = self.n_tokens
        self.q = torch.randn((n, hkv * g, D), generator=gen).to(self.dt)
        self.k_tree = torch.randn((n, hkv, D), generator=gen).mul_(key_scale).to(self.dt)
        self.v_tree = torch.randn((n, hkv, D), generator=gen).to(self.dt)

    def slot(self, b, h, j):
        """Index of pair j of row (b, h) into the first three dimensions of K and V; None in a hole."""
        if not self.page:
            return b, h, j
        page = int(self.table[b, j // self.page])
        return (page, h, j % self.page) if 0 <= page < self.n_pages else None

    def cached(self, b, h):
        n = int(self.lens[b, h])
        if not self.page:
            return self.K[b, h, :n].double().numpy(), self.V[b, h, :n].double().numpy(), np.ones(n, bool)
        K, V, there = np.zeros((n, self.D)), np.zeros((n, self.D)), np.zeros(n, bool)
        for j in range(n):
            s = self.slot(b, h, j)
            if s is not None:
                K[j], V[j], there[j] = self.K[s].double().numpy(), self.V[s].double().numpy(), True
        return K, V, there

    def trees(self):
        for b, (_, parent) in enumerate(self.seqs):
            if 0 < len(parent) <= od.MOST_NODES:
                t0 = int(self.q_start[b])
                yield b, parent, slice(t0, t0 + len(parent))

    def reference(self, weight=UB):
        """weight: how far a bf16 weight may be off as it meets V, relative."""
        Hq = self.H * self.g
        ref = dict(out=np.full((self.n_tokens, Hq, self.D), 7.0), M=np.full((self.n_tokens, Hq), 7.0), L=np.full((self.n_tokens, Hq), 7.0))
        tol = {k: np.zeros_like(v) for k, v in ref.items()}
        for b, parent, tok in self.trees():
            rows = [self.cached(b, h) for h in range(self.H)]
            q, kt, vt = (x[tok].double().numpy() for x in (self.q, self.k_tree, self.v_tree))
            with np.errstate(invalid="ignore", over="ignore"):
                out, M, L, wv = od.attend(q, [r[0] for r in rows], [r[1] for r in rows], [r[2] for r in rows], kt, vt, parent, self.window, self.n_sink, self.scale)
            ref["out"][tok], ref["M"][tok], ref["L"][tok] = out, M, L
            # What fp32 allows.  A logit is a sum of D products (each fma rounds once: D u times the sum of magnitudes) and a few scalings; a
            # weight's exponent is off by its own logit's error and the reference's.  Sums of n weights: n u.  exp2: 2 steps.
            mag = np.zeros((len(parent), Hq))
            for h in range(self.H):
                heads = slice(h * self.g, (h + 1) * self.g)
                keys = np.nan_to_num(np.abs(np.concatenate([rows[h][0], kt[:, h]])), posinf=0)
                mag[:, heads] = (np.nan_to_num(np.abs(q[:, heads]), posinf=0) @ keys.T).max(axis=2, initial=0)
            n = int(self.lens[b].max()) + len(parent)
            d = (self.D + 4) * U * mag * abs(self.scale) / np.log(2.0) + U
            rel = 2 * np.log(2.0) * d + (2 * n + 8) * U
            half = U if self.dtype == "f32" else UB
            # bf16: every weight is rounded before it meets V, and the result once more (half a step); two terms of a weight are twice as many products to sum
            tol["out"][tok] = (rel[:, :, None] + (0 if self.dtype == "f32" else weight + n * U)) * wv + half * np.abs(out) * (1 + rel[:, :, None] + half) + 1e-30
            tol["M"][tok], tol["L"][tok] = d, rel * L
        return ref, tol

    def dev(self):
        import paper_2602_03203_amd as fk
        s = {k: getattr(self, k).cuda() for k in ("K", "V", "q_start", "parent", "q", "k_tree", "v_tree")}
        Hq = self.H * self.g
        if self.page:
            s["table"], s["len"] = self.table.cuda(), torch.tensor(self.lens[:, 0].copy()).cuda()
            s["desc"] = fk.PagedDesc(self.B, Hq, self.H, self.D, self.page, self.n_pages, self.max_pages, self.dtype)
            s["ws"] = fk.new_paged_tree_attn_workspace(s["desc"], self.n_tokens, self.max_tree, self.max_len)
        else:
            s["len"] = torch.tensor(self.lens).cuda()
            s["desc"] = fk.CacheDesc(self.B, Hq, self.H, self.D, self.cap, self.dtype)
            s["ws"] = fk.new_tree_attn_workspace(s["desc"], self.n_tokens, self.max_tree, self.max_len)
        s["out"] = torch.full_like(s["q"], 7.0)
        s["stats"] = torch.full((self.n_tokens, Hq, 2), 7.0, device="cuda")
        s["ws"][16384:] = 255   # behind the counters contents do not matter: NaN where floats lie
        return s

    def run(self, s, stats=True, stream=None):
        import paper_2602_03203_amd as fk
        tail = (s["k_tree"], s["v_tree"], s["parent"], s["q_start"], self.max_tree, self.max_len)
        end = (self.scale, s["out"], s["stats"] if stats else None, s["ws"])
        if self.page:
            fk.fk_paged_tree_attn(s["desc"], s["q"], s["K"], s["V"], s["table"], s["len"], *tail, self.window, self.n_sink, *end, stream=stream)
        else:
            fk.fk_tree_attn(s["desc"], s["q"], s["K"], s["V"], s["len"], *tail, *end, stream=stream)

    def check(self, s, ref, tol, what="", stats=True):
        got = dict(out=s["out"].double().cpu().numpy())
        if stats:
            got.update(M=s["stats"][..., 0].double().cpu().numpy(), L=s["stats"][..., 1].double().cpu().numpy())
        for k, x in got.items():
            r, e = ref[k], tol[k]
            if k == "M":   # (the largest of logits with a NaN among them is not defined)
                x, r, e = (np.where(np.isnan(ref["L"]), 0, v) for v in (x, r, e))
            same = (np.isnan(r) & np.isnan(x)) | (r == x)
            with np.errstate(invalid="ignore"):
                bad = ~same & ~(np.abs(x - r) <= e)
            if bad.any():
                i = np.unravel_index(np.argmax(np.where(bad, np.nan_to_num(np.abs(x - r), nan=1e30) / np.maximum(e, 1e-30), 0)), r.shape)
                raise AssertionError(f"{what} {k}: {bad.sum()} of {bad.size} off, worst at {i}: {x[i]!r}, not {r[i]!r} +- {e[i]!r}")

    def go(self, what="", stats=True):
        s = self.dev()
        self.run(s, stats)
        torch.cuda.synchronize()
        ref, tol = self.reference()
        self.check(s, ref, tol, what, stats)
        return s
