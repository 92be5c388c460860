"""Cases of the paged prompt cache: seeded inputs, the oracle's results and the error that the arithmetic allows."""
from __future__ import annotations

import numpy as np
import torch

from oracle import paged as op

U = 2.0 ** -24       # half a step of fp32, relative
UB = 2.0 ** -8       # half a step of bf16, relative


class Case:
    """chunks: [(kv_len, chunk), ...] one per sequence.  Host tensors, bf16 values exact in float64."""

    def __init__(self, dtype, D, g, hkv, page, chunks, window=0, n_sink=0, scale=None, seed=0, before=0, behind=0, spare=2, key_scale=1.0, room=0):
        gen = torch.Generator().manual_seed(seed)
        self.dtype, self.D, self.g, self.H, self.page, self.chunks = dtype, D, g, hkv, page, chunks
        self.window, self.n_sink, self.scale = window, n_sink, D ** -0.5 if scale is None else scale
        self.dt = torch.float32 if dtype == "f32" else torch.bfloat16
        used = [-(-max(n, 1) // page) for n, _ in chunks]
        self.max_pages, self.n_pages = max(used) + 1 + room, sum(used) + spare   # room: for sequences this much longer, which max_len then covers
        self.table = torch.full((len(chunks), self.max_pages), -1, dtype=torch.int32)
        order = torch.randperm(self.n_pages, generator=gen)
        at = 0
        for b, u in enumerate(used):
            self.table[b, :u] = order[at:at + u].int()
            at += u
        shape = (self.n_pages, hkv, page, D)
        self.K, self.V = torch.randn(shape, generator=gen).mul_(key_scale).to(self.dt), torch.randn(shape, generator=gen).to(self.dt)
        self.kv_len = torch.tensor([n for n, _ in chunks], dtype=torch.int32)
        starts = before + np.concatenate([[0], np.cumsum([c for _, c in chunks])])
        self.q_start = torch.tensor(starts, dtype=torch.int32)
        self.n_tokens = int(starts[-1]) + behind
        self.q = torch.randn((self.n_tokens, hkv * g, D), generator=gen).to(self.dt)
        self.k_new = torch.randn((self.n_tokens, hkv, D), generator=gen).mul_(key_scale).to(self.dt)
        self.v_new = torch.randn((self.n_tokens, hkv, D), generator=gen).to(self.dt)
        self.acc = torch.rand((len(chunks), hkv, self.max_pages * page), generator=gen)
        self.max_chunk, self.max_len = max(1, max(c for _, c in chunks)), max(1, max(n for n, _ in chunks)) if room == 0 else self.max_pages * page

    def appended(self):
        """The pools after the append, position by position."""
        K, V = self.K.clone(), self.V.clone()
        for b, (n, c) in enumerate(self.chunks):
            for i in range(c):
                p, t = n - c + i, int(self.q_start[b]) + i
                if p < 0:
                    continue
                page = int(self.table[b, p // self.page])
                if 0 <= page < self.n_pages:
                    K[page, :, p % self.page], V[page, :, p % self.page] = self.k_new[t], self.v_new[t]
        return K, V

    def reference(self, K=None, V=None):
        """out, stats, acc of the oracle and their tolerances; tokens outside of all chunks: NaN in out (not compared)."""
        if K is None:
            K, V = self.appended()
        K, V, q = K.double().numpy(), V.double().numpy(), self.q.double().numpy()
        Hq = self.H * self.g
        ref = dict(out=np.full((self.n_tokens, Hq, self.D), np.nan), M=np.full((self.n_tokens, Hq), np.nan), L=np.full((self.n_tokens, Hq), np.nan),
                   acc=self.acc.double().numpy().copy())
        tol = {k: np.zeros_like(v) for k, v in ref.items()}
        for b, (n, c) in enumerate(self.chunks):
            if c == 0:
                continue
            t0, first = int(self.q_start[b]), n - c
            kk, present = op.pairs(K, self.table[b].numpy(), n)
            vv, _ = op.pairs(V, self.table[b].numpy(), n)
            qq = q[t0:t0 + c]
            with np.errstate(invalid="ignore", over="ignore"):
                out, M, L, W = op.attend(qq, kk, vv, present, first, self.window, self.n_sink, self.scale)
            tok = slice(t0, t0 + c)
            ref["out"][tok], ref["M"][tok], ref["L"][tok] = out, M, L
            f0 = max(first, 0)
            old = present[:f0]
            new = op.accumulate(ref["acc"][b, :, :n], W, self.H, f0)
            # What fp32 allows.  A logit is a sum of D products (each fma rounds once: D u times the sum of magnitudes) and a few scalings; a
            # weight's exponent is off by its own logit's error and the reference's.  Sums of n weights: n u.  exp2: 2 steps.
            fin_q, fin_k = np.nan_to_num(np.abs(qq), posinf=0), np.nan_to_num(np.abs(kk), posinf=0)
            mag = np.einsum("thgd,hnd->thgn", fin_q.reshape(c, self.H, self.g, self.D), fin_k).max(axis=3, initial=0).reshape(c, Hq) if n else np.zeros((c, Hq))
            d = (self.D + 4) * U * mag * abs(self.scale) / np.log(2.0) + U
            rel = 2 * np.log(2.0) * d + (2 * n + 8) * U
            wv = np.einsum("thgn,hnd->thgd", np.nan_to_num(W).reshape(c, self.H, self.g, n), np.nan_to_num(np.abs(vv), posinf=0)).reshape(c, Hq, self.D)
            half = U if self.dtype == "f32" else UB
            # bf16: every weight is rounded before it meets V (half a step), and the result once more
            tol["out"][tok] = (rel[:, :, None] + (0 if self.dtype == "f32" else UB)) * wv + half * np.abs(out) * (1 + rel[:, :, None] + half) + 1e-30
            tol["M"][tok], tol["L"][tok] = d, rel * L
            tol["acc"][b, :, :n] = rel.max(initial=0) * op.received(W, self.H) + (c * self.g + 2) * U * np.abs(new)
            ref["acc"][b, :, :n] = new
            assert old.size == f0
        return ref, tol

    def dev(self):
        import paper_2602_03203_amd as fk
        s = {k: getattr(self, k).cuda() for k in ("K", "V", "table", "kv_len", "q_start", "q", "k_new", "v_new", "acc")}
        s["desc"] = fk.PagedDesc(len(self.chunks), self.H * self.g, self.H, self.D, self.page, self.n_pages, self.max_pages, self.dtype)
        s["out"] = torch.full_like(s["q"], 7.0)
        s["stats"] = torch.full((self.n_tokens, self.H * self.g, 2), 7.0, device="cuda")
        s["ws"] = fk.new_paged_attn_workspace(s["desc"], self.n_tokens, self.max_chunk, self.max_len)
        s["wws"] = fk.new_paged_weights_workspace(s["desc"], self.n_tokens, self.max_chunk, self.max_len)
        s["ws"].fill_(255)   # contents do not matter: NaN where floats lie
        s["wws"].fill_(255)
        return s

    def run(self, s, append=True, weights=True, stats=True):
        import paper_2602_03203_amd as fk
        view = (s["table"], s["kv_len"], s["q_start"])
        if append:
            fk.fk_paged_append(s["desc"], s["K"], s["V"], *view, s["k_new"], s["v_new"])
        fk.fk_paged_attn(s["desc"], s["q"], s["K"], s["V"], *view, self.max_chunk, self.max_len, self.window, self.n_sink, self.scale, s["out"],
                         s["stats"] if stats else None, s["ws"])
        if weights:
            fk.fk_paged_weights(s["desc"], s["q"], s["K"], *view, self.max_chunk, self.max_len, self.window, self.n_sink, self.scale, s["stats"],
                                s["acc"], s["wws"])

    def check(self, s, ref, tol, weights=True, what=""):
        got = dict(out=s["out"].double().cpu().numpy(), M=s["stats"][..., 0].double().cpu().numpy(), L=s["stats"][..., 1].double().cpu().numpy())
        if weights:
            got["acc"] = s["acc"].double().cpu().numpy()
        inside = np.zeros(self.n_tokens, bool)
        for b, (_, c) in enumerate(self.chunks):
            inside[int(self.q_start[b]):int(self.q_start[b]) + c] = True
        for k in ("out", "M", "L"):
            assert (got[k][~inside] == 7.0).all(), f"{what} {k}: tokens outside of all chunks were touched"
        for k, x in got.items():
            r, e = (ref[k], tol[k]) if k == "acc" else (ref[k][inside], tol[k][inside])
            x = x if k == "acc" else x[inside]
            if k == "M":   # (the largest of logits with a NaN among them is not defined)
                x, r, e = (np.where(np.isnan(ref["L"][inside]), 0, v) for v in (x, r, e))
            same = (np.isnan(r) & np.isnan(x)) | (r == x)
            with np.errstate(invalid="ignore"):
                bad = ~same & ~(np.abs(x - r) <= e)
            if bad.any():
                i = np.unravel_index(np.argmax(np.where(bad, np.nan_to_num(np.abs(x - r), nan=1e30) / np.maximum(e, 1e-30), 0)), r.shape)
                raise AssertionError(f"{what} {k}: {bad.sum()} of {bad.size} off, worst at {i}: {x[i]!r}, not {r[i]!r} +- {e[i]!r}")
