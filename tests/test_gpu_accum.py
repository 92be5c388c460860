"""Eviction by accumulated attention weight against the oracle: steps, compaction, whole runs out of a prompt's pages."""
import numpy as np
import pytest
import torch

from oracle import paged as op
from paged_util import U, UB, Case

pytestmark = pytest.mark.gpu


def _fk():
    import paper_2602_03203_amd as fk
    return fk


class Rows:
    def __init__(self, dtype, D, g, hkv, lens, cap, steps, seed=0, scale=None):
        gen = torch.Generator().manual_seed(seed)
        B = len(lens)
        dt = torch.float32 if dtype == "f32" else torch.bfloat16
        self.dtype, self.D, self.g, self.H, self.lens, self.cap, self.steps = dtype, D, g, hkv, lens, cap, steps
        self.scale = D ** -0.5 if scale is None else scale
        self.K, self.V = torch.randn((B, hkv, cap, D), generator=gen).to(dt), torch.randn((B, hkv, cap, D), generator=gen).to(dt)
        self.q = torch.randn((steps, B, hkv * g, D), generator=gen).to(dt)
        self.k, self.v = torch.randn((steps, B, hkv, D), generator=gen).to(dt), torch.randn((steps, B, hkv, D), generator=gen).to(dt)
        self.len = torch.tensor(lens, dtype=torch.int32)[:, None].repeat(1, hkv).contiguous()
        self.pos = torch.arange(cap, dtype=torch.int32).expand(B, hkv, cap).contiguous()
        self.acc = torch.rand((B, hkv, cap), generator=gen)
        self.pos_new = (torch.tensor(lens, dtype=torch.int32) + torch.arange(steps, dtype=torch.int32)[:, None]).contiguous()

    def dev(self):
        fk = _fk()
        s = {k: getattr(self, k).cuda() for k in ("K", "V", "q", "k", "v", "len", "pos", "acc", "pos_new")}
        s["desc"] = fk.CacheDesc(len(self.lens), self.H * self.g, self.H, self.D, self.cap, self.dtype)
        s["ws"] = fk.new_acc_workspace(s["desc"])
        s["ws"].fill_(255)
        s["out"] = torch.empty_like(s["q"])
        return s

    def run(self, s, max_len=None):
        fk = _fk()
        for t in range(self.steps):
            fk.fk_decode_step_acc(s["desc"], s["q"][t], s["K"], s["V"], s["pos"], s["len"], s["k"][t], s["v"][t], s["pos_new"][t],
                                  max_len or min(max(self.lens) + t + 1, self.cap), self.scale, s["acc"], s["out"][t], s["ws"])

    def check(self, s, what=""):
        K, V, acc = self.K.double().numpy().copy(), self.V.double().numpy().copy(), self.acc.double().numpy().copy()
        got_out, got_acc = s["out"].double().cpu().numpy(), s["acc"].double().cpu().numpy()
        tol = np.zeros_like(acc)
        n = list(self.lens)
        for t in range(self.steps):
            for b in range(len(n)):
                fresh = n[b] < self.cap
                if fresh:
                    K[b, :, n[b]], V[b, :, n[b]] = self.k[t, b].double().numpy(), self.v[t, b].double().numpy()
                    n[b] += 1
                m = n[b]
                q = self.q[t, b].double().numpy()[None]
                out, M, L, W = op.attend(q, K[b, :, :m], V[b, :, :m], np.ones(m, bool), m - 1, 0, 0, self.scale)
                acc[b, :, :m] = op.accumulate(acc[b, :, :m], W, self.H, m - 1 if fresh else m)
                # (as in paged_util: D products a logit, exponents off by their own and the reference's error, sums of m weights)
                mag = np.einsum("hgd,hnd->hgn", np.abs(q[0]).reshape(self.H, self.g, self.D), np.abs(K[b, :, :m])).max(initial=0)
                rel = 2 * np.log(2.0) * ((self.D + 4) * U * mag * abs(self.scale) / np.log(2.0) + U) + (2 * m + 8) * U
                wv = np.einsum("hgn,hnd->hgd", W[0].reshape(self.H, self.g, m), np.abs(V[b, :, :m])).reshape(self.H * self.g, self.D)
                half = U if self.dtype == "f32" else UB
                e = (rel + (0 if self.dtype == "f32" else UB)) * wv + half * np.abs(out[0]) * (1 + rel + half)
                bad = np.abs(got_out[t, b] - out[0]) > e
                assert not bad.any(), f"{what} step {t} sequence {b}: {bad.sum()} outputs off by up to {(np.abs(got_out[t, b] - out[0]) / np.maximum(e, 1e-30)).max()} of the bound"
                if fresh:
                    tol[b, :, m - 1] = 0
                tol[b, :, :m] += rel * op.received(W, self.H) + (self.g + 2) * U * np.abs(acc[b, :, :m])
        bad = np.abs(got_acc - acc) > tol
        assert not bad.any(), f"{what}: {bad.sum()} accumulated weights off, worst {np.abs(got_acc - acc).max()} at {np.argwhere(bad)[0]}"
        assert s["len"].cpu().tolist() == [[x] * self.H for x in n]
        for b in range(len(n)):
            assert torch.equal(s["K"][b].cpu().double(), torch.from_numpy(K[b])) and torch.equal(s["V"][b].cpu().double(), torch.from_numpy(V[b]))
            new = list(range(self.lens[b], n[b]))
            assert s["pos"][b, 0, self.lens[b]:n[b]].tolist() == new


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("g", [1, 2, 3, 4, 5, 6, 7, 8])
def test_steps(dtype, D, g):
    c = Rows(dtype, D, g, 2, [0, 1, 15, 31, 32, 63, 64, 200, 255, 319], 320, 3, seed=g)   # the last row fills up at the first step
    s = c.dev()
    c.run(s)
    c.check(s)


@pytest.mark.parametrize("dtype, D, g, hkv, lens", [("bf16", 128, 4, 8, [2100, 500]), ("bf16", 64, 8, 1, [3000]), ("f32", 128, 4, 2, [1500, 40]), ("bf16", 128, 1, 1, [5000]),
                                                    ("bf16", 128, 2, 4, [700] * 40), ("f32", 64, 1, 8, [900] * 18)])
def test_longer_rows(dtype, D, g, hkv, lens):
    c = Rows(dtype, D, g, hkv, lens, (max(lens) + 64) // 64 * 64, 2, seed=3)
    s = c.dev()
    c.run(s)
    c.check(s)


@pytest.mark.parametrize("dtype, D, g, n", [("bf16", 64, 4, 2334), ("bf16", 64, 4, 2400), ("bf16", 128, 8, 1150), ("bf16", 64, 7, 1330), ("f32", 64, 4, 1100), ("f32", 128, 5, 1860)])
def test_many_rows_around_what_lds_holds(dtype, D, g, n):
    """As many rows as take a workgroup each, with logits that do and do not fit LDS, and that grow beyond it from one step to the next."""
    c = Rows(dtype, D, g, 8, [n, n - 1, 1, 33, n, 1025, 500] * 3, n + 3, 3, seed=11)
    s = c.dev()
    c.run(s)
    c.check(s)


@pytest.mark.parametrize("g", [1, 4])
def test_many_splits(g):
    """One row over more splits than a wavefront has half lanes."""
    c = Rows("bf16", 64, g, 1, [9000], 9010, 2, seed=12)
    s = c.dev()
    c.run(s)
    c.check(s)


def test_hint_below_the_row_length():
    for dtype, D in (("bf16", 128), ("f32", 64)):
        c = Rows(dtype, D, 4, 2, [900, 33], 1024, 2, seed=4)
        s = c.dev()
        c.run(s, max_len=1)
        c.check(s)


def test_what_lies_behind_a_row_does_not_reach_it():
    for dtype, D in (("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)):
        c = Rows(dtype, D, 4, 1, [40, 300], 384, 2, seed=5)
        for b, n in enumerate(c.lens):
            c.K[b, :, n + 2:], c.V[b, :, n + 2:], c.acc[b, :, n:] = float("nan"), float("inf"), float("nan")
        s = c.dev()
        c.run(s)
        for b, n in enumerate(c.lens):
            assert torch.isnan(s["acc"][b, :, n + 2:]).all() and torch.isfinite(s["acc"][b, :, :n + 2]).all()
            assert torch.isfinite(s["out"][:, b].float()).all()


@pytest.mark.parametrize("dtype, D, lens", [("bf16", 128, [900, 2000]), ("f32", 64, [130, 140])])
def test_equal_bits_and_graph_replays(dtype, D, lens):
    c = Rows(dtype, D, 4, 2, lens, 2112, 3, seed=6)
    s = c.dev()
    c.run(s)
    want = {k: s[k].clone() for k in ("out", "acc", "len")}
    start = {k: getattr(c, k).cuda() for k in ("len", "acc")}
    s["len"].copy_(start["len"])
    s["acc"].copy_(start["acc"])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.run(s)
    for i in range(3):
        s["len"].copy_(start["len"])
        s["acc"].copy_(start["acc"])
        s["out"].zero_()
        g.replay()
        torch.cuda.synchronize()
        for k, x in want.items():
            assert torch.equal(x.view(torch.uint8), s[k].view(torch.uint8)), (i, k)
        s["ws"].fill_(i)


@pytest.mark.parametrize("dtype, D", [("bf16", 128), ("f32", 64), ("bf16", 64)])
@pytest.mark.parametrize("budget, recent, n", [(64, 16, 80), (512, 32, 700), (600, 128, 1500), (2048, 128, 2176), (100, 0, 90)])
def test_compact_moves_the_weights(dtype, D, budget, recent, n):
    fk = _fk()
    c = Rows(dtype, D, 1, 2, [n, max(1, n // 2), budget], max(n, budget) + 7, 1, seed=7)
    s = c.dev()
    keep = torch.zeros((3, 2, budget), dtype=torch.int32, device="cuda")
    fk.fk_select_keep(s["desc"], s["acc"], s["pos"], s["len"], max(n, budget), budget, recent, keep)
    other = {k: s[k].clone() for k in ("K", "V", "pos", "len")}
    before = s["acc"].clone()
    fk.fk_compact_acc(s["desc"], s["K"], s["V"], s["pos"], s["acc"], s["len"], keep, budget)
    fk.fk_compact(s["desc"], other["K"], other["V"], other["pos"], other["len"], keep, budget)
    for k, x in other.items():
        assert torch.equal(x.view(torch.uint8), s[k].view(torch.uint8)), k
    want = before.clone()
    for b, m in enumerate(c.lens):
        if m > budget:
            want[b, :, :budget] = before[b].gather(1, keep[b].long())
    assert torch.equal(want, s["acc"])


@pytest.mark.parametrize("dtype, D, window", [("bf16", 128, 0), ("f32", 64, 0), ("bf16", 64, 40)])
def test_from_a_prompt_to_evictions(dtype, D, window):
    """A whole run: prompts in chunks into pages with their weights, compression into rows, steps with evictions, every stage against
    the oracle on what the device selected."""
    fk = _fk()
    g, H, page, budget, recent, L = 4, 2, 16, 64, 8, 16
    lens, chunk = [150, 101, 40], 64
    B = len(lens)
    gen = torch.Generator().manual_seed(19)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    rnd = lambda *shape: torch.randn(shape, generator=gen).to(dt)   # noqa: E731
    full = [(rnd(n, H * g, D), rnd(n, H, D), rnd(n, H, D)) for n in lens]
    c = Case(dtype, D, g, H, page, [(n, 0) for n in lens], window, 2, seed=20)
    s = c.dev()
    s["acc"].fill_(float("nan"))      # every slot starts with its chunk
    cap = c.max_pages * page
    want = [np.zeros((H, n)) for n in lens]
    tol = [np.zeros((H, n)) for n in lens]
    scale = D ** -0.5
    for at in range(0, max(lens), chunk):
        part = [(min(at, n), min(at + chunk, n)) for n in lens]
        q, k, v = (torch.cat([x[i][a:e] for x, (a, e) in zip(full, part)]).cuda() for i in range(3))
        starts = torch.tensor(np.concatenate([[0], np.cumsum([e - a for a, e in part])]), dtype=torch.int32, device="cuda")
        kv = torch.tensor([e for _, e in part], dtype=torch.int32, device="cuda")
        out, stats = torch.empty_like(q), torch.empty((q.shape[0], H * g, 2), device="cuda")
        ws, wws = (f(s["desc"], q.shape[0], chunk, max(lens)) for f in (fk.new_paged_attn_workspace, fk.new_paged_weights_workspace))
        view = (s["table"], kv, starts)
        fk.fk_paged_append(s["desc"], s["K"], s["V"], *view, k, v)
        fk.fk_paged_attn(s["desc"], q, s["K"], s["V"], *view, chunk, max(lens), window, 2, scale, out, stats, ws)
        fk.fk_paged_weights(s["desc"], q, s["K"], *view, chunk, max(lens), window, 2, scale, stats, s["acc"], wws)
        for b, (a, e) in enumerate(part):
            if a == e:
                continue
            o, _, _, W = op.attend(full[b][0][a:e].double().numpy(), full[b][1][:e].transpose(0, 1).double().numpy(),
                                   full[b][2][:e].transpose(0, 1).double().numpy(), np.ones(e, bool), a, window, 2, scale)
            got = out[int(starts[b]):int(starts[b + 1])].double().cpu().numpy()
            lim = (2e-4 if dtype == "f32" else 2 * UB + 1e-3) * np.einsum("thn,hnd->thd", W, np.repeat(np.abs(full[b][2][:e].transpose(0, 1).double().numpy()), g, 0)) + UB * np.abs(o) * (dtype != "f32")
            assert (np.abs(got - o) <= lim).all()
            want[b][:, :e] = op.accumulate(want[b][:, :e], W, H, a)
            tol[b][:, :e] += 1e-3 * op.received(W, H) + 1e-6
    acc = s["acc"].cpu().double().numpy()
    for b, n in enumerate(lens):
        assert (np.abs(acc[b, :, :n] - want[b]) <= tol[b]).all() and np.isnan(acc[b, :, n:]).all()
    # into the rows
    rows = fk.CacheDesc(B, H * g, H, D, 128, dtype)
    row_len = torch.tensor(lens, dtype=torch.int32, device="cuda")[:, None].repeat(1, H).contiguous()
    keep = torch.zeros((B, H, budget), dtype=torch.int32, device="cuda")
    fk.fk_select_keep(fk.CacheDesc(B, H * g, H, D, cap, dtype), s["acc"], None, row_len, max(lens), budget, recent, keep)
    Kr, Vr = (torch.zeros((B, H, 128, D), dtype=dt, device="cuda") for _ in range(2))
    pos, ln, acc_r = torch.zeros((B, H, 128), dtype=torch.int32, device="cuda"), torch.zeros((B, H), dtype=torch.int32, device="cuda"), fk.new_acc(rows)
    kv = torch.tensor(lens, dtype=torch.int32, device="cuda")
    fk.fk_paged_compress(s["desc"], s["K"], s["V"], s["table"], kv, s["acc"], keep, budget, rows, Kr, Vr, pos, ln, acc_r)
    m = [min(n, budget) for n in lens]
    assert ln.tolist() == [[x] * H for x in m]
    state = [[[full[b][1][:, h].double().numpy()[pos[b, h, :m[b]].cpu().numpy()], full[b][2][:, h].double().numpy()[pos[b, h, :m[b]].cpu().numpy()],
               acc[b, h][pos[b, h, :m[b]].cpu().numpy()]] for h in range(H)] for b in range(B)]
    ws = fk.new_acc_workspace(rows)
    for t in range(2 * L):
        q, k, v = rnd(B, H * g, D), rnd(B, H, D), rnd(B, H, D)
        out = torch.empty((B, H * g, D), dtype=dt, device="cuda")
        fk.fk_decode_step_acc(rows, q.cuda(), Kr, Vr, pos, ln, k.cuda(), v.cuda(), torch.tensor([n + t for n in lens], dtype=torch.int32, device="cuda"),
                              128, scale, acc_r, out, ws)
        for b in range(B):
            for h in range(H):
                K, V, A = state[b][h]
                K, V, A = np.vstack([K, k[b, h].double().numpy()]), np.vstack([V, v[b, h].double().numpy()]), np.append(A, 0.0)
                o, _, _, W = op.attend(q[b, h * g:(h + 1) * g].double().numpy()[None], K[None], V[None], np.ones(len(A), bool), len(A) - 1, 0, 0, scale)
                assert np.abs(out[b, h * g:(h + 1) * g].double().cpu().numpy() - o[0]).max() <= (1e-4 if dtype == "f32" else 4 * UB) * max(1, np.abs(V).max())
                state[b][h] = [K, V, A + W.sum(axis=(0, 1))]
        if (t + 1) % L == 0:
            fk.fk_select_keep(rows, acc_r, pos, ln, 128, budget, recent, keep)
            counts = ln.cpu().tolist()
            fk.fk_compact_acc(rows, Kr, Vr, pos, acc_r, ln, keep, budget)
            kp = keep.cpu().numpy()
            for b in range(B):
                for h in range(H):
                    if counts[b][h] > budget:
                        state[b][h] = [x[kp[b, h]] for x in state[b][h]]
                    x = acc_r[b, h, :len(state[b][h][2])].double().cpu().numpy()
                    assert np.abs(x - state[b][h][2]).max() <= 1e-3 * (t + 1)
                    assert np.array_equal(Kr[b, h, :len(x)].double().cpu().numpy(), state[b][h][0])
