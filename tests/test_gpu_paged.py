"""The paged prompt cache against the oracle: appends, attention of chunks, windows with sinks, accumulated weights, compression."""
import numpy as np
import pytest
import torch

from paged_util import Case

pytestmark = pytest.mark.gpu


def _fk():
    import paper_2602_03203_amd as fk
    return fk


def _go(case, what="", weights=True):
    s = case.dev()
    case.run(s, weights=weights)
    torch.cuda.synchronize()
    K, V = case.appended()
    assert torch.equal(s["K"].cpu().view(torch.uint8), K.view(torch.uint8)) and torch.equal(s["V"].cpu().view(torch.uint8), V.view(torch.uint8)), f"{what}: the pool differs"
    ref, tol = case.reference(K, V)
    case.check(s, ref, tol, weights, what)
    return s


SINGLE = [(1, 1), (2, 1), (15, 1), (16, 1), (17, 1), (0, 0), (31, 1), (32, 1), (33, 1), (63, 1), (64, 1), (65, 1), (127, 1), (128, 1), (129, 1), (300, 1), (77, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("g, hkv, page", [(1, 2, 16), (3, 1, 32), (4, 2, 64), (8, 1, 16), (7, 1, 128)])
def test_single_tokens(dtype, D, g, hkv, page):
    _go(Case(dtype, D, g, hkv, page, SINGLE, seed=g))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("g, chunks", [(1, [(5, 5), (40, 17), (300, 129)]), (4, [(2, 2), (70, 4), (70, 5), (200, 33)]), (8, [(64, 64), (130, 2), (257, 3)]),
                                       (5, [(90, 90), (33, 1), (500, 26)]), (2, [(128, 128), (129, 64), (1000, 65)]), (7, [(37, 18), (37, 19), (64, 37)])])
def test_chunks(dtype, D, g, chunks):
    _go(Case(dtype, D, g, 2, 16, chunks, seed=g))


@pytest.mark.parametrize("dtype, D, g, page, chunks", [("bf16", 128, 4, 64, [(1500, 200)]), ("bf16", 64, 4, 16, [(1100, 300), (1025, 1)]), ("bf16", 128, 1, 256, [(700, 513)]),
                                                       ("f32", 128, 4, 32, [(900, 70)]), ("f32", 64, 8, 16, [(600, 65), (601, 1)]), ("bf16", 128, 8, 1024, [(1030, 40), (1024, 1), (1023, 7)])])
def test_longer_chunks(dtype, D, g, page, chunks):
    _go(Case(dtype, D, g, 1, page, chunks, seed=3))


@pytest.mark.parametrize("dtype, D", [("f32", 64), ("bf16", 64), ("bf16", 128), ("f32", 128)])
@pytest.mark.parametrize("window, sink", [(1, 0), (1, 1), (7, 0), (16, 4), (64, 4), (100, 70), (33, 200), (5000, 4)])
def test_windows_and_sinks(dtype, D, window, sink):
    _go(Case(dtype, D, 4, 1, 16, [(1, 1), (3, 1), (64, 1), (65, 1), (300, 1), (260, 100), (90, 90), (333, 33), (20, 2)], window, sink, seed=window))


@pytest.mark.parametrize("dtype, D", [("bf16", 128), ("f32", 64), ("bf16", 64)])
@pytest.mark.parametrize("window", [0, 20])
def test_holes(dtype, D, window):
    """Pages that are not there: nothing is stored in them and nobody sees their pairs; a query with holes alone sees nothing."""
    c = Case(dtype, D, 4, 2, 16, [(100, 1), (100, 40), (16, 16), (200, 3), (5, 1)], window, 2, seed=5)
    c.table[0, 2] = c.n_pages
    c.table[0, 6] = -7
    c.table[1, 5], c.table[1, 0] = -1, 1 << 30
    c.table[2, 0] = -1
    c.table[3, 3:9] = -1
    c.table[4, 0] = -(1 << 31)
    _go(c)


@pytest.mark.parametrize("dtype, D", [("bf16", 128), ("f32", 64)])
def test_tokens_before_the_first_position(dtype, D):
    """A chunk longer than its sequence: its first tokens see nothing and are not stored."""
    _go(Case(dtype, D, 4, 1, 16, [(3, 10), (0, 4), (40, 45), (33, 1)], seed=6))


def test_tokens_outside_of_all_chunks_are_not_touched():
    for dtype, D, chunks in (("bf16", 128, [(40, 3), (50, 20)]), ("f32", 64, [(33, 1), (20, 1)])):
        _go(Case(dtype, D, 4, 1, 16, chunks, seed=7, before=5, behind=9))


@pytest.mark.parametrize("dtype, D", [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("bad", [float("inf"), float("nan"), -float("inf")])
def test_hidden_values_stay_hidden(dtype, D, bad):
    """Infinities and NaN that a query does not see - behind the sequence, outside of the window, later tokens of the chunk - do not reach it;
    those that it sees do."""
    c = Case(dtype, D, 4, 2, 16, [(37, 1), (300, 1), (100, 40), (290, 2), (70, 70)], 48, 3, seed=8)
    K, V = c.appended()
    for b, (n, m) in enumerate(c.chunks):   # behind the end, in the last page and in the spare ones
        page = int(c.table[b, (n - 1) // 16])
        if n % 16:
            c.K[page, :, n % 16:], c.V[page, :, n % 16:] = bad, bad
    used = set(c.table[c.table >= 0].tolist())
    for page in set(range(c.n_pages)) - used:
        c.K[page], c.V[page] = bad, bad
    c.K[int(c.table[1, 100 // 16]), :, 100 % 16] = bad      # outside of the window
    c.V[int(c.table[1, 100 // 16]), :, 100 % 16] = bad
    t = int(c.q_start[2]) + 25                                # one value of a later token
    c.v_new[t, 0, 5] = bad
    c.k_new[int(c.q_start[4]) + 66, 1, 3] = bad
    c.v_new[int(c.q_start[4]) + 3, 1, D - 1] = bad            # seen by 48 tokens, then outside of the window
    c.v_new[int(c.q_start[3]) + 1, 0, 0] = bad                # the second of two tokens
    _go(c, weights=False)


@pytest.mark.parametrize("dtype, D", [("bf16", 128), ("f32", 64)])
def test_hidden_values_and_weights(dtype, D):
    c = Case(dtype, D, 4, 1, 16, [(37, 5), (100, 1)], 20, 2, seed=9)
    c.K[int(c.table[0, 2]), :, 5:] = float("nan")
    c.K[int(c.table[1, 3]), :, 2] = float("inf")     # outside of the window
    s = c.dev()
    c.run(s)
    ref, tol = c.reference()
    c.check(s, ref, tol)


@pytest.mark.parametrize("dtype, D, scale", [("bf16", 128, -0.1), ("f32", 64, -0.2), ("bf16", 64, 0.0), ("f32", 128, 0.0), ("bf16", 128, 3.0), ("bf16", 64, -0.0)])
def test_scales(dtype, D, scale):
    _go(Case(dtype, D, 4, 1, 16, [(60, 1), (150, 20)], scale=scale, seed=10))


@pytest.mark.parametrize("dtype, D", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_huge_logits(dtype, D):
    """Logits whose rounding is beyond an exponential's range: the largest key takes all."""
    c = Case(dtype, D, 4, 1, 16, [(200, 1), (150, 40)], scale=1e12, seed=11)
    K, V = c.appended()
    ref, _ = c.reference(K, V)
    s = c.dev()
    c.run(s)
    out = s["out"].double().cpu().numpy()
    tol = 2.0 ** -8 if dtype == "bf16" else 1e-6
    assert np.isfinite(out).all() and (np.abs(out - ref["out"]) <= tol * np.abs(ref["out"]) + 1e-30).all()
    acc = s["acc"].double().cpu().numpy()
    assert (np.abs(acc - ref["acc"]) <= 1e-4).all()


def test_hints_only_size_the_launch():
    """max_chunk and max_len below what there is: the same results."""
    for dtype, D in (("bf16", 128), ("f32", 64)):
        c = Case(dtype, D, 4, 2, 16, [(500, 60), (300, 1), (40, 40)], seed=12)
        c.max_chunk = c.max_len = 1
        _go(c)


def test_stats_are_optional_and_scratch_contents_do_not_matter():
    c = Case("bf16", 128, 4, 2, 16, [(700, 1), (300, 50)], seed=13)
    s = _go(c)
    want = s["out"].clone()
    s["out"].fill_(7)
    s["ws"].fill_(170)
    c.run(s, weights=False, stats=False)
    assert torch.equal(want.view(torch.int16), s["out"].view(torch.int16))


@pytest.mark.parametrize("dtype, D", [("bf16", 128), ("f32", 64), ("bf16", 64)])
def test_equal_calls_give_equal_bits(dtype, D):
    c = Case(dtype, D, 4, 2, 32, [(2000, 1), (900, 200), (1500, 3)], seed=14)
    s = c.dev()
    c.run(s)
    want = [s[k].clone() for k in ("out", "stats", "acc")]
    for _ in range(3):
        s["acc"].copy_(c.acc)
        c.run(s)
        for x, k in zip(want, ("out", "stats", "acc")):
            assert torch.equal(x.view(torch.uint8), s[k].view(torch.uint8)), k


def test_shared_prefix_pages():
    """Two sequences whose first pages are the same ones."""
    c = Case("bf16", 128, 4, 1, 16, [(100, 20), (90, 5)], seed=15)
    c.table[1, :4] = c.table[0, :4]
    _go(c)


def test_other_stream_and_graph():
    """On a stream of its own, and captured: every replay gives the eager results, also with another graph on the same workspace between."""
    fk = _fk()
    c, c2 = Case("bf16", 128, 4, 2, 64, [(900, 1), (1800, 1), (300, 64)], seed=16), Case("bf16", 128, 4, 2, 64, [(700, 1), (1300, 30), (64, 64)], seed=17)
    s, s2 = c.dev(), c2.dev()
    big = max(s["ws"].numel(), s2["ws"].numel())
    s["ws"] = s2["ws"] = torch.empty(big, dtype=torch.uint8, device="cuda")
    wbig = max(s["wws"].numel(), s2["wws"].numel())
    s["wws"] = s2["wws"] = torch.empty(wbig, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.run(s)
        c2.run(s2)
    side.synchronize()
    want = {k: (s[k].clone(), s2[k].clone()) for k in ("out", "stats", "acc")}
    graphs = []
    for cc, ss in ((c, s), (c2, s2)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            cc.run(ss)
        graphs.append(g)
    for i in range(4):
        for ss, cc in ((s, c), (s2, c2)):
            ss["out"].fill_(0)
            ss["stats"].fill_(0)
            ss["acc"].copy_(cc.acc)
        graphs[i % 2].replay()
        graphs[1 - i % 2].replay()
        torch.cuda.synchronize()
        for k, (a, b) in want.items():
            assert torch.equal(a.view(torch.uint8), s[k].view(torch.uint8)) and torch.equal(b.view(torch.uint8), s2[k].view(torch.uint8)), (i, k)
        s["ws"].fill_(i)
    assert fk is not None


@pytest.mark.parametrize("dtype, D", [("bf16", 128), ("f32", 64)])
def test_pool_beyond_4_gib(dtype, D):
    """Pages at the far end of a pool of more than 2^32 bytes."""
    c = Case(dtype, D, 4, 2, 64, [(500, 1), (300, 40)], seed=18)
    ref, tol = c.reference()
    page_bytes = 2 * 64 * D * (2 if dtype == "bf16" else 4)
    far = (1 << 32) // page_bytes + 50
    s = c.dev()
    for k in ("K", "V"):
        big = torch.empty((far + c.n_pages, *s[k].shape[1:]), dtype=s[k].dtype, device="cuda")
        big[far:] = s[k]
        s[k] = big
    s["table"] = torch.where(s["table"] >= 0, s["table"] + far, s["table"])
    s["desc"].n_pages += far
    c.run(s)
    c.check(s, ref, tol)
    del s
    torch.cuda.empty_cache()


# ---- compression ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype, D", [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("budget, cap", [(1, 64), (64, 64), (65, 200), (130, 192)])
@pytest.mark.parametrize("with_acc", [True, False])
def test_compress(dtype, D, budget, cap, with_acc):
    fk = _fk()
    lens = [300, 130, 64, 65, 1, 0, 129]
    c = Case(dtype, D, 2, 2, 16, [(n, 0) for n in lens], seed=budget)
    if budget == 130:
        c.table[0, 3] = -1     # a hole: its slots stay as they are
    s = c.dev()
    B, H = len(lens), 2
    row_len = c.kv_len.repeat_interleave(H).reshape(B, H).contiguous().cuda()
    keep = torch.full((B, H, budget), -9, dtype=torch.int32, device="cuda")
    long, rows = fk.CacheDesc(B, 4, H, D, c.max_pages * 16, dtype), fk.CacheDesc(B, 4, H, D, cap, dtype)
    fk.fk_select_keep(long, s["acc"], None, row_len, max(lens), budget, min(16, budget), keep)
    Kr, Vr = (torch.full((B, H, cap, D), 3.0, dtype=s["K"].dtype, device="cuda") for _ in range(2))
    pos, ln = torch.full((B, H, cap), -5, dtype=torch.int32, device="cuda"), torch.zeros((B, H), dtype=torch.int32, device="cuda")
    acc_r = torch.full((B, H, cap), 4.0, device="cuda")
    fk.fk_paged_compress(s["desc"], s["K"], s["V"], s["table"], s["kv_len"], s["acc"] if with_acc else None, keep, budget, rows, Kr, Vr, pos, ln,
                         acc_r if with_acc else None)
    kp, Kc, Vc, pc, ac = keep.cpu(), Kr.cpu(), Vr.cpu(), pos.cpu(), acc_r.cpu()
    for b, n in enumerate(lens):
        assert ln[b].tolist() == [min(n, budget)] * H
        for h in range(H):
            for j in range(cap):
                p = int(kp[b, h, j]) if j < min(n, budget) else -1
                page = int(c.table[b, p // 16]) if p >= 0 else -1
                if page < 0:
                    assert (Kc[b, h, j] == 3).all() and (Vc[b, h, j] == 3).all() and pc[b, h, j] == -5 and ac[b, h, j] == 4
                    continue
                assert torch.equal(Kc[b, h, j], c.K[page, h, p % 16]) and torch.equal(Vc[b, h, j], c.V[page, h, p % 16])
                assert pc[b, h, j] == p and ac[b, h, j] == (c.acc[b, h, p] if with_acc else 4)


def test_compress_ignores_indices_outside_of_the_sequence():
    fk = _fk()
    c = Case("bf16", 128, 1, 1, 16, [(40, 0)], seed=1)
    s = c.dev()
    rows = fk.CacheDesc(1, 1, 1, 128, 64, "bf16")
    keep = torch.tensor([[[3, -1, 39, 40, 1 << 30, -(1 << 31), 7, 8]]], dtype=torch.int32, device="cuda")
    Kr = torch.full((1, 1, 64, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    Vr, pos, ln = Kr.clone(), torch.full((1, 1, 64), -5, dtype=torch.int32, device="cuda"), torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    fk.fk_paged_compress(s["desc"], s["K"], s["V"], s["table"], s["kv_len"], None, keep, 8, rows, Kr, Vr, pos, ln, None)
    assert pos[0, 0, :8].tolist() == [3, -5, 39, -5, -5, -5, 7, 8] and int(ln) == 8
    assert (Kr[0, 0, [1, 3, 4, 5]] == 3).all() and torch.equal(Kr[0, 0, 2].cpu(), c.K[int(c.table[0, 2]), 0, 7])
