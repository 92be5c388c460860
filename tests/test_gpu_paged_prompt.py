"""The kernel for chunks of many query rows, alone and beside single tokens, against the oracle.  Calls of little work are the other kernel's, by their
length bound: these have tables, and a bound, for sequences much longer than theirs."""
import copy
import subprocess
import sys

import numpy as np
import pytest
import torch

from paged_util import Case

pytestmark = pytest.mark.gpu

TYPES = [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)]


def _case(dtype, D, g, hkv, page, chunks, *args, **kw):
    tokens = sum(c for _, c in chunks)
    room = (1 << 21) // (max(1, tokens * g // 16) * hkv) // page + 1
    return Case(dtype, D, g, hkv, page, chunks, *args, room=room, **kw)


def _go(case, what="", weights=False):
    s = case.dev()
    case.run(s, weights=weights)
    torch.cuda.synchronize()
    K, V = case.appended()
    ref, tol = case.reference(K, V)
    case.check(s, ref, tol, weights, what)
    return s


@pytest.mark.parametrize("dtype, D", TYPES)
@pytest.mark.parametrize("g, chunks", [(1, [(17, 17), (40, 17), (300, 129)]), (4, [(5, 5), (70, 5), (200, 33)]), (8, [(64, 64), (130, 3), (257, 3)]),
                                       (5, [(90, 90), (33, 4), (500, 26)]), (2, [(128, 128), (129, 64), (1000, 65)]), (7, [(37, 18), (37, 19), (64, 37)])])
def test_chunks(dtype, D, g, chunks):
    _go(_case(dtype, D, g, 2, 16, chunks, seed=g), weights=True)


@pytest.mark.parametrize("dtype, D", TYPES)
@pytest.mark.parametrize("page", [16, 32, 64, 256])
def test_beside_single_tokens(dtype, D, page):
    _go(_case(dtype, D, 4, 2, page, [(1, 1), (150, 40), (300, 1), (0, 0), (64, 64), (129, 2), (77, 0), (90, 4), (513, 5), (40, 1)], seed=page))


@pytest.mark.parametrize("dtype, D", TYPES)
@pytest.mark.parametrize("g, chunks", [(4, [(2600, 20)]), (1, [(1700, 130), (1025, 1)]), (8, [(3000, 1), (2111, 17), (40, 3), (1050, 1)])])
def test_splits(dtype, D, g, chunks):
    """Pairs enough for several splits, of both kinds."""
    _go(_case(dtype, D, g, 1, 64, chunks, seed=40 + g))


@pytest.mark.parametrize("dtype, D", TYPES)
@pytest.mark.parametrize("window", [0, 300])
def test_splits_of_short_sequences(dtype, D, window):
    """Work enough for this kernel by the bounds that the sequences have: splits of few pairs."""
    _go(Case(dtype, D, 4, 8, 64, [(1100, 500), (900, 30), (1, 1), (1000, 7)], window, 2, seed=45))


@pytest.mark.parametrize("dtype, D", TYPES)
@pytest.mark.parametrize("window, sink", [(1, 0), (1, 1), (7, 0), (16, 4), (64, 4), (100, 70), (33, 200), (5000, 4), (600, 600)])
def test_windows_and_sinks(dtype, D, window, sink):
    _go(_case(dtype, D, 4, 1, 16, [(1, 1), (64, 5), (65, 1), (300, 1), (260, 100), (90, 90), (333, 33), (20, 6), (1400, 50)], window, sink, seed=window))


@pytest.mark.parametrize("dtype, D", TYPES)
@pytest.mark.parametrize("window", [0, 20])
@pytest.mark.parametrize("page", [16, 64])
def test_holes(dtype, D, window, page):
    c = _case(dtype, D, 4, 2, page, [(100, 5), (300, 140), (16, 16), (200, 33), (5, 5), (210, 1)], window, 2, seed=5)
    c.table[0, 0] = c.n_pages
    c.table[1, 1], c.table[1, 3] = -1, 1 << 30
    c.table[2, 0] = -1
    c.table[3, 1:4] = -1
    c.table[4, 0] = -(1 << 31)
    c.table[5, 2] = -7
    _go(c, weights=True)


@pytest.mark.parametrize("dtype, D", TYPES)
def test_tokens_before_the_first_position_and_outside_of_all_chunks(dtype, D):
    _go(_case(dtype, D, 4, 1, 16, [(3, 10), (0, 4), (40, 45), (33, 1), (70, 20)], seed=6, before=5, behind=9))


@pytest.mark.parametrize("dtype, D", TYPES)
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("bad", [float("inf"), float("nan"), -float("inf")])
def test_hidden_values_stay_hidden(dtype, D, page, bad):
    c = _case(dtype, D, 4, 2, page, [(37, 5), (300, 90), (100, 40), (290, 6), (70, 70)], 48, 3, seed=8)
    for b, (n, m) in enumerate(c.chunks):   # behind the end, in the last page and in the spare ones
        at = int(c.table[b, (n - 1) // page])
        if n % page:
            c.K[at, :, n % page:], c.V[at, :, n % page:] = bad, bad
    used = set(c.table[c.table >= 0].tolist())
    for at in set(range(c.n_pages)) - used:
        c.K[at], c.V[at] = bad, bad
    c.K[int(c.table[1, 100 // page]), :, 100 % page] = bad      # outside of the window
    c.V[int(c.table[1, 100 // page]), :, 100 % page] = bad
    c.v_new[int(c.q_start[2]) + 25, 0, 5] = bad                 # one value of a later token
    c.k_new[int(c.q_start[4]) + 66, 1, 3] = bad
    c.v_new[int(c.q_start[4]) + 3, 1, D - 1] = bad              # seen by 48 tokens, then outside of the window
    c.v_new[int(c.q_start[1]) + 1, 0, 0] = bad
    c.v_new[int(c.q_start[1]) + 60, 0, 7] = bad                 # two in one tile of rows
    _go(c)


@pytest.mark.parametrize("dtype, D, scale", [("bf16", 128, -0.1), ("f32", 64, -0.2), ("bf16", 64, 0.0), ("f32", 128, 0.0), ("bf16", 128, 3.0), ("f32", 128, -0.1)])
def test_scales(dtype, D, scale):
    _go(_case(dtype, D, 4, 1, 16, [(60, 1), (150, 20), (40, 40)], scale=scale, seed=10), weights=True)


@pytest.mark.parametrize("dtype, D", TYPES)
def test_growing_logits(dtype, D):
    """Keys that grow along the sequence: the reference has to follow many times."""
    c = _case(dtype, D, 4, 1, 16, [(400, 60), (300, 300)], seed=21)
    c.K *= 0.1
    for b, (n, m) in enumerate(c.chunks):
        for p in range(n - m):
            c.K[int(c.table[b, p // 16]), :, p % 16] = (c.q[int(c.q_start[b]), 0].float() * (p / 40)).to(c.dt)
        for i in range(m):
            c.k_new[int(c.q_start[b]) + i] = (c.q[int(c.q_start[b]), 0].float() * ((n - m + i) / 40)).to(c.dt)
    _go(c, weights=True)


@pytest.mark.parametrize("dtype, D", TYPES)
def test_huge_logits(dtype, D):
    """Logits whose rounding is beyond an exponential's range: the largest key takes all."""
    c = _case(dtype, D, 4, 1, 16, [(200, 1), (150, 40), (90, 90)], scale=1e12, seed=11)
    K, V = c.appended()
    ref, _ = c.reference(K, V)
    s = c.dev()
    c.run(s)
    out, acc = s["out"].double().cpu().numpy(), s["acc"].double().cpu().numpy()
    tol = 2.0 ** -8 if dtype == "bf16" else 1e-6
    assert np.isfinite(out).all() and (np.abs(out - ref["out"]) <= tol * np.abs(ref["out"]) + 1e-30).all()
    assert (np.abs(acc - ref["acc"]) <= 1e-4).all()


@pytest.mark.parametrize("dtype, D", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("max_chunk", [5, 6, 17, 40])
def test_chunks_longer_than_their_bound(dtype, D, max_chunk):
    c = _case(dtype, D, 4, 2, 16, [(500, 160), (300, 1), (40, 40), (200, 3), (1500, 1)], seed=12)
    c.max_chunk = max_chunk
    _go(c)


@pytest.mark.parametrize("dtype, D", TYPES)
def test_equal_calls_give_equal_bits(dtype, D):
    c = _case(dtype, D, 4, 2, 32, [(2000, 1), (900, 200), (1500, 3), (2500, 20)], seed=14)
    s = c.dev()
    c.run(s, weights=False)
    want = [s[k].clone() for k in ("out", "stats")]
    for i in range(3):
        s["ws"].fill_(i * 85)
        c.run(s, weights=False)
        for x, k in zip(want, ("out", "stats")):
            assert torch.equal(x.view(torch.uint8), s[k].view(torch.uint8)), k


def test_captured_on_one_workspace():
    """Replays of two graphs on one workspace give the eager results."""
    c, c2 = _case("bf16", 128, 4, 2, 64, [(900, 1), (1800, 1), (1300, 64)], seed=16), _case("bf16", 128, 4, 2, 64, [(700, 1), (1300, 30), (64, 64)], seed=17)
    s, s2 = c.dev(), c2.dev()
    s["ws"] = s2["ws"] = torch.empty(max(s["ws"].numel(), s2["ws"].numel()), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.run(s, weights=False)
        c2.run(s2, weights=False)
    side.synchronize()
    want = {k: (s[k].clone(), s2[k].clone()) for k in ("out", "stats")}
    graphs = []
    for cc, ss in ((c, s), (c2, s2)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            cc.run(ss, weights=False)
        graphs.append(g)
    for i in range(4):
        for x in (s, s2):
            x["out"].fill_(0)
            x["stats"].fill_(0)
        graphs[i % 2].replay()
        graphs[1 - i % 2].replay()
        torch.cuda.synchronize()
        for k, (a, b) in want.items():
            assert torch.equal(a.view(torch.uint8), s[k].view(torch.uint8)) and torch.equal(b.view(torch.uint8), s2[k].view(torch.uint8)), (i, k)
        s["ws"].fill_(i)


def test_many_sequences():
    """More sequences than one wavefront looks at in a step, a few with chunks."""
    _go(_case("bf16", 64, 4, 1, 16, [(20 + b % 50, 1 if b % 9 else 17) for b in range(150)], seed=30))


@pytest.mark.parametrize("long", [True, False])
def test_replayed_with_other_sequences(long):
    """A captured call follows what the device arrays hold at its replay: other lengths, other chunks, the same buffers."""
    make = _case if long else Case
    c = make("bf16", 128, 4, 2, 64, [(900, 1), (1300, 64), (700, 5)], seed=50)
    s = c.dev()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.run(s)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.run(s)
    for chunks in ([(850, 64), (1290, 1), (640, 5)], [(900, 0), (33, 33), (700, 37)], [(900, 1), (1300, 64), (700, 5)], [(1, 1), (1, 1), (70, 68)]):
        c2 = copy.copy(c)
        c2.chunks = chunks
        c2.kv_len = torch.tensor([n for n, _ in chunks], dtype=torch.int32)
        c2.q_start = torch.tensor(np.concatenate([[0], np.cumsum([m for _, m in chunks])]), dtype=torch.int32)
        for k in ("K", "V", "kv_len", "q_start", "acc"):
            s[k].copy_(getattr(c2, k))
        s["out"].fill_(7.0)
        s["stats"].fill_(7.0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        ref, tol = c2.reference()
        c2.check(s, ref, tol, what=str(chunks))


@pytest.mark.parametrize("dtype, D", TYPES)
def test_lengths_beyond_the_table(dtype, D):
    """kv_len is taken as what the table has entries for; a negative one as 0."""
    c = Case(dtype, D, 4, 2, 16, [(40, 3), (70, 30), (20, 2)], seed=51)
    room = c.max_pages * 16
    c.kv_len = torch.tensor([room + 12345, 1 << 30, -5], dtype=torch.int32)
    c.chunks = [(room, 3), (room, 30), (0, 2)]
    _go(c, weights=True)


def test_first_call_of_a_process_is_captured():
    """Nothing but the capture has called the library: both kinds of tiles, weights and the step that accumulates."""
    code = """
import sys
sys.path[:0] = [%r, %r]
import torch
import paper_2602_03203_amd as fk
from test_gpu_paged_prompt import _case
c = _case("f32", 128, 4, 2, 64, [(900, 1), (1300, 64)], seed=52)
s = c.dev()
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    c.run(s)
g.replay()
torch.cuda.synchronize()
ref, tol = c.reference()
c.check(s, ref, tol)
print("as it should be")
""" % (str(__file__).rsplit("/", 2)[0], str(__file__).rsplit("/", 1)[0])
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and "as it should be" in r.stdout, r.stdout[-500:] + r.stderr[-2000:]


def test_scale_that_is_no_number():
    c = _case("bf16", 64, 4, 1, 16, [(30, 1), (60, 20)], seed=53)
    c.scale = float("nan")
    s = c.dev()
    c.run(s, weights=False)
    torch.cuda.synchronize()
    assert torch.isnan(s["out"]).all()


@pytest.mark.parametrize("dtype, D", TYPES)
@pytest.mark.parametrize("long", [True, False])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_weights_of_queries_without_numbers(dtype, D, long, bad):
    """A query that is not finite gives the pairs that it sees no number, and all others theirs."""
    make = _case if long else Case
    c = make(dtype, D, 4, 1, 16, [(90, 40), (200, 150), (33, 1)], 20, 2, seed=54)
    c.q[13, 2, 5] = bad
    c.q[60, 0] = bad
    c.k_new[100, 0, 3] = bad     # a key, seen by the queries behind it that reach it
    s = c.dev()
    c.run(s)
    torch.cuda.synchronize()
    ref, tol = c.reference()
    assert np.isnan(ref["acc"]).any() and np.isfinite(ref["acc"][:, :, :300]).sum() > 100
    got = s["acc"].double().cpu().numpy()
    assert (np.isnan(got) == np.isnan(ref["acc"])).all()
    ok = np.isfinite(ref["acc"])
    assert (np.abs(got - ref["acc"])[ok] <= np.where(np.isfinite(tol["acc"]), tol["acc"], 1e-5)[ok]).all()


@pytest.mark.parametrize("dtype, D, page", [("bf16", 64, 16), ("f32", 64, 64)])
def test_workspace_under_a_window(dtype, D, page):
    """Windows change how work is split, the workspace does not know them: nothing behind it is written."""
    for chunks, window in (([(700 + 31 * b, 1 + b % 5) for b in range(70)], 6000), ([(900, 4)] * 3, 500), ([(1300, 70), (1100, 1)], 700)):
        c = Case(dtype, D, 8, 2, page, chunks, window, 2, seed=56, room=6400 // page)
        s = c.dev()
        behind = 1 << 16
        for k in ("ws", "wws"):
            n = s[k].numel()
            s[k + "_all"] = torch.full((n + behind,), 77, dtype=torch.uint8, device="cuda")
            s[k] = s[k + "_all"][:n]
        c.run(s)
        torch.cuda.synchronize()
        for k in ("ws", "wws"):
            assert (s[k + "_all"][s[k].numel():] == 77).all(), (k, len(chunks))
        ref, tol = c.reference()
        c.check(s, ref, tol)
