"""Attention of drafted trees over rows and pages against the oracle."""
import numpy as np
import pytest
import torch

from drafts_util import UB, TreeCase, tree

pytestmark = pytest.mark.gpu

LENS = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300]


def _sizes(*nodes):
    """Sequences of these tree sizes over lengths around the tiles' borders."""
    return [(LENS[(3 * i + n) % len(LENS)], tree(n, seed=i)) for i, n in enumerate(nodes)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("g, hkv, page", [(1, 2, 0), (4, 2, 0), (8, 1, 16), (7, 1, 32), (3, 2, 64), (5, 1, 0)])
def test_small_trees(dtype, D, g, hkv, page):
    """Up to 16 rows of queries and up to 32, every length, no tree at all among them."""
    most = 16 // g, 32 // g
    for nodes in sorted(set(most)):
        if nodes:
            TreeCase(dtype, D, g, hkv, [(n, tree(1 + i % nodes, seed=i)) for i, n in enumerate(LENS)] + [(40, []), (33, tree(nodes, depth=0))], page, seed=g).go(f"{nodes} nodes")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("g, nodes, page", [(4, (9, 16, 13), 0), (4, (17, 30, 1), 16), (1, (64, 33, 63), 0), (8, (8, 7, 5), 64), (2, (65, 100, 31), 0), (7, (26, 20, 3), 32),
                                            (4, (65, 64, 40), 128), (1, (256, 129, 255), 0), (8, (33, 2, 17), 16), (5, (256, 1, 14), 0)])
def test_larger_trees(dtype, D, g, nodes, page):
    TreeCase(dtype, D, g, 1, _sizes(*nodes), page, seed=g).go()


@pytest.mark.parametrize("dtype, D, g, nodes, lens, page", [("bf16", 128, 4, 12, (2111, 2177), 0), ("bf16", 128, 4, 40, (3000, 1500), 64), ("bf16", 64, 1, 5, (5000,), 16),
                                                            ("f32", 64, 4, 8, (1300, 700), 0), ("f32", 128, 8, 20, (900,), 32), ("bf16", 128, 2, 200, (1200,), 0), ("bf16", 64, 8, 8, (2050, 4100), 1024)])
def test_long_rows(dtype, D, g, nodes, lens, page):
    """Pairs split over workgroups and merged."""
    TreeCase(dtype, D, g, 1, [(n, tree(nodes, seed=n)) for n in lens], page, seed=nodes).go()


@pytest.mark.parametrize("dtype, D", [("f32", 64), ("bf16", 128)])
def test_heads_of_a_sequence_keep_different_numbers(dtype, D):
    TreeCase(dtype, D, 4, 3, [([5, 70, 0], tree(6)), ([300, 33, 129], tree(20)), ([1, 1, 64], tree(3))], seed=1).go()


@pytest.mark.parametrize("dtype, D", [("f32", 64), ("bf16", 64), ("bf16", 128), ("f32", 128)])
@pytest.mark.parametrize("nodes", [3, 11, 40])
@pytest.mark.parametrize("window, sink", [(1, 0), (2, 0), (3, 1), (16, 4), (64, 4), (100, 70), (33, 200), (5000, 4), (3, 2 ** 31 - 1)])
def test_windows_and_sinks(dtype, D, nodes, window, sink):
    """Ancestors leave a window too; those at the first positions stay."""
    TreeCase(dtype, D, 4, 1, [(0, tree(nodes, depth=0)), (1, tree(nodes)), (3, tree(nodes, 1)), (64, tree(nodes, 2)), (130, tree(nodes, depth=0)), (333, tree(nodes, 3))], 16, window, sink,
             seed=window).go()


@pytest.mark.parametrize("dtype, D", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("nodes", [3, 12, 40])
@pytest.mark.parametrize("window", [0, 20])
def test_holes(dtype, D, nodes, window):
    """Pairs in pages that are not there are seen by nobody, whatever number the table holds."""
    c = TreeCase(dtype, D, 4, 2, [(100, tree(nodes)), (40, tree(nodes, 1)), (16, tree(nodes, 2)), (200, tree(nodes, 3))], 16, window, 0, seed=5)
    c.table[0, 1] = -1
    c.table[1, 0] = c.n_pages
    c.table[1, 2] = -2 ** 31
    c.table[2, 0] = 2 ** 31 - 1   # nothing but its own tree is left
    c.table[3, 3:9] = -1
    c.go()


@pytest.mark.parametrize("dtype, D", [("bf16", 128), ("f32", 64), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("nodes", [4, 7, 12, 50])
@pytest.mark.parametrize("page", [0, 16])
def test_values_that_a_node_does_not_see(dtype, D, nodes, page):
    """Infinities and NaN behind a row's end and in other branches reach nobody; in a node's own way and in the cache they reach those that see them."""
    seqs = [(33, tree(nodes, 1)), (64, tree(nodes, 2)), (0, tree(nodes, 3)), (129, tree(nodes, 4))]
    c = TreeCase(dtype, D, 4, 1, seqs, page, seed=8)
    if page:
        for b, n in ((0, 33), (3, 129)):
            s = c.slot(b, 0, n - 1)
            c.K[s[0], 0, s[2] + 1:], c.V[s[0], 0, s[2] + 1:] = float("nan"), float("inf")
        spare = sorted(set(range(c.n_pages)) - set(c.table.flatten().tolist()))
        c.K[spare], c.V[spare] = float("nan"), float("nan")
    else:
        for b, n in enumerate((33, 64, 0, 129)):
            c.K[b, 0, n:], c.V[b, 0, n:] = float("nan"), float("inf")
    t = c.q_start.tolist()
    c.v_tree[t[0] + nodes - 1, 0, 3] = float("inf")      # a leaf's value
    c.v_tree[t[1] + 1, 0, 5] = float("nan")              # an inner node's
    c.v_tree[t[1] + 2, 0, 6] = -float("inf")
    c.k_tree[t[2] + nodes - 1, 0, 0] = float("nan")      # a leaf's key
    c.V[c.slot(3, 0, 70)][9] = float("inf")              # everybody sees this one
    c.q[t[3], 2, 1] = float("nan")                       # one query head of the root
    ref, tol = c.reference()
    assert np.isfinite(ref["out"][t[0]:t[0] + nodes - 1]).all() and np.isnan(ref["out"][t[1]:t[2]]).any() and np.isfinite(ref["out"][t[1]]).all()
    s = c.dev()
    c.run(s)
    torch.cuda.synchronize()
    c.check(s, ref, tol)


def test_infinite_values_under_a_window():
    """The border of a window crosses a tile: nodes of different depth see different pairs of it."""
    for dtype, D, nodes in (("bf16", 128, 4), ("bf16", 128, 14), ("f32", 64, 40)):
        c = TreeCase(dtype, D, 4, 1, [(100, tree(nodes, depth=0)), (90, tree(nodes, 3))], 16, 30, 2, seed=nodes)
        for b, n in ((0, 100), (1, 90)):
            for j, x in ((n - 29, float("inf")), (n - 28, float("nan")), (n - 35, float("nan")), (1, -float("inf"))):
                c.V[c.slot(b, 0, j)][j % D] = x
        c.go(f"{dtype} {nodes}")


@pytest.mark.parametrize("dtype, D, nodes", [("bf16", 128, 4), ("bf16", 64, 8), ("f32", 128, 4), ("bf16", 128, 16), ("f32", 64, 30), ("bf16", 128, 30)])
@pytest.mark.parametrize("key_scale, scale", [(1.0, -0.2), (1.0, 0.0), (30.0, None), (3000.0, 1.0), (1.0, -0.0)])
def test_scales_and_large_logits(dtype, D, nodes, key_scale, scale):
    TreeCase(dtype, D, 4, 1, [(70, tree(nodes)), (300, tree(nodes, 1)), (1, tree(nodes, 2))], 0, scale=scale, key_scale=key_scale, seed=nodes).go()


@pytest.mark.parametrize("nodes", [4, 8, 16, 40])
def test_logits_that_are_no_numbers(nodes):
    """All logits -inf: zeros and (-inf, 0); a scale that is NaN shows."""
    for dtype, D in (("bf16", 128), ("f32", 64)):
        c = TreeCase(dtype, D, 4, 1, [(40, tree(nodes, depth=0))], 0, seed=2)
        c.K[:], c.k_tree[:], c.q[:] = 0, 0, 0
        c.K[..., 0], c.k_tree[..., 0], c.q[..., 0] = float("inf"), float("inf"), -1.0
        c.q[..., 1:] = 0
        c.K[..., 1:], c.k_tree[..., 1:] = 1.0, 1.0
        c.go(dtype)
        c.scale = float("nan")
        s = c.dev()
        c.run(s)
        assert torch.isnan(s["stats"][..., 1]).all() and torch.isnan(s["out"].float()).all()


@pytest.mark.parametrize("dtype, D", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("max_tree", [1, 4, 8, 20, 256])
def test_bounds_that_do_not_hold(dtype, D, max_tree):
    """max_tree and max_len only size the launch; trees are longer and shorter, tokens lie before and behind them."""
    seqs = [(300, tree(70, 1)), (5, tree(2)), (1000, tree(256, 2)), (0, []), (64, tree(33, 3))]
    for page in (0, 16):
        TreeCase(dtype, D, 4, 1, seqs, page, before=3, behind=9, max_tree=max_tree, max_len=1 if max_tree < 20 else None, seed=max_tree).go(f"page {page}")


def test_too_many_nodes_are_passed_over():
    seqs = [(30, tree(5)), (40, tree(257)), (20, tree(256, 1)), (10, tree(300)), (50, tree(4))]
    for g in (1, 4):
        TreeCase("bf16", 64, g, 1, seqs, 0, seed=g).go()


def test_parents_that_are_none():
    """A parent at its child's place or behind it, or below 0, stands for none."""
    p = tree(12, 5)
    p[3], p[4], p[7], p[9], p[0] = 3, 11, -7, 2 ** 31 - 1, 0
    for dtype, D in (("bf16", 128), ("f32", 64)):
        for g in (1, 2, 4, 8):
            TreeCase(dtype, D, g, 1, [(20, p), (0, [5, -2 ** 31, 0])], 0, seed=g).go()


def test_many_short_trees_are_dealt_out():
    """Many sequences with one long tree: places are dealt to the tiles there are."""
    seqs = [(17 + b, tree(200 if b == 41 else 1 + b % 3, b)) for b in range(90)]
    TreeCase("bf16", 128, 4, 1, seqs, 0, seed=3).go()
    TreeCase("f32", 64, 2, 1, seqs[:50], 16, seed=4).go()


def test_no_stats_and_no_tokens():
    import paper_2602_03203_amd as fk
    TreeCase("bf16", 128, 4, 2, [(100, tree(6)), (50, tree(30))], 0).go(stats=False)
    c = TreeCase("bf16", 128, 4, 2, [(100, []), (50, [])], 0)
    s = c.dev()
    c.run(s)
    torch.cuda.synchronize()
    assert fk.fk_tree_attn_workspace(s["desc"], 0, 1, 5) > 0


@pytest.mark.parametrize("dtype, D, nodes, n, page", [("bf16", 128, 4, 3000, 0), ("bf16", 128, 13, 2000, 64), ("f32", 64, 50, 900, 0), ("bf16", 64, 64, 1500, 16)])
def test_equal_bits_other_stream_and_graphs(dtype, D, nodes, n, page):
    """Equal calls give equal bits; on a stream of its own; captured, with two graphs on one workspace and other lengths, trees and values between replays."""
    a = TreeCase(dtype, D, 4, 2, [(n, tree(nodes, 1)), (n // 2, tree(nodes, 2))], page, seed=1)
    b = TreeCase(dtype, D, 4, 2, [(n // 3, tree(nodes, 3)), (n, tree(nodes, depth=0))], page, seed=2)
    if page:   # the same buffers' shapes
        big = max(a.n_pages, b.n_pages)
        for c in (a, b):
            c.K, c.V = (torch.cat([x, x[:1].expand(big - x.shape[0], -1, -1, -1)]) if x.shape[0] < big else x for x in (c.K, c.V))
            c.n_pages = big
    sa, sb = a.dev(), b.dev()
    (ra, ta), (rb, tb) = a.reference(), b.reference()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a.run(sa, stream=side)
    side.synchronize()
    a.check(sa, ra, ta)
    first = sa["out"].clone(), sa["stats"].clone()
    a.run(sa)
    assert torch.equal(first[0], sa["out"]) and torch.equal(first[1], sa["stats"])
    sb["ws"] = sa["ws"]
    graphs = []
    for c, s in ((a, sa), (b, sb)):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            c.run(s)
        graphs.append(gr)
    keep = {k: sa[k].clone() for k in ("K", "V", "len", "q_start", "parent", "q", "k_tree", "v_tree") + (("table",) if page else ())}
    for turn in range(4):
        for s in (sa, sb):
            s["out"].fill_(0)
            s["stats"].fill_(0)
        graphs[turn % 2].replay()
        graphs[1 - turn % 2].replay()
        torch.cuda.synchronize()
        a.check(sa, *((ra, ta) if turn % 2 == 0 else (rb, tb)), f"replay {turn}")
        b.check(sb, rb, tb, f"replay {turn}")
        for k, x in keep.items():   # the captured call of a now works on b's values, then on its own again
            sa[k].copy_(sb[k] if turn % 2 == 0 else x)


def test_pairs_beyond_32_bit_offsets():
    """A pool of more than 2^31 elements: pages at its end."""
    D, page, H = 128, 1024, 8
    pages = (2 ** 31) // (H * page * D) + 12
    import paper_2602_03203_amd as fk
    K = torch.zeros((pages, H, page, D), dtype=torch.bfloat16, device="cuda")
    V = torch.zeros_like(K)
    for nodes in (3, 7, 15, 40):
        c = TreeCase("bf16", D, 4, H, [(3000, tree(nodes, 1)), (1025, tree(nodes, 2))], page, seed=nodes)
        at = [pages - 1 - i for i in range(c.n_pages)]
        K[at], V[at] = c.K.cuda(), c.V.cuda()
        s = c.dev()
        s["table"] = torch.where(s["table"] >= 0, pages - 1 - s["table"], s["table"]).int().contiguous()
        s["K"], s["V"] = K, V
        s["desc"] = fk.PagedDesc(c.B, H * 4, H, D, page, pages, c.max_pages, "bf16")
        c.run(s)
        torch.cuda.synchronize()
        c.check(s, *c.reference())


def test_rows_beyond_32_bit_offsets():
    """Rows that begin 2^31 elements into the cache."""
    import paper_2602_03203_amd as fk
    D, H, cap = 128, 3, 1 << 23
    K = torch.zeros((1, H, cap, D), dtype=torch.bfloat16, device="cuda")
    V = torch.zeros_like(K)
    for g, nodes, n in ((4, 3, 3000), (4, 7, 1025), (4, 15, 2000), (1, 256, 700), (8, 256, 300)):
        c = TreeCase("bf16", D, g, H, [(n, tree(nodes, 1))], seed=nodes)
        K[:, :, :c.cap], V[:, :, :c.cap] = c.K.cuda(), c.V.cuda()
        s = c.dev()
        s["K"], s["V"], s["desc"] = K, V, fk.CacheDesc(1, H * g, H, D, cap, "bf16")
        s["ws"] = fk.new_tree_attn_workspace(s["desc"], c.n_tokens, c.max_tree, c.max_len)
        c.run(s)
        torch.cuda.synchronize()
        c.check(s, *c.reference(), f"{nodes} nodes")


def test_calls_of_any_sizes_share_a_workspace():
    """Rows and pages, few and many splits, in turns: the counters are where every call looks for them."""
    cases = [TreeCase("bf16", 128, 4, 2, [(3000, tree(4, 1)), (2500, tree(3))], 0, seed=1), TreeCase("bf16", 128, 4, 1, [(4000, tree(50, 2))], 64, seed=2),
             TreeCase("f32", 64, 8, 1, [(900, tree(40, 3)), (100, tree(8)), (2000, tree(2))], 0, seed=3), TreeCase("bf16", 64, 4, 4, [(1500, tree(33, 4))], 16, seed=4)]
    devs = [c.dev() for c in cases]
    ws = torch.zeros(max(s["ws"].numel() for s in devs), dtype=torch.uint8, device="cuda")
    refs = [c.reference() for c in cases]
    for turn in range(3):
        for c, s in zip(cases, devs):
            s["ws"] = ws
            s["out"].fill_(7)
            c.run(s)
        torch.cuda.synchronize()
        for i, (c, s, r) in enumerate(zip(cases, devs, refs)):
            c.check(s, *r, f"turn {turn} case {i}")


# two terms of bf16 for a weight: the first cut off, by a step of bf16 (2^-7 of it) at most, the second off by half a step (2^-8) of that rest; the rest is 2^-20 of the
# weight too large, which is rounded with it
TWO_TERMS = 2.0 ** -15 + 2.0 ** -19


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("g, nodes, page", [(4, 4, 0), (4, 8, 16), (8, 4, 0), (4, 12, 0), (1, 50, 32), (4, 40, 0), (8, 30, 16)])
def test_equal_weights_next_to_a_larger_one(D, g, nodes, page):
    """All pairs but one have the same weight, which rounds down by nearly half a step of bf16: an error that no average takes away."""
    w = (1 + 0.97 * UB) / 8
    c = TreeCase("bf16", D, g, 1, [(250, tree(nodes, depth=0)), (100, tree(nodes, 1))], page, scale=-float(np.log(w)), seed=nodes)
    c.q[:], c.K[:], c.k_tree[:] = 0, 0, 0
    c.q[..., 0], c.K[..., 0], c.k_tree[..., 0] = 1, -1, -1
    gen = torch.Generator().manual_seed(D)
    c.V[:] = torch.rand(D, generator=gen).add_(0.5).to(c.dt)   # alike for all pairs but the first of a row
    c.v_tree[:] = c.V[(0,) * (c.V.dim() - 1)]
    for b in range(2):
        c.K[c.slot(b, 0, 0)], c.V[c.slot(b, 0, 0)] = 0, 0
    s = c.dev()
    c.run(s)
    torch.cuda.synchronize()
    c.check(s, *c.reference(TWO_TERMS))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("g, nodes, lens, page, window", [(4, 4, (300, 33), 0, 0), (7, 3, (300, 129), 16, 0), (4, 8, (65, 200), 0, 0), (4, 12, (1100, 700), 0, 0), (4, 16, (300, 17), 64, 100),
                                                          (7, 26, (800,), 0, 0), (8, 30, (900, 64), 32, 0), (1, 200, (64, 600), 0, 0), (4, 3, (2500,), 0, 0), (2, 15, (0, 1), 16, 0)])
def test_weights_keep_sixteen_bits(D, g, nodes, lens, page, window):
    c = TreeCase("bf16", D, g, 2, [(n, tree(nodes, n)) for n in lens], page, window, 4 if window else 0, seed=nodes)
    s = c.dev()
    c.run(s)
    torch.cuda.synchronize()
    c.check(s, *c.reference(TWO_TERMS))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("g, nodes, page", [(4, 4, 0), (4, 8, 16), (4, 12, 0), (8, 30, 16), (4, 64, 0)])
def test_infinite_values_of_equal_weights(D, g, nodes, page):
    """All weights are 1, whose second term has nothing to hold: infinities that are seen stay infinities of their sign, in the cache and on a node's way."""
    c = TreeCase("bf16", D, g, 1, [(250, tree(nodes, depth=0)), (90, tree(nodes, 1)), (700, tree(nodes, 2))], page, seed=nodes)
    c.q[:] = 0
    for b, j in ((0, 3), (1, 89), (2, 600)):
        c.V[c.slot(b, 0, j)][7], c.V[c.slot(b, 0, j)][D - 1] = float("inf"), -float("inf")
    c.v_tree[int(c.q_start[1]) + nodes // 2, 0, 20] = float("inf")
    ref = c.reference(TWO_TERMS)
    assert np.isinf(ref[0]["out"]).any() and not np.isnan(ref[0]["out"]).any()
    s = c.dev()
    c.run(s)
    torch.cuda.synchronize()
    c.check(s, *ref)


@pytest.mark.parametrize("dtype, D, page", [("bf16", 128, 0), ("bf16", 64, 64), ("f32", 64, 0)])
def test_one_workspace_for_smaller_calls(dtype, D, page):
    """Allocated once for the largest trees, which split nothing, it serves smaller ones, which do: the same bits as with a workspace of their own."""
    import paper_2602_03203_amd as fk
    B, H, g, cap = 16, 8, 4, 2048
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(D)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dt)   # noqa: E731
    i32 = dict(dtype=torch.int32, device="cuda")
    K, V = (r(B * cap // page, H, page, D) if page else r(B, H, cap, D) for _ in range(2))
    if page:
        desc, size = fk.PagedDesc(B, H * g, H, D, page, K.shape[0], cap // page, dtype), fk.fk_paged_tree_attn_workspace
        where = (torch.arange(K.shape[0], **i32).reshape(B, -1), torch.full((B,), cap, **i32))
    else:
        desc, size, where = fk.CacheDesc(B, H * g, H, D, cap, dtype), fk.fk_tree_attn_workspace, (torch.full((B, H), cap, **i32),)
    most = torch.zeros(size(desc, B * 256, 256, cap), dtype=torch.uint8, device="cuda")
    for nodes, max_len in ((64, cap), (256, cap), (8, cap), (30, cap), (1, 1200), (16, cap), (100, cap)):
        n = B * nodes
        parent = torch.tensor([p for b in range(B) for p in tree(nodes, b)], **i32)
        q_start = torch.arange(0, n + 1, nodes, **i32)
        q, kt, vt = r(n, H * g, D), r(n, H, D), r(n, H, D)
        outs = []
        for ws in (most, torch.zeros(size(desc, n, nodes, max_len), dtype=torch.uint8, device="cuda")):
            out, stats = torch.full_like(q, 7), torch.full((n, H * g, 2), 7.0, device="cuda")
            tail = (out, stats, ws)
            if page:
                fk.fk_paged_tree_attn(desc, q, K, V, *where, kt, vt, parent, q_start, nodes, max_len, 0, 0, D ** -0.5, *tail)
            else:
                fk.fk_tree_attn(desc, q, K, V, *where, kt, vt, parent, q_start, nodes, max_len, D ** -0.5, *tail)
            outs.append((out, stats))
        torch.cuda.synchronize()
        assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1]) and torch.isfinite(outs[0][1]).all(), f"{nodes} nodes"
    assert not most[:16384].any()   # the counters are at zero again
