"""The accepted paths join the rows or the pages; a round of drafts as a whole, beside the framework's own steps."""
import numpy as np
import pytest
import torch

from drafts_util import TreeCase, U, UB, tree
from oracle import drafts as od

pytestmark = pytest.mark.gpu


def _paths(seqs, seed):
    """Of every tree some node's path from its root."""
    rng = np.random.default_rng(seed)
    return [od.ancestors(p, int(rng.integers(0, len(p))))[::-1] if p else [] for _, p in seqs]


def _lay(c, paths, counts):
    path = np.full(c.n_tokens, -1, np.int32)
    for p, s in zip(paths, c.q_start.tolist()):
        path[s:s + len(p)] = p
    return torch.tensor(path), torch.tensor(counts, dtype=torch.int32)


def _rows(c, paths, counts, with_acc, first):
    """Expected K, V, pos, len, acc behind a commit, on the host."""
    K, V, lens = c.K.clone(), c.V.clone(), c.lens.copy()
    pos = torch.arange(c.B * c.H * c.cap, dtype=torch.int32).reshape(c.B, c.H, c.cap)
    acc = torch.rand((c.B, c.H, c.cap), generator=torch.Generator().manual_seed(9))
    start = pos.clone(), acc.clone()
    for b, (_, parent) in enumerate(c.seqs):
        way = od.path_of(paths[b], counts[b], len(parent))
        for h in range(c.H):
            for i, node in enumerate(way):
                if lens[b, h] == c.cap:
                    break
                s, t = lens[b, h], int(c.q_start[b]) + node
                K[b, h, s], V[b, h, s], pos[b, h, s], acc[b, h, s] = c.k_tree[t, h], c.v_tree[t, h], first[b] + i, 0
                lens[b, h] += 1
    return K, V, pos, lens, acc if with_acc else start[1], start


def _same(a, b):
    return torch.equal(a.cpu().contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


@pytest.mark.parametrize("dtype, D", [("f32", 64), ("f32", 128), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("with_acc", [False, True])
def test_rows(dtype, D, with_acc):
    """Full rows, rows with less room than the path is long, empty trees, paths cut short, counts beyond the tree and below zero."""
    import paper_2602_03203_amd as fk
    seqs = [([7, 100, 0], tree(9, 1)), ([104, 105, 103], tree(8, depth=0)), (50, []), (3, tree(200, depth=0)), (40, tree(30, 2)), (12, tree(5, depth=0)), (13, tree(5, depth=0)), (1, tree(300, 1))]
    c = TreeCase(dtype, D, 2, 3, seqs, seed=4, before=2, behind=3, room=1)
    paths = _paths(seqs, 1)
    paths[1], paths[3], paths[5], paths[6], paths[7] = list(range(8)), list(range(200)), [0, 1, 5, 2], [0, -1], [0, 299]
    counts = [len(p) for p in paths]
    counts[2], counts[4], counts[5] = 3, -2, 99
    path, accepted = _lay(c, paths, counts)
    first = [1000 * b for b in range(c.B)]
    K, V, pos, lens, acc, (pos0, acc0) = _rows(c, paths, counts, with_acc, first)
    d = [x.cuda() for x in (c.K, c.V, pos0, torch.tensor(c.lens), acc0)]
    desc = fk.CacheDesc(c.B, c.H * c.g, c.H, D, c.cap, dtype)
    fk.fk_commit_drafts(desc, *d[:4], d[4] if with_acc else None, c.k_tree.cuda(), c.v_tree.cuda(), c.q_start.cuda(), path.cuda(), accepted.cuda(),
                        torch.tensor(first, dtype=torch.int32).cuda())
    torch.cuda.synchronize()
    for got, want, name in zip(d, (K, V, pos, torch.tensor(lens), acc), ("K", "V", "pos", "len", "acc")):
        assert _same(got, want), name


@pytest.mark.parametrize("dtype, D, page", [("f32", 64, 16), ("bf16", 128, 16), ("bf16", 64, 64), ("f32", 128, 32)])
def test_pages(dtype, D, page):
    """Across page borders, into holes, beyond the page table."""
    import paper_2602_03203_amd as fk
    seqs = [(page - 3, tree(40, depth=0)), (2 * page, tree(9, 2)), (5, []), (0, tree(20, 3)), (page + 1, tree(25, depth=0)), (3 * page - 2, tree(200, depth=0))]
    c = TreeCase(dtype, D, 1, 2, seqs, page, seed=4, before=1, behind=2)
    rng = torch.Generator().manual_seed(3)
    c.n_pages = 40
    c.K, c.V = (torch.randn((40, 2, page, D), generator=rng).to(c.dt) for _ in range(2))
    c.table = torch.randperm(40, generator=rng)[:c.B * c.max_pages].reshape(c.B, -1).int()
    c.table[4, 1] = -1
    c.table[0, 2] = 40
    paths = _paths(seqs, 2)
    paths[0], paths[4], paths[5] = list(range(40)), list(range(25)), list(range(200))
    path, accepted = _lay(c, paths, [len(p) for p in paths])
    K, V, lens = c.K.clone(), c.V.clone(), c.lens[:, 0].copy()
    for b, p in enumerate(paths):
        for node in p:
            if lens[b] == c.max_pages * page:
                break
            for h in range(2):
                s = c.slot(b, h, int(lens[b]))
                if s is not None:
                    K[s], V[s] = c.k_tree[int(c.q_start[b]) + node, h], c.v_tree[int(c.q_start[b]) + node, h]
            lens[b] += 1
    d = [c.K.cuda(), c.V.cuda(), torch.tensor(c.lens[:, 0].copy()).cuda()]
    fk.fk_paged_commit_drafts(fk.PagedDesc(c.B, 2, 2, D, page, 40, c.max_pages, dtype), d[0], d[1], c.table.cuda(), d[2], c.k_tree.cuda(), c.v_tree.cuda(), c.q_start.cuda(),
                              path.cuda(), accepted.cuda())
    torch.cuda.synchronize()
    for got, want, name in zip(d, (K, V, torch.tensor(lens)), ("K", "V", "kv_len")):
        assert _same(got, want), name


def test_many_rows():
    """More rows and sequences than a grid's second dimension holds."""
    import paper_2602_03203_amd as fk
    B, D = 70000, 64
    i32 = dict(dtype=torch.int32, device="cuda")
    kt = torch.randn((B, 1, D), device="cuda").bfloat16()
    q_start, path, ones = torch.arange(B + 1, **i32), torch.zeros(B, **i32), torch.ones(B, **i32)
    K, pos, ln = torch.zeros((B, 1, 2, D), device="cuda").bfloat16(), torch.zeros((B, 1, 2), **i32), torch.ones((B, 1), **i32)
    V = K.clone()
    fk.fk_commit_drafts(fk.CacheDesc(B, 1, 1, D, 2, "bf16"), K, V, pos, ln, None, kt, kt, q_start, path, ones, q_start[:B].contiguous())
    assert torch.equal(K[:, :, 1], kt) and (ln == 2).all() and torch.equal(pos[:, 0, 1], q_start[:B]) and (K[:, :, 0] == 0).all()


def test_paths_of_more_than_32_bits_of_chunks():
    """Commits take paths of any length: 4097 nodes of 65535 heads are more 16-byte chunks than 32 bits count.  All places but the last lie in holes."""
    import paper_2602_03203_amd as fk
    n, H, D, page = 4097, 65535, 64, 16
    i32 = dict(dtype=torch.int32, device="cuda")
    kt = torch.empty((n, H, D), dtype=torch.bfloat16, device="cuda")
    kt[-1] = torch.randn((H, D), device="cuda").bfloat16()
    K, V = (torch.zeros((1, H, page, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.full((1, n // page + 1), -1, **i32)
    table[0, -1] = 0
    length = torch.zeros(1, **i32)
    fk.fk_paged_commit_drafts(fk.PagedDesc(1, H, H, D, page, 1, n // page + 1, "bf16"), K, V, table, length, kt, kt, torch.tensor([0, n], **i32), torch.full((n,), n - 1, **i32),
                              torch.tensor([n], **i32))
    assert length.item() == n
    for x in (K, V):
        assert torch.equal(x[0, :, 0], kt[-1]) and not x[0, :, 1:].any()


@pytest.mark.parametrize("dtype, D", [("bf16", 128), ("f32", 64), ("bf16", 64)])
def test_a_round_is_the_steps_of_its_tokens(dtype, D):
    """Two rounds of drafts: positions, attention, verification, commit.  The cache holds what decode steps of the accepted tokens would have left, and the path's
    outputs are those steps' outputs to within rounding."""
    import paper_2602_03203_amd as fk
    B, H, g, n0, V = 3, 2, 4, 150, 400
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    rng = np.random.default_rng(7)
    gen = torch.Generator(device="cuda").manual_seed(7)
    cap, scale = n0 + 60, D ** -0.5
    desc, rope = fk.CacheDesc(B, H * g, H, D, cap, dtype), fk.RopeDesc(H * g, H, D, D, "half", dtype)
    freq = fk.rope_frequencies(D, 1e6).cuda()
    r = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dt)   # noqa: E731
    i32 = dict(dtype=torch.int32, device="cuda")
    K, Vc, pos, ln = r(B, H, cap, D), r(B, H, cap, D), torch.arange(cap, **i32).expand(B, H, cap).contiguous(), torch.full((B, H), n0, **i32)
    acc = torch.rand((B, H, cap), generator=gen, device="cuda")
    steps = [x.clone() for x in (K, Vc, pos, ln)]
    verify_ws, step_ws = fk.new_verify_workspace(B, V), fk.new_attn_workspace(desc)
    at = torch.full((B,), n0, **i32)   # the root's position
    total = 0
    for turn in range(2):
        trees = [tree(14, 10 * turn + b, depth=4) for b in range(B)]
        sizes = [len(t) for t in trees]
        n = sum(sizes)
        q_start, parent = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), **i32), torch.tensor(np.concatenate(trees), **i32)
        level = torch.tensor([len(od.ancestors(t, i)) - 1 for t in trees for i in range(len(t))], **i32)
        q, k, v = r(n, H * g, D), r(n, H, D), r(n, H, D)
        where = at.repeat_interleave(torch.tensor(sizes, device="cuda")) + level
        fk.fk_rope(rope, q, k, where, freq, q, k)
        out, stats = torch.empty_like(q), torch.empty((n, H * g, 2), device="cuda")
        max_len = int(ln.max())
        fk.fk_tree_attn(desc, q, K, Vc, ln, k, v, parent, q_start, max(sizes), max_len, scale, out, stats, fk.new_tree_attn_workspace(desc, n, max(sizes), max_len))
        target = torch.softmax(2 * torch.randn((n, V), generator=gen, device="cuda"), -1)
        draft = torch.softmax(target.log() + 0.3 * torch.randn((n, V), generator=gen, device="cuda"), -1)
        tokens = torch.tensor([int(rng.choice(V, p=(w := draft[int(s) + max(p, 0)].double().cpu().numpy()) / w.sum())) for t, s in zip(trees, q_start.tolist()) for p in t], **i32)
        path, count, nxt = torch.empty(n, **i32), torch.empty(B, **i32), torch.empty(B, **i32)
        fk.fk_verify_drafts(target, draft, tokens, parent, q_start, torch.rand(n, generator=gen, device="cuda"), path, count, nxt, verify_ws)
        fk.fk_commit_drafts(desc, K, Vc, pos, ln, acc, k, v, q_start, path, count, at)
        # the same tokens one by one, sequences with shorter paths waiting
        ways = [path[s:s + int(c)].tolist() for s, c in zip(q_start.tolist(), count)]
        total += sum(len(w) for w in ways)
        for i in range(max(len(w) for w in ways)):
            nodes = [q_start[b].item() + (w[i] if i < len(w) else w[-1]) for b, w in enumerate(ways)]
            before = [x.clone() for x in steps]
            got = torch.empty((B, H * g, D), dtype=dt, device="cuda")
            fk.fk_decode_step(desc, q[nodes].contiguous(), *steps, k[nodes].contiguous(), v[nodes].contiguous(), at + i, cap, scale, got, step_ws)
            for b, w in enumerate(ways):
                if i >= len(w):   # not this one's token
                    for x, y in zip(steps, before):
                        x[b] = y[b]
                    continue
                # both round their weights to bf16 at most, of |V| < 6 here, and the output once; fp32: sums of 200 weights and exponents of logits below 32
                allowed = 2 * UB * 6 + 2 * UB * 6 if dtype == "bf16" else (2 * 210 + 4 * 32 * (D + 8)) * U * 6
                assert (out[nodes[b]].float() - got[b].float()).abs().max().item() <= allowed
        live = (torch.arange(cap, device="cuda") < ln[..., None])
        assert torch.equal(ln, steps[3])
        for x, y in zip((K, Vc, pos), steps):
            assert torch.equal(x[live], y[live])
        fresh = live & (torch.arange(cap, device="cuda") >= at[:, None, None])
        assert (acc[fresh] == 0).all()
        at = at + count
    assert total > 2 * B   # something was accepted


def test_other_stream_and_graph():
    import paper_2602_03203_amd as fk
    seqs = [(20, tree(9, 1)), (30, tree(8, depth=0))]
    c = TreeCase("bf16", 64, 2, 2, seqs, seed=4, room=40)
    paths = _paths(seqs, 1)
    path, accepted = _lay(c, paths, [len(p) for p in paths])
    K, V, pos, lens, acc, (pos0, acc0) = _rows(c, paths, [len(p) for p in paths], True, [100, 200])
    d = [x.cuda() for x in (c.K, c.V, pos0, torch.tensor(c.lens), acc0)]
    tail = [x.cuda() for x in (c.k_tree, c.v_tree, c.q_start, path, accepted, torch.tensor([100, 200], dtype=torch.int32))]
    desc = fk.CacheDesc(2, 4, 2, 64, c.cap, "bf16")
    start = [x.clone() for x in d]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    fk.fk_commit_drafts(desc, *d, *tail, stream=side)
    side.synchronize()
    want = (K, V, pos, torch.tensor(lens), acc)
    assert all(_same(x, y) for x, y in zip(d, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fk.fk_commit_drafts(desc, *d, *tail)
    for _ in range(3):
        for x, y in zip(d, start):
            x.copy_(y)
        g.replay()
        torch.cuda.synchronize()
        assert all(_same(x, y) for x, y in zip(d, want))
