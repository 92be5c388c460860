"""Verification of drafted tokens against the oracle: equal paths and tokens."""
import numpy as np
import pytest
import torch

from drafts_util import tree
from oracle import drafts as od

pytestmark = pytest.mark.gpu


class Trees:
    def __init__(self, trees, vocab, drawn=True, noise=0.5, seed=0, before=0, behind=0, sharp=2.0):
        rng = np.random.default_rng(seed)
        self.trees, self.vocab = trees, vocab
        sizes = [len(t) for t in trees]
        self.q_start = (before + np.concatenate([[0], np.cumsum(sizes)])).astype(np.int32)
        self.n = int(self.q_start[-1]) + behind
        z = sharp * rng.standard_normal((self.n, vocab))
        soft = lambda z: (np.exp(z - z.max(-1, keepdims=True)) / np.exp(z - z.max(-1, keepdims=True)).sum(-1, keepdims=True)).astype(np.float32)   # noqa: E731
        self.target, self.draft = soft(z), soft(z + noise * rng.standard_normal((self.n, vocab))) if drawn else None
        self.parent = np.full(self.n, 7, np.int32)
        self.tokens = rng.integers(0, vocab, self.n).astype(np.int32)
        for t, s in zip(trees, self.q_start):
            self.parent[s:s + len(t)] = t
            for i, p in enumerate(t):
                if 0 <= p < i:
                    if drawn:
                        w = self.draft[s + p].astype(np.float64)
                        self.tokens[s + i] = rng.choice(vocab, p=w / w.sum())
                    else:   # the likeliest ones, one after the other
                        order = np.argsort(-self.target[s + p] * np.exp(noise * rng.standard_normal(vocab)))
                        self.tokens[s + i] = order[sum(1 for x in t[:i] if x == p) % vocab]
        self.uniform = rng.random(self.n).astype(np.float32)

    def reference(self):
        path, count, following = np.full(self.n, -9, np.int32), [], []
        for b, t in enumerate(self.trees):
            s = slice(self.q_start[b], self.q_start[b + 1])
            way, x = od.verify(self.target[s].astype(np.float64), None if self.draft is None else self.draft[s].astype(np.float64), self.tokens[s], self.parent[s],
                               self.uniform[s].astype(np.float64))
            if len(t) <= od.MOST_NODES:
                path[s] = way + [-1] * (len(t) - len(way))
            count.append(len(way))
            following.append(x)
        return path, np.array(count, np.int32), np.array(following, np.int32)

    def dev(self):
        import paper_2602_03203_amd as fk
        c = lambda x: None if x is None else torch.tensor(x).cuda()   # noqa: E731
        return [c(self.target), c(self.draft), c(self.tokens), c(self.parent), c(self.q_start), c(self.uniform), torch.full((self.n,), -9, dtype=torch.int32, device="cuda"),
                torch.full((len(self.trees),), -9, dtype=torch.int32, device="cuda"), torch.full((len(self.trees),), -9, dtype=torch.int32, device="cuda"),
                fk.new_verify_workspace(len(self.trees), self.vocab)]

    def check(self, d, what=""):
        for got, want, name in zip(d[6:9], self.reference(), ("path", "accepted", "next")):
            assert np.array_equal(got.cpu().numpy(), want), f"{what} {name}: {got.cpu().numpy()} not {want}"

    def go(self, what=""):
        import paper_2602_03203_amd as fk
        d = self.dev()
        for turn in range(2):   # (the counters are at zero again behind a call)
            for x in d[6:9]:
                x.fill_(-9)
            fk.fk_verify_drafts(*d)
            torch.cuda.synchronize()
            self.check(d, f"{what} {turn}")
        return d


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("vocab", [1, 2, 3, 5, 63, 64, 65, 257, 1000, 2047, 2048, 2049, 5003, 33333])
def test_vocabularies(drawn, vocab):
    Trees([tree(n, n) for n in (1, 2, 3, 5, 9, 17)] + [tree(6, depth=0), []] + [tree(12, s, depth=2) for s in range(4)], vocab, drawn, seed=vocab, before=2, behind=3).go()


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("noise", [0.0, 0.2, 1.0, 4.0])
@pytest.mark.parametrize("sharp", [0.3, 3.0])
def test_many_trees(drawn, noise, sharp):
    """Nearly equal and very different distributions: paths of all lengths, rejections among many children."""
    for seed in range(3):
        c = Trees([tree(40, s, depth=3, fan=40) for s in range(20)] + [tree(12, depth=0) for _ in range(20)] + [[-1] + [0] * 30 for _ in range(10)], 300, drawn, noise, seed, sharp=sharp)
        c.go(f"seed {seed}")
    if noise == 0.2 and drawn:
        assert len(set(c.reference()[1])) > 3


@pytest.mark.parametrize("drawn", [True, False])
def test_large_trees_and_large_vocabularies(drawn):
    Trees([tree(256, 1), tree(255, 2, depth=2, fan=255), tree(65, 3), tree(257, 4), tree(64, depth=0)], 700, drawn, 1.0, seed=5).go()
    Trees([tree(9, 1, depth=2), tree(3, 2)], 200001, drawn, 1.0, seed=6).go()
    Trees([[-1, 0]], 1 << 21, drawn, 1.0, seed=7).go()


def test_equal_distributions_accept_everything():
    """draft = target: a drawn token is accepted whatever its number is (0 <= u < 1)."""
    c = Trees([tree(20, depth=0) for _ in range(8)], 500, noise=0.0)
    c.draft = c.target.copy()
    c.uniform[:] = 1 - 2.0 ** -24
    d = c.go()
    assert (d[7] == 20).all()


def test_special_rows():
    """Nothing left of r: target's own row; nothing at all: -1; negative numbers and NaN count as nothing; tokens outside; the first and the last number."""
    V = 130
    c = Trees([[-1, 0, 0], [-1, 0], [-1, 0], [-1], [-1, 0, 0], [-1], [-1], [-1, 0]], V, seed=3)
    s = c.q_start
    p, q = c.target, c.draft
    q[s[0]] = 2 * p[s[0]]                                # every child rejected (u = 1/2 and more), nothing is left of r
    c.uniform[s[0] + 1:s[1]] = 0.75
    p[s[1]] = 0                                          # no mass
    p[s[2]], q[s[2]] = -1, 0.5
    p[s[2], 17] = 0.25
    c.tokens[s[2] + 1] = 18
    p[s[3]] = float("nan")
    p[s[3], 5], p[s[3], 9] = 1e-30, 1e-30
    c.tokens[s[4] + 1], c.tokens[s[4] + 2] = -1, V       # outside
    p[s[5]] = 0
    p[s[5], V - 1], c.uniform[s[5]] = 1.0, 0.0
    p[s[6]] = 0
    p[s[6], 0], c.uniform[s[6]] = 1.0, 1 - 2.0 ** -24
    c.tokens[s[7] + 1], c.uniform[s[7] + 1], c.uniform[s[7]] = int(np.argmax(p[s[7]])), 0.0, 0.0
    d = c.go()
    assert d[8].tolist()[1:4] == [-1, 17, 5 if c.uniform[s[3]] < 0.5 else 9] and d[8].tolist()[5:7] == [V - 1, 0] and d[7].tolist()[7] == 2
    c.draft = None
    c.go("likeliest")


def test_the_same_token_twice():
    """Likeliest tokens: a second child with a rejected token is rejected and nothing is taken off twice."""
    c = Trees([[-1] + [0] * 6 for _ in range(60)], 8, False, seed=2, sharp=0.5)
    c.tokens[:] = np.tile([0, 1, 1, 2, 1, 2, 3], 60)
    c.go()


def test_equal_calls_other_stream_and_graphs():
    import paper_2602_03203_amd as fk
    a = Trees([tree(30, s, depth=3, fan=30) for s in range(6)], 40001, True, 1.5, seed=1)
    b = Trees([tree(30, s, depth=3, fan=30) for s in range(6)], 40001, True, 1.5, seed=2)
    da, db = a.dev(), b.dev()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    fk.fk_verify_drafts(*da, stream=side)
    side.synchronize()
    a.check(da)
    db[9] = da[9]   # one workspace
    graphs = []
    for d in (da, db):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            fk.fk_verify_drafts(*d)
        graphs.append(g)
    keep = [x.clone() for x in da[:6]]
    for turn in range(4):
        for x in da[6:9] + db[6:9]:
            x.fill_(-9)
        graphs[turn % 2].replay()
        graphs[1 - turn % 2].replay()
        torch.cuda.synchronize()
        (a if turn % 2 == 0 else b).check(da, f"replay {turn}")
        b.check(db, f"replay {turn}")
        for x, y, z in zip(da[:6], db[:6], keep):
            x.copy_(y if turn % 2 == 0 else z)


def test_rows_beyond_32_bit_offsets():
    """n_tokens * vocab beyond 2^31: the row of the last node."""
    import paper_2602_03203_amd as fk
    V, n = (1 << 23) + 1, 260
    target = torch.zeros((n, V), device="cuda")
    target[n - 2, 12345], target[n - 1, V - 2] = 1.0, 1.0
    target[255 + 3, 12345] = 1.0
    i32 = dict(dtype=torch.int32, device="cuda")
    q_start = torch.tensor([n - 2, n], **i32)
    tokens, parent = torch.full((n,), 12345, **i32), torch.zeros(n, **i32)
    path, acc, nxt = torch.zeros(n, **i32), torch.zeros(1, **i32), torch.zeros(1, **i32)
    fk.fk_verify_drafts(target, None, tokens, parent, q_start, torch.full((n,), 0.5, device="cuda"), path, acc, nxt, fk.new_verify_workspace(1, V))
    assert acc.item() == 2 and nxt.item() == V - 2 and path[n - 2:].tolist() == [0, 1]


def test_calls_of_any_sizes_share_a_workspace():
    """Other batches and vocabularies in turns: a sum of an earlier call is never taken for one of this call."""
    import paper_2602_03203_amd as fk
    cases = [Trees([tree(20, s, depth=2, fan=20) for s in range(b)], v, drawn, 1.5, seed=b) for b, v, drawn in ((3, 9001, True), (7, 40000, True), (1, 130001, True), (5, 9001, False), (2, 5000, True))]
    devs = [c.dev() for c in cases]
    ws = torch.zeros(max(d[9].numel() for d in devs), dtype=torch.uint8, device="cuda")
    for turn in range(4):
        for d in devs:
            for x in d[6:9]:
                x.fill_(-9)
            fk.fk_verify_drafts(*d[:9], ws)
        torch.cuda.synchronize()
        for i, (c, d) in enumerate(zip(cases, devs)):
            c.check(d, f"turn {turn} case {i}")


def test_more_rejections_than_sums_are_told():
    """Sixty children of one node, all rejected: the first sums are shared, the others everybody forms."""
    c = Trees([[-1] + [0] * 60 for _ in range(3)], 20000, True, 0.3, seed=4)
    c.uniform[:] = 1 - 2.0 ** -24
    d = c.go()
    assert d[7].max().item() >= 1
    c.tokens[:] = 5   # (and the same token every time, which the draft likes better than the target)
    c.target[:, 5] *= 0.5
    c.go()


@pytest.mark.parametrize("vocab", [130, 5003, 40001])
def test_draft_rows_that_play_no_part(vocab):
    """Nobody drew from the row of a node without children, which may hold anything; nor does a draft's row count where nothing was rejected, or where nothing is left of r
    and the target's own row takes its place."""
    c = Trees([[-1], [-1], [-1, 0, 0, 1], [-1, 0, 1, 2], [-1, 0], [-1, -1], tree(30, 1, depth=3)], vocab, seed=vocab, sharp=1.0)
    s, p, q = c.q_start, c.target, c.draft
    with_children = {s[b] + x for b, t in enumerate(c.trees) for x in t if x >= 0}
    leaves = [i for i in range(c.n) if i not in with_children]
    q[leaves] = np.nan
    q[leaves[::2], ::3] = np.inf
    q[leaves[::3], 1::2] = -np.inf
    c.uniform[s[3]:s[4]] = 0.0                           # a chain, all accepted: its leaf's row is the target's
    keep = int(c.tokens[s[4] + 1])
    q[s[4]] = 2 * p[s[4]]                                # nothing is left: the target's own row, infinities of the draft or not
    q[s[4], [x for x in range(0, vocab, 7) if x != keep]] = np.inf
    c.uniform[s[4] + 1] = 0.75
    for u in (0.0, 0.3, 0.999):
        c.uniform[s[:-1]] = u
        path, count, following = c.reference()
        assert count[3] == 4 and count[4] == 1 and (following >= 0).all()
        c.go(f"u {u}")


@pytest.mark.parametrize("vocab", [700, 5003, 40001])
def test_many_rejections_before_an_acceptance(vocab):
    """Sixty different children of the root, then two hundred, are rejected before one is accepted or none is: c and m, carried from sum to sum, decide about each one behind them."""
    rng = np.random.default_rng(vocab)
    wide = [60, 200, 60, 200, 60, 200]
    c = Trees([[-1] + [0] * (n + 20) for n in wide], vocab, True, seed=vocab)
    c.uniform[:] = rng.random(c.n)
    for b, n in enumerate(wide):
        s = int(c.q_start[b])
        picked = rng.permutation(vocab)[:n + 20]
        likely, others = picked[:n], picked[n:]   # the draft likes the first ones far better than the target, the others a little
        p, q = rng.dirichlet(np.ones(vocab)), rng.random(vocab)
        share = 0.9 / n
        p[likely] = 0.1 * share * rng.random(n)
        p /= p.sum()
        q = p * np.exp(2 * rng.standard_normal(vocab)) * 0.7 / n
        q[likely] = share
        c.target[s], c.draft[s] = p, q / q.sum()
        c.tokens[s + 1:s + 1 + n], c.tokens[s + 1 + n:s + 21 + n] = likely, others
        c.uniform[s + 1:s + 1 + n] = 0.9 + 0.09 * rng.random(n)
        if b >= 4:
            c.target[s, others] = 0   # nobody is accepted
    path, count, _ = c.reference()
    rejected = [int(path[s + 1]) - 1 if k > 1 else n + 20 for s, k, n in zip(c.q_start, count, wide)]
    assert min(rejected[::2]) >= 60 and min(rejected[1::2]) >= 200 and 2 in count and (count[4:] == 1).all() and max(r - n for r, n in zip(rejected[:4], wide)) > 0, rejected
    d = c.go()
    if vocab > 4096:   # every workgroup's sums of every rejection are told, two words each, and none is formed by everybody again
        assert int(d[9][256:].view(torch.int64).count_nonzero()) >= 2 * 2 * sum(rejected)
