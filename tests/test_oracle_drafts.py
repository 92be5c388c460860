"""The oracle of drafted tokens against closed forms: what verification hands on is distributed as the target, whatever the draft is."""
import itertools

import numpy as np
import pytest

from oracle import drafts as od


def test_ancestors():
    parent = [-1, 0, 1, 1, 3, 9, 6, -4]
    assert [od.ancestors(parent, i) for i in range(8)] == [[0], [1, 0], [2, 1, 0], [3, 1, 0], [4, 3, 1, 0], [5], [6], [7]]


def test_a_chain_is_causal_attention():
    rng = np.random.default_rng(0)
    n, T, D = 6, 5, 8
    K, V = rng.standard_normal((2, n + T, D))
    q = rng.standard_normal((T, 1, D))
    out, M, L, _ = od.attend(q, [K[:n]], [V[:n]], [np.ones(n, bool)], K[n:, None], V[n:, None], [-1, 0, 1, 2, 3], 0, 0, 0.5)
    for i in range(T):
        s = K[:n + i + 1] @ q[i, 0] * 0.5
        w = np.exp(s) / np.exp(s).sum()
        assert np.allclose(out[i, 0], w @ V[:n + i + 1])
        assert np.isclose(M[i, 0] * np.log(2) + np.log(L[i, 0]), np.log(np.exp(s).sum()))


def test_turning_keeps_lengths_and_differences():
    """<turned q at i, turned k at j> depends on i - j alone."""
    rng = np.random.default_rng(1)
    freq = 10000.0 ** (-np.arange(0, 8, 2) / 8)
    for layout in ("half", "interleaved"):
        q, k = rng.standard_normal((2, 1, 1, 8))
        dots = [(od.rotate(q, np.array([i]), freq, layout, 8) * od.rotate(k, np.array([i - 5]), freq, layout, 8)).sum() for i in (5, 9, 1000)]
        assert np.ptp(dots) < 1e-9
        assert np.allclose(od.rotate(od.rotate(q, np.array([7]), freq, layout, 8), np.array([7]), freq, layout, 8, inverse=True), q)


@pytest.mark.parametrize("children", [1, 2, 3])
def test_the_first_token_is_distributed_as_the_target(children):
    """All draws of the children and a fine grid of their numbers; the last number enters through the mean over its grid."""
    rng = np.random.default_rng(children)
    p, q = rng.dirichlet(np.ones(3)), rng.dirichlet(np.ones(3))
    parent, grid = [-1] + [0] * children, (np.arange(24 if children > 1 else 400) + 0.5) / (24 if children > 1 else 400)
    target, draft = np.stack([p] * (children + 1)), np.stack([q] * (children + 1))
    law, last = np.zeros(3), (np.arange(60) + 0.5) / 60
    for draws in itertools.product(range(3), repeat=children):
        chance = np.prod(q[list(draws)])
        for us in itertools.product(grid, repeat=children):
            path, _ = od.verify(target, draft, [0, *draws], parent, [0.0, *us])
            weight = chance / grid.size ** children
            if len(path) > 1:
                law[draws[path[1] - 1]] += weight
            else:
                for u in (last if children == 1 else last[::10]):
                    law[od.verify(target, draft, [0, *draws], parent, [u, *us])[1]] += weight / (last if children == 1 else last[::10]).size
    assert np.abs(law - p).max() < (0.03 if children == 1 else 0.12)


def test_the_law_exactly():
    """The same without grids: acceptance probabilities and what is left, by the recursion of the definition, add up to the target."""
    rng = np.random.default_rng(5)
    for _ in range(50):
        V = 6
        p, q = rng.dirichlet(np.ones(V) * 0.5), rng.dirichlet(np.ones(V) * 0.5)
        law, reach, r, c, m = np.zeros(V), 1.0, p.copy(), 0.0, 1.0
        for k in range(4):
            yes = np.minimum(q, r)              # q(x) min(1, r(x) / q(x))
            law += reach * yes
            reach *= 1 - yes.sum()
            r = np.maximum(r - q, 0) / np.maximum(r - q, 0).sum()
            c, m = c + m, np.maximum(p - (c + m) * q, 0).sum()      # the two numbers that the kernel carries
            assert np.allclose(r, np.maximum(p - c * q, 0) / m)
        assert np.allclose(law + reach * r, p)


def test_likeliest_tokens():
    """Drafts that were not drawn: the law is the target's, over the children's numbers."""
    p = np.array([0.5, 0.3, 0.15, 0.05])
    target, grid, law = np.stack([p] * 3), (np.arange(200) + 0.5) / 200, np.zeros(4)
    for a in grid:
        for b in grid[::4]:
            path, _ = od.verify(target, None, [0, 1, 0], [-1, 0, 0], [0.0, a, b])
            if len(path) > 1:
                law[[1, 0][path[1] - 1]] += 1 / (200 * 50)
            else:
                for u in grid[::20]:
                    law[od.verify(target, None, [0, 1, 0], [-1, 0, 0], [u, a, b])[1]] += 1 / (200 * 50 * 10)
    assert np.abs(law - p).max() < 0.02


def test_edges():
    assert od.verify(np.zeros((0, 4)), None, [], [], []) == ([], -1)
    assert od.verify(np.zeros((1, 4)), None, [0], [-1], [0.5]) == ([0], -1)
    assert od.verify(np.array([[0, 1.0, 0, 0]]), None, [0], [-1], [0.999]) == ([0], 1)
    p, q = np.array([[0.5, 0.5]] * 2), np.array([[1.0, 1.0]] * 2)
    assert od.verify(p, q, [0, 1], [-1, 0], [0.6, 0.5]) == ([0], 1)   # nothing is left: the target's own
    assert od.path_of([0, 3, 9, 1], 4, 5) == [0, 3] and od.path_of([0, 1], -1, 5) == [] and od.path_of([0, 1, 2], 9, 2) == [0, 1]
