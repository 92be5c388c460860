"""Pins of the oracle of the paged prompt cache: closed forms, and agreement with the C oracle of the decode step."""
import numpy as np
import pytest

from oracle import paged as op


def _rand(shape, seed):
    return np.random.default_rng(seed).standard_normal(shape)


@pytest.mark.parametrize("p, window, sink, want", [(5, 0, 0, [0, 1, 2, 3, 4, 5]), (5, 2, 0, [4, 5]), (5, 2, 1, [0, 4, 5]), (5, 1, 9, [0, 1, 2, 3, 4, 5]),
                                                   (0, 3, 0, [0]), (-1, 0, 4, []), (5, 100, 0, [0, 1, 2, 3, 4, 5])])
def test_visible_pairs(p, window, sink, want):
    assert np.flatnonzero(op.visible(p, 8, window, sink, np.ones(8, bool))).tolist() == want
    hole = np.ones(8, bool)
    hole[4:] = False
    assert np.flatnonzero(op.visible(p, 8, window, sink, hole)).tolist() == [j for j in want if j < 4]


def test_pairs_follow_the_page_table():
    pool = _rand((5, 2, 4, 3), 0)
    x, present = op.pairs(pool, np.array([3, -1, 5, 0]), 14)
    assert np.array_equal(x[:, :4], pool[3]) and np.array_equal(x[:, 12:14], pool[0][:, :2])
    assert present.tolist() == [True] * 4 + [False] * 8 + [True] * 2


def test_one_pair_and_identical_keys():
    q, V = _rand((3, 4, 8), 1), _rand((2, 3, 8), 2)
    K = np.broadcast_to(_rand((2, 1, 8), 3), (2, 3, 8))
    out, M, L, W = op.attend(q, K, V, np.ones(3, bool), 0, 0, 0, 0.3)
    for t in range(3):
        assert np.allclose(out[t].reshape(2, 2, 8), V[:, None, :t + 1].mean(axis=2)) and np.allclose(L[t], t + 1)
    assert np.allclose(M, np.einsum("thgd,hd->thg", q.reshape(3, 2, 2, 8), K[:, 0]).reshape(3, 4) * 0.3 / np.log(2))


def test_chunk_equals_the_c_oracle_step_by_step(ora):
    """Every token of a chunk is a decode step of the C oracle on the pairs up to it."""
    H, g, D, n, c = 2, 3, 64, 40, 5
    q = _rand((c, H * g, D), 4).astype(np.float32)
    K, V = _rand((H, n, D), 5).astype(np.float32), _rand((H, n, D), 6).astype(np.float32)
    out, _, _, W = op.attend(q.astype(np.float64), K.astype(np.float64), V.astype(np.float64), np.ones(n, bool), n - c, 0, 0, 0.2)
    for t in range(c):
        m = n - c + t + 1
        pos = np.broadcast_to(np.arange(n, dtype=np.int32), (1, H, n)).copy()
        cache = ora.Cache("f32", K[None].copy(), V[None].copy(), pos, np.array([m], np.int32))
        assert np.allclose(ora.decode_attn(cache, q[None, t], 0.2)[0], out[t], atol=1e-12)
    assert np.allclose(W.sum(axis=2), 1)
    assert np.allclose(op.received(W, H).sum(axis=1), c * g)        # a group's queries give one unit each


def test_accumulated_weights_start_from_zero_and_add():
    W = np.zeros((2, 2, 4))
    W[0, :, :3], W[1, :, :4] = 1 / 3, 1 / 4
    acc = op.accumulate(np.full((1, 4), 5.0), W, 1, 2)
    assert np.allclose(acc, [[5 + 2 / 3 + 0.5, 5 + 2 / 3 + 0.5, 2 / 3 + 0.5, 0.5]])


def test_nothing_seen():
    out, M, L, W = op.attend(_rand((2, 2, 4), 0), _rand((1, 1, 4), 1), _rand((1, 1, 4), 2), np.zeros(1, bool), 0, 0, 0, 1.0)
    assert (out == 0).all() and (M == -np.inf).all() and (L == 0).all() and (W == 0).all()
