"""(M, L) of the paged attention and the weights formed with them: the same from both kernels, whatever the logits are."""
import copy

import numpy as np
import pytest
import torch

from paged_util import U, Case
from test_gpu_paged_prompt import TYPES, _case

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def _attended(c):
    s = c.dev()
    c.run(s)
    torch.cuda.synchronize()
    return s, s["out"].double().cpu().numpy(), s["stats"].double().cpu().numpy()


@pytest.mark.parametrize("dtype, D", TYPES)
@pytest.mark.parametrize("many_rows", [True, False])
@pytest.mark.parametrize("window", [0, 20])
def test_a_query_without_numbers_has_a_sum_without_one(dtype, D, many_rows, window):
    """(-inf, 0) says that a query sees nothing; one that sees pairs and is no number has NaN in its results and in L."""
    make = _case if many_rows else Case
    c = make(dtype, D, 4, 1, 16, [(90, 40), (200, 150), (33, 1), (3, 10)], window, 2, seed=54)
    c.q[13, 2, 5] = NAN
    c.q[60], c.q[190, 3, 1] = NAN, NAN     # (190: the single token)
    c.q[192] = NAN                          # before the first position: sees nothing
    s, out, stats = _attended(c)
    ref, _ = c.reference()
    seen = ref["L"] > 0
    want = np.isnan(ref["L"])
    assert want[13, 2] and want[60].all() and want[190, 3] and want.sum() == 6 and not want[192].any()
    assert (np.isnan(stats[..., 1]) == want).all() and (np.isnan(out).all(axis=2) == want).all() and (np.isnan(out).any(axis=2) == want).all()
    none = ~seen & ~want
    assert none[191:198].all() and (stats[none] == [-INF, 0]).all() and (out[none] == 0).all()


@pytest.mark.parametrize("dtype, D", TYPES)
@pytest.mark.parametrize("chunks", [[(2600, 20)], [(3000, 1), (2111, 40)], [(2900, 1)]])
def test_splits_without_numbers(dtype, D, chunks):
    """NaN keys over a whole split of a tile's pairs, beside splits of finite ones: sums, results and received weights of the head that meets them are NaN."""
    c = _case(dtype, D, 4, 2, 64, chunks, seed=41)
    for b in range(len(chunks)):
        for page in range(16):
            c.K[int(c.table[b, page]), 0] = NAN       # pairs 0 .. 1023 of head 0
    s, out, stats = _attended(c)
    assert np.isnan(out[:, :4]).all() and np.isnan(stats[:, :4, 1]).all()
    assert np.isfinite(out[:, 4:]).all() and np.isfinite(stats[:, 4:]).all()
    acc = s["acc"].cpu()
    for b, (n, _) in enumerate(chunks):
        assert torch.isnan(acc[b, 0, :n]).all() and torch.isfinite(acc[b, 1]).all()


@pytest.mark.parametrize("dtype, D", TYPES)
@pytest.mark.parametrize("many_rows", [True, False])
def test_a_scale_without_a_number(dtype, D, many_rows):
    c = (_case if many_rows else Case)(dtype, D, 4, 1, 16, [(30, 1), (60, 20)], scale=NAN, seed=53)
    _, out, stats = _attended(c)
    assert np.isnan(out).all() and np.isnan(stats[..., 1]).all()


@pytest.mark.parametrize("dtype, D", TYPES)
@pytest.mark.parametrize("many_rows", [True, False])
def test_logits_of_minus_infinity_alone(dtype, D, many_rows):
    """As where nothing is seen: zeros and (-inf, 0), no weight for anyone."""
    c = (_case if many_rows else Case)(dtype, D, 4, 2, 16, [(100, 40), (33, 1)], seed=55)
    for page in range(7):
        c.K[int(c.table[0, page]), 0, :, 3] = -INF
    c.k_new[:40, 0, 3] = -INF
    c.q[:40, :4, 3] = 1.0
    c.q[7, 2, 3] = -1.0          # +inf among them: no number
    s, out, stats = _attended(c)
    nan = np.zeros(out.shape[:2], bool)
    nan[7, 2] = True
    assert (np.isnan(stats[..., 1]) == nan).all() and (np.isnan(out).all(axis=2) == nan).all()
    none = ~nan[:40, :4]
    assert (out[:40, :4][none] == 0).all() and (stats[:40, :4][none] == [-INF, 0]).all()
    assert (stats[:40, 4:, 1] > 0).all() and (stats[40:, :, 1] > 0).all()
    acc = s["acc"].cpu()
    assert torch.isnan(acc[0, 0, :68]).all() and (acc[0, 0, 68:100] == 0).all()      # (token 7 is at position 67)


@pytest.mark.parametrize("dtype, D", TYPES)
@pytest.mark.parametrize("log_scale", [4, 7, 10, 14, 18, 20, 21])
@pytest.mark.parametrize("many_rows", [True, False])
def test_a_querys_weights_add_up_to_one(dtype, D, log_scale, many_rows):
    """Whatever the logits' size, weights are taken against the maximum and the sum that the attention found, by the same exponents: a query's weights add up to
    one.  Logits of up to about 2^3 times the scale here (times sqrt(64 .. 128))."""
    chunks = [(200, 60), (333, 1), (90, 17), (70, 70)]
    c = (_case if many_rows else Case)(dtype, D, 4, 2, 16, chunks, scale=2.0 ** log_scale / 8, seed=60 + log_scale)
    s, out, stats = _attended(c)
    top = np.abs(stats[..., 0]).max()
    assert 2.0 ** log_scale < top < 2.0 ** (log_scale + 7)
    acc, first = s["acc"].double().cpu().numpy(), c.acc.double().numpy()
    for b, (n, m) in enumerate(chunks):
        gained = (acc[b, :, :n].sum(axis=1) - first[b, :, :n - m].sum(axis=1)) / (4 * m)
        # Exponents of attention and weights: the same logits, rounded or not - below 2^8 the rounding is 2^-17 at most, each side once, times ln 2; sums of n weights of
        # 4 m queries, two steps an exponential and a reciprocal; the pairs' earlier sums, up to n of up to 1 with a rounding for each addition
        tol = 2 * 2.0 ** -17 * np.log(2.0) + (n + 4 * m + 16) * U + 2 * n * U / (4 * m)
        assert (np.abs(gained - 1) <= tol).all(), (b, gained - 1, tol, top)


@pytest.mark.parametrize("dtype, D", TYPES)
@pytest.mark.parametrize("log_scale", [7, 18, 21])
def test_both_kernels_report_the_same(dtype, D, log_scale):
    """One call by its bound few rows' and many rows': maxima bit for bit, sums as near as fp32 sums are."""
    chunks = [(200, 60), (90, 17), (70, 70)]
    few = Case(dtype, D, 4, 2, 16, chunks, scale=2.0 ** log_scale / 8, seed=70)
    many = copy.copy(few)
    many.max_pages = (1 << 21) // (147 * 4 // 16 * 2) // 16 + 1
    many.table = torch.nn.functional.pad(few.table, (0, many.max_pages - few.max_pages), value=-1)
    many.acc = torch.nn.functional.pad(few.acc, (0, (many.max_pages - few.max_pages) * 16))
    many.max_len = many.max_pages * 16
    (_, o1, s1), (_, o2, s2) = _attended(few), _attended(many)
    assert (s1[..., 0] == s2[..., 0]).all()
    # exponents below 2^8 may be off by a logit's rounding, 2^-17 at most, in either
    assert (np.abs(s1[..., 1] - s2[..., 1]) <= s1[..., 1] * (2 * 2.0 ** -17 * np.log(2.0) + (2 * 200 + 8) * U)).all()
