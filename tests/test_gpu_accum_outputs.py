"""Outputs of the step that accumulates its weights are those of the plain step: head_dim 64 with all bits of the weights, head_dim 128 normalised by the weights
as they meet V; infinities, and rows without any number, as there."""
import numpy as np
import pytest
import torch

from oracle import paged as op
from paged_util import U
from test_gpu_accum import Rows

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _fk():
    import paper_2602_03203_amd as fk
    return fk


# rows of one workgroup of eight wavefronts and of four, and of several splits
@pytest.mark.parametrize("g, hkv, lens", [(1, 2, [0, 1, 15, 31, 32, 63, 200]), (4, 2, [1, 40, 63, 300]), (5, 1, [33, 150]), (8, 2, [20, 129]), (4, 1, [2000, 900]),
                                          (7, 1, [1500]), (3, 2, [700, 33]), (2, 8, [90, 40, 7, 64] * 16)])
def test_head_dim_64_keeps_all_bits_of_the_weights(g, hkv, lens):
    c = Rows("bf16", 64, g, hkv, lens, max(lens) + 5, 2, seed=30 + g)
    s = c.dev()
    c.run(s)
    torch.cuda.synchronize()
    K, V, n = c.K.double().numpy().copy(), c.V.double().numpy().copy(), list(lens)
    got = s["out"].double().cpu().numpy()
    for t in range(c.steps):
        for b in range(len(n)):
            K[b, :, n[b]], V[b, :, n[b]] = c.k[t, b].double().numpy(), c.v[t, b].double().numpy()
            n[b] += 1
            m = n[b]
            q = c.q[t, b].double().numpy()[None]
            out, _, _, W = op.attend(q, K[b, :, :m], V[b, :, :m], np.ones(m, bool), m - 1, 0, 0, c.scale)
            # D products a logit, exponents off by their own and the reference's error, sums of m weights (in fp32 all of it); then one rounding to bf16,
            # half a step of the binade that the value lies in
            mag = np.einsum("hgd,hnd->hgn", np.abs(q[0]).reshape(hkv, g, 64), np.abs(K[b, :, :m])).max(initial=0)
            rel = 2 * np.log(2.0) * ((64 + 4) * U * mag * c.scale / np.log(2.0) + U) + (2 * m + 8) * U
            wv = np.einsum("hgn,hnd->hgd", W[0].reshape(hkv, g, m), np.abs(V[b, :, :m])).reshape(hkv * g, 64)
            near = np.abs(out[0]) + rel * wv + 1e-30
            bad = np.abs(got[t, b] - out[0]) > rel * wv + 2.0 ** (np.floor(np.log2(near)) - 8)
            assert not bad.any(), f"step {t} sequence {b}: {bad.sum()} of {bad.size} off by more than fp32 and one rounding"


@pytest.mark.parametrize("g, hkv, lens", [(1, 1, [31, 63]), (4, 2, [320, 95]), (8, 1, [128]), (4, 1, [2100, 1000]), (5, 1, [1600]), (2, 8, [64, 33] * 32)])
def test_head_dim_128_is_normalised_by_the_rounded_weights(g, hkv, lens):
    """Weights whose rounding to bf16 is nearly half a step up, all of them: values that are all the same come out as they are, with the sum of the same
    rounded weights; with the sum of the unrounded ones 0.3 % off, more than the value's last bit."""
    fk = _fk()
    c = Rows("bf16", 128, g, hkv, lens, max(lens) + 5, 1, seed=1)
    value = 255 / 128          # the largest below 2: half a step is 2^-8, 0.2 % of it
    c.q.zero_()
    c.q[..., 0] = 1
    c.K.zero_()
    c.K[..., 0] = -1
    c.K[:, :, ::32] = 0        # one of every tile is the largest, so all wavefronts' and splits' maxima are the same
    c.k.zero_()
    c.k[..., 0] = -1
    for b, n in enumerate(lens):
        if n % 32 == 0:
            c.k[:, b] = 0
    c.V.fill_(value)
    c.v.fill_(value)
    c.scale = -float(np.log(0.5 * (1 + 1.1 * 2.0 ** -8)))      # the others' weight: 0.5 + 1.1 half steps, rounded to 0.5 + 2
    s = c.dev()
    plain = s["out"].clone()
    K, V, pos, ln = (s[k].clone() for k in ("K", "V", "pos", "len"))
    c.run(s)
    fk.fk_decode_step(s["desc"], s["q"][0], K, V, pos, ln, s["k"][0], s["v"][0], s["pos_new"][0], max(lens) + 1, c.scale, plain[0], fk.new_attn_workspace(s["desc"]))
    torch.cuda.synchronize()
    assert (plain == value).all()
    assert (s["out"] == value).all(), s["out"][s["out"] != value].flatten()[:4]
    # the accumulated weights are those of the unrounded exponentials
    w = 0.5 * (1 + 1.1 * 2.0 ** -8)
    for b, n in enumerate(lens):
        x = np.where(np.arange(n + 1) % 32 == 0, 1.0, w)
        want = c.acc[b, :, :n + 1].double().numpy().copy()
        want[:, n] = 0
        want += g * x / x.sum()
        assert (np.abs(s["acc"][b, :, :n + 1].double().cpu().numpy() - want) <= (2 * n + 40) * U * g * x / x.sum() + 4 * g * U * want).all()


@pytest.mark.parametrize("dtype, D", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("n", [90, 160, 1500])
@pytest.mark.parametrize("g", [1, 4, 7])
def test_infinite_values(dtype, D, n, g):
    """A pair of weight p > 0 gives p * inf = inf in its channel, every other channel is what it is without it; of cached and of new pairs."""
    c = Rows(dtype, D, g, 2, [n, n - 3], n + 20, 8, seed=n + g)
    c.K[0, 1, 45] = 4.0 * c.q[3, 0, g]       # the largest weight of a row: nothing is left for a remainder
    cached = [(0, 1, 45, 17, INF), (0, 1, 46, 18, -INF), (0, 1, 47, 19, NAN), (1, 0, 5, 3, INF), (1, 0, 70, 4, -INF), (1, 0, 71, 3, INF)]
    fresh = [(2, 0, 0, 17, INF), (2, 0, 0, 18, -INF), (3, 0, 0, 19, NAN), (5, 1, 1, 3, -INF)]
    runs = []
    for bad in (True, False):
        for b, h, slot, ch, x in cached:
            c.V[b, h, slot, ch] = x if bad else 0
        for t, b, h, ch, x in fresh:
            c.v[t, b, h, ch] = x if bad else 0
        s = c.dev()
        c.run(s)
        torch.cuda.synchronize()
        runs.append((s["out"].float().cpu(), s["acc"].cpu()))
    (o, acc), (r, acc_r) = runs
    places = [(0, b, h, ch, x) for b, h, _, ch, x in cached] + fresh
    for t, b, h, ch, x in places:
        got = o[t:, b, h * g:(h + 1) * g, ch]
        assert bool(torch.isnan(got).all() if x != x else (got == x).all()), f"row ({b},{h}) channel {ch} from step {t}: {got.flatten()[:4]} for {x}"
    for t, b, h, ch, _ in places:
        o[t:, b, h * g:(h + 1) * g, ch] = r[t:, b, h * g:(h + 1) * g, ch]
    assert torch.equal(o, r) and torch.equal(acc[:, :, :n], acc_r[:, :, :n])


@pytest.mark.parametrize("dtype, D", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("n", [40, 1500])
def test_rows_without_any_number(dtype, D, n):
    """All logits of a head -inf: 0 / 0, as in the plain step; other heads have their results."""
    fk = _fk()
    c = Rows(dtype, D, 4, 2, [n, n - 7], n + 5, 1, seed=5)
    c.K[0, 0, :, 3], c.k[0, 0, 0, 3] = -INF, -INF
    c.q[0, 0, :4, 3] = torch.tensor([1.0, 0.5, 2.0, 1.0]).to(DT[dtype])
    s = c.dev()
    plain, K, V, pos, ln = s["out"].clone(), s["K"].clone(), s["V"].clone(), s["pos"].clone(), s["len"].clone()
    c.run(s)
    fk.fk_decode_step(s["desc"], s["q"][0], K, V, pos, ln, s["k"][0], s["v"][0], s["pos_new"][0], n + 1, c.scale, plain[0], fk.new_attn_workspace(s["desc"]))
    torch.cuda.synchronize()
    assert torch.isnan(plain[0, 0, :4]).all() and torch.isfinite(plain[0, 0, 4:]).all() and torch.isfinite(plain[0, 1]).all()
    assert torch.equal(torch.isnan(s["out"]), torch.isnan(plain))
    assert torch.isnan(s["acc"][0, 0, :n + 1]).all() and torch.isfinite(s["acc"][0, 1]).all() and torch.isfinite(s["acc"][1]).all()
