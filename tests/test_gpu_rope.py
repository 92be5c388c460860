"""Rotary positions against the oracle: layouts, parts of the head, strides, far positions, in place, there and back."""
import numpy as np
import pytest
import torch

from oracle import drafts as od

pytestmark = pytest.mark.gpu

U, UB = 2.0 ** -24, 2.0 ** -8


def _fk():
    import paper_2602_03203_amd as fk
    return fk


def _allowed(x, y, pos, freq, layout, rot, magnitude, dtype):
    """Turns are formed by three roundings in 64 bits and one to 32 (half a turn: pi u); sine and cosine are within four steps each, the products and their sum
    round three times: 16 u in all of magnitude (|u| + |w|), and the output's rounding."""
    half = U if dtype == "f32" else UB
    e = np.zeros_like(x)
    a = np.abs(pos.astype(np.float64)[:, None] * freq[None]) * 2.0 ** -50 + 16 * U
    for i in range(rot // 2):
        u, w = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
        m = magnitude * (np.abs(x[:, :, u]) + np.abs(x[:, :, w])) * a[:, i, None]
        e[:, :, u], e[:, :, w] = m, m
    e[:, :, :rot] += half * (np.abs(y[:, :, :rot]) + e[:, :, :rot])
    return e


def _case(dtype, D, rot, layout, hq, hkv, n, pos=None, strides=None, inplace=False, magnitude=1.0, inverse=False, scaling=("none", {}), seed=0, base=1e6):
    fk = _fk()
    gen = torch.Generator().manual_seed(seed)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    pad = strides or [0, 0, 0, 0]

    def make(heads, extra):
        x = torch.randn((n, heads * D + extra), generator=gen).to(dt).cuda()
        return x, x[:, :heads * D].unflatten(1, (heads, D))
    (qb, q), (kb, k) = make(hq, pad[0]), make(hkv, pad[1])
    if inplace:
        qo, ko, qob, kob = q, k, qb, kb
    else:
        (qob, qo), (kob, ko) = make(hq, pad[2]), make(hkv, pad[3])
    if pos is None:
        pos = torch.randint(0, 40000, (n,), generator=gen, dtype=torch.int32)
    freq = fk.rope_frequencies(rot, base, scaling[0], **scaling[1])
    x, before = [t.double().cpu().numpy() for t in (q, k)], [qob.clone(), kob.clone()]
    desc = fk.RopeDesc(hq, hkv, D, rot, layout, dtype, magnitude, inverse)
    fk.fk_rope(desc, q, k, pos.cuda(), freq.cuda(), qo, ko)
    torch.cuda.synchronize()
    for a, y, whole, was, heads in ((x[0], qo, qob, before[0], hq), (x[1], ko, kob, before[1], hkv)):
        ref = od.rotate(a, pos.numpy(), freq.numpy(), layout, rot, magnitude, inverse)
        got = y.double().cpu().numpy()
        tol = _allowed(a, ref, pos.numpy(), freq.numpy(), layout, rot, magnitude, dtype)
        bad = np.abs(got - ref) > tol
        assert not bad.any(), f"{bad.sum()} of {bad.size} off, worst {np.abs(got - ref)[bad].max()}"
        assert torch.equal(whole[:, heads * D:], was[:, heads * D:]), "written between the tokens"
    return q, k, qo, ko


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("D, rot", [(64, 64), (64, 32), (64, 2), (64, 48), (64, 62), (64, 6), (128, 128), (128, 64), (128, 96), (128, 112), (128, 50), (128, 8), (128, 4)])
def test_layouts_and_parts_of_the_head(dtype, layout, D, rot):
    _case(dtype, D, rot, layout, 8, 2, 7, seed=rot)
    _case(dtype, D, rot, layout, 3, 1, 5, inplace=True, seed=rot)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 2, 3, 63, 257, 2047, 2048, 2049, 4099])
@pytest.mark.parametrize("hq, hkv, rot", [(4, 1, 128), (5, 5, 40), (32, 8, 128)])
def test_numbers_of_tokens(dtype, n, hq, hkv, rot):
    _case(dtype, 128, rot, "half", hq, hkv, n, seed=n)
    _case(dtype, 128, rot, "interleaved", hq, hkv, n, seed=n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rot, layout", [(64, "half"), (64, "interleaved"), (34, "half")])
@pytest.mark.parametrize("inplace", [False, True])
def test_strides(dtype, rot, layout, inplace):
    pad = [64, 8, 64, 8] if inplace else [128, 640, 8, 24]
    for n in (1, 9, 2500):
        _case(dtype, 64, rot, layout, 6, 2, n, strides=pad, inplace=inplace, seed=n)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_far_positions(layout):
    """Every kind of int32: the slowest and the fastest pairs keep their angles."""
    pos = torch.tensor([0, 1, -1, 2 ** 20 + 1, 2 ** 24 + 3, 2 ** 31 - 1, -2 ** 31, -12345678], dtype=torch.int32)
    for dtype in ("f32", "bf16"):
        _case(dtype, 128, 128, layout, 2, 1, 8, pos=pos)


@pytest.mark.parametrize("scaling", [("linear", dict(factor=8.0)), ("base", dict(factor=4.0)), ("parts", dict(factor=4.0, context=32768, low=1.0, high=32.0))])
def test_scaled_and_magnified(scaling):
    _case("f32", 128, 128, "half", 4, 2, 33, scaling=scaling, magnitude=1.1386, base=10000.0)
    _case("bf16", 64, 40, "interleaved", 4, 2, 33, scaling=scaling, magnitude=0.5, base=10000.0, inverse=True)


def test_there_and_back():
    """The inverse turns back: twice three roundings in fp32."""
    fk = _fk()
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, k = torch.randn((300, 4, 128), generator=gen, device="cuda"), torch.randn((300, 2, 128), generator=gen, device="cuda")
    pos, freq = torch.arange(300, dtype=torch.int32, device="cuda") * 7919, fk.rope_frequencies(96, 5e5).cuda()
    y, z, ky, kz = torch.empty_like(x), torch.empty_like(x), torch.empty_like(k), torch.empty_like(k)
    fk.fk_rope(fk.RopeDesc(4, 2, 128, 96, "half", "f32"), x, k, pos, freq, y, ky)
    fk.fk_rope(fk.RopeDesc(4, 2, 128, 96, "half", "f32", inverse=True), y, ky, pos, freq, z, kz)
    # each way 16 u of |u| + |w| <= sqrt(2) times the pair's length, which turning keeps
    length = (x[..., :48] ** 2 + x[..., 48:96] ** 2).sqrt()
    for part in (slice(0, 48), slice(48, 96)):
        assert ((z - x)[..., part].abs() <= 2 * 17 * U * 2 ** 0.5 * length).all()
    assert torch.equal(z[..., 96:], x[..., 96:])


def test_gradient():
    """The gradient of sum(turned * w) is w turned back, against the oracle's differences: turning is linear, so they are exact in 64 bits."""
    fk = _fk()
    rng = np.random.default_rng(0)
    for layout, mag in (("half", 1.0), ("interleaved", 1.3)):
        x, w = rng.standard_normal((3, 2, 64)), rng.standard_normal((3, 2, 64)).astype(np.float32)
        pos, freq = np.array([5, 1000, 70000], np.int32), fk.rope_frequencies(32, 1e4)
        loss = lambda x: (od.rotate(x, pos, freq.numpy(), layout, 32, mag) * w).sum()   # noqa: E731,B023
        g = torch.empty((3, 2, 64), device="cuda")
        fk.fk_rope(fk.RopeDesc(2, 0, 64, 32, layout, "f32", mag, inverse=True), torch.tensor(w).cuda(), None, torch.tensor(pos).cuda(), freq.cuda(), g, None)
        for i in np.ndindex(3, 2, 64):
            e = np.zeros_like(x)
            e[i] = 0.5
            assert abs(loss(x + e) - loss(x - e) - g[i].item()) <= 16 * U * 2 * mag * np.abs(w[i[:2]]).max() + 1e-12


def test_one_of_the_two_and_none():
    fk = _fk()
    k = torch.randn((5, 2, 64), device="cuda")
    pos, freq, out = torch.arange(5, dtype=torch.int32, device="cuda"), fk.rope_frequencies(64).cuda(), torch.empty_like(k)
    fk.fk_rope(fk.RopeDesc(0, 2, 64, 64, "half", "f32"), None, k, pos, freq, None, out)
    ref = od.rotate(k.double().cpu().numpy(), pos.cpu().numpy(), freq.cpu().numpy(), "half", 64)
    assert np.abs(out.double().cpu().numpy() - ref).max() < 1e-5
    e = torch.empty((0, 2, 64), device="cuda")
    fk.fk_rope(fk.RopeDesc(0, 2, 64, 64, "half", "f32"), None, e, pos, freq, None, e)
    torch.cuda.synchronize()


def test_other_stream_and_graph():
    fk = _fk()
    q, k = torch.randn((40, 8, 128), device="cuda").bfloat16(), torch.randn((40, 2, 128), device="cuda").bfloat16()
    pos, freq = torch.arange(40, dtype=torch.int32, device="cuda"), fk.rope_frequencies(128).cuda()
    desc = fk.RopeDesc(8, 2, 128, 128, "half", "bf16")
    want, got = (torch.empty_like(q), torch.empty_like(k)), (torch.empty_like(q), torch.empty_like(k))
    fk.fk_rope(desc, q, k, pos, freq, *want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    fk.fk_rope(desc, q, k, pos, freq, *got, stream=side)
    side.synchronize()
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fk.fk_rope(desc, q, k, pos, freq, *got)
    for turn in range(3):
        pos.add_(1000)
        fk.fk_rope(desc, q, k, pos, freq, *want)
        got[0].zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


def test_refused():
    """Tokens that share memory, heads that do not lie side by side, frequencies in 32 bits."""
    fk = _fk()
    q, pos, freq = torch.randn((6, 4, 64), device="cuda"), torch.arange(6, dtype=torch.int32, device="cuda"), fk.rope_frequencies(64).cuda()
    desc = fk.RopeDesc(4, 0, 64, 64, "half", "f32")
    for x, f in ((q[:1].expand(6, -1, -1), freq), (q.transpose(0, 1).contiguous().transpose(0, 1), freq), (q, freq.float()), (q, freq[:31])):
        with pytest.raises(AssertionError):
            fk.fk_rope(desc, x, None, pos, f, torch.empty_like(q), None)
    with pytest.raises(fk.FkError):   # in place, but the outputs' tokens lie closer together
        wide = torch.randn((6, 8, 64), device="cuda")
        fk.fk_rope(desc, wide[:, :4], None, pos, freq, wide.view(-1)[:6 * 4 * 64].view(6, 4, 64), None)


@pytest.mark.parametrize("rot, layout", [(50, "half"), (50, "interleaved"), (64, "half"), (6, "interleaved")])
def test_channels_that_do_not_turn_keep_their_bits(rot, layout):
    """Every bf16 there is, NaN of all kinds among them, behind the rotated channels: copied as they are, whatever the width of the loads."""
    fk = _fk()
    D, n = 128, 2 ** 16 // (128 - 64) + 1
    k = torch.ones((n, 1, D), dtype=torch.bfloat16, device="cuda")
    x = k.view(torch.int16)
    x[..., rot:] = torch.arange(n * (D - rot), device="cuda").remainder(2 ** 16).sub(2 ** 15).to(torch.int16).reshape(n, 1, D - rot)
    assert x[..., rot:].unique().numel() == 2 ** 16
    out = torch.empty_like(k)
    fk.fk_rope(fk.RopeDesc(0, 1, D, rot, layout, "bf16"), None, k, torch.arange(n, dtype=torch.int32, device="cuda"), fk.rope_frequencies(rot).cuda(), None, out)
    assert torch.equal(out.view(torch.int16)[..., rot:], x[..., rot:])
