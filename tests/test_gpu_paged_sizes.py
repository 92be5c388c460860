"""Sizes of the paged calls at which their launches change: more rows than a grid's second dimension holds, wide blocks of keys under a window."""
import numpy as np
import pytest
import torch

from paged_util import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("with_acc", [True, False])
def test_compress_more_than_65535_rows(with_acc):
    import paper_2602_03203_amd as fk
    B, H, D, ps, budget, cap, pages = 35000, 2, 64, 16, 70, 72, 300
    gen = torch.Generator(device="cuda").manual_seed(3)
    K, V = (torch.randn((pages, H, ps, D), generator=gen, device="cuda").bfloat16() for _ in range(2))
    table = torch.randint(0, pages, (B, 6), generator=gen, device="cuda", dtype=torch.int32)      # (sequences share pages)
    kv_len = torch.randint(0, 97, (B,), generator=gen, device="cuda", dtype=torch.int32)
    keep = torch.rand((B, H, 96), generator=gen, device="cuda").argsort(dim=2)[:, :, :budget].sort(dim=2).values.int() % kv_len.clamp(min=1)[:, None, None]
    keep = keep.int().contiguous()
    acc = torch.rand((B, H, 96), generator=gen, device="cuda") if with_acc else None
    Kr, Vr = (torch.full((B, H, cap, D), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pos, ln = torch.full((B, H, cap), -5, dtype=torch.int32, device="cuda"), torch.full((B, H), -5, dtype=torch.int32, device="cuda")
    acc_r = torch.full((B, H, cap), 4.0, device="cuda") if with_acc else None
    fk.fk_paged_compress(fk.PagedDesc(B, 2 * H, H, D, ps, pages, 6, "bf16"), K, V, table, kv_len, acc, keep, budget, fk.CacheDesc(B, 2 * H, H, D, cap, "bf16"),
                         Kr, Vr, pos, ln, acc_r)
    torch.cuda.synchronize()
    want_len = kv_len.clamp(max=budget)[:, None].expand(B, H)
    assert torch.equal(ln, want_len)
    live = torch.arange(budget, device="cuda") < want_len[:, :, None]
    k = keep.long()
    page = table.long()[torch.arange(B, device="cuda")[:, None, None], k // ps]
    h = torch.arange(H, device="cuda")[:, None].expand(B, H, budget)
    for pool, rows in ((K, Kr), (V, Vr)):
        for at in range(0, B, 5000):     # (a part at a time: the whole comparison would be gigabytes)
            e = slice(at, at + 5000)
            want = torch.where(live[e, :, :, None], pool[page[e], h[e], k[e] % ps], torch.tensor(3.0, dtype=torch.bfloat16, device="cuda"))
            assert torch.equal(rows[e, :, :budget], want)
        assert (rows[:, :, budget:] == 3).all()
    assert torch.equal(pos[:, :, :budget], torch.where(live, keep, -5)) and (pos[:, :, budget:] == -5).all()
    if with_acc:
        assert torch.equal(acc_r[:, :, :budget], torch.where(live, acc.gather(2, k), 4.0)) and (acc_r[:, :, budget:] == 4).all()


@pytest.mark.parametrize("dtype, D, sink", [("bf16", 64, 0), ("bf16", 64, 5), ("f32", 128, 0), ("f32", 128, 5), ("bf16", 128, 300)])
def test_wide_key_blocks_under_a_window(dtype, D, sink):
    """Rows, pairs and queries enough for wavefronts of many keys and split queries; blocks of keys that no query reaches have no partial sums (what the workspace
    holds there is NaN)."""
    chunks = [(3000, 300), (2600, 1), (1500, 290)] + [(40 + 9 * b, 1 + b % 3) for b in range(29 if dtype == "bf16" else 13)]
    c = Case(dtype, D, 8, 2, 64, chunks, 700, sink, seed=61)
    s = c.dev()
    c.run(s)
    torch.cuda.synchronize()
    assert s["wws"].numel() > 2 * s["acc"].numel() * 4      # (several splits)
    ref, tol = c.reference()
    c.check(s, ref, tol)
    assert torch.equal(s["acc"][0, :, max(sink, 0) // 256 * 256 + 256:1792].cpu(), c.acc[0, :, max(sink, 0) // 256 * 256 + 256:1792])     # whole blocks behind the sinks that nobody sees
    assert np.isfinite(s["acc"].cpu().numpy()).all()
