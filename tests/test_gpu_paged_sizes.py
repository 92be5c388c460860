"""Sizes of the paged calls at which their launches change: more rows than a grid's second dimension holds."""
import pytest
import torch

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
