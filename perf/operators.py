"""The prompt's side of a generation over a budgeted cache, as measurable cases.

A prompt lies in a paged cache until it is compressed into the rows of the budget.  Every case is a plain dict; `kind`
says which operators one pass runs:

  attn      a batch of chunks of new tokens (prompt chunks, single tokens, both) joins the paged cache and attends over it:
            fk_paged_append, fk_paged_attn; with `window` only the last `window` pairs and the first `sink` are visible
  weights   the attention weight that the pairs of the paged cache received from a chunk: fk_paged_weights
  steps     sequential decoding over the budgeted rows, every step accumulating the weights that its pairs received:
            fk_decode_step_acc
  evict     an eviction event by accumulated weight: fk_select_keep, fk_compact_acc
  compress  a prompt's pairs with the largest accumulated weight move from their pages into the rows of the budget:
            fk_select_keep_ws, fk_paged_compress

Keys, values and queries are normal, one key in a hundred three times as long (sparse heavy keys); pages lie in the pool in random
order.  A ragged batch's lengths follow from the case, all values from the seed.  Selection gets its accumulated weights as an
input: a pair at the cut to within rounding may fall on either side of it.
"""
from __future__ import annotations

import math
import random

import torch

own = False

LOG2E = 1.4426950408889634


def listed():
    return [
        # one token each for two short sequences of the tiny fp32 workload: launches and latency
        dict(name="step_tiny_f32", kind="attn", dtype="f32", batch=2, hkv=2, g=4, d=64, page=16, lo=144, hi=144, chunk=1, prompts=0, window=0, sink=0),
        # one token each for sixteen sequences of the Qwen3-4B layer shape whose prompts have not been compressed
        dict(name="step_b16", kind="attn", dtype="bf16", batch=16, hkv=8, g=4, d=128, page=64, lo=1024, hi=8192, chunk=1, prompts=0, window=0, sink=0),
        # a server's batch on a small model's layer: four prompt chunks beside twenty single tokens
        dict(name="mixed_b24", kind="attn", dtype="bf16", batch=24, hkv=4, g=4, d=64, page=16, lo=300, hi=4096, chunk=256, prompts=4, window=0, sink=0),
        # the last 2048 tokens of a 16384-token prompt
        dict(name="prompt_16k", kind="attn", dtype="bf16", batch=1, hkv=8, g=4, d=128, page=64, lo=16384, hi=16384, chunk=2048, prompts=1, window=0, sink=0),
        # one token each for the ragged batch, each seeing its last 4096 pairs and four sinks
        dict(name="sink_step_b64", kind="attn", dtype="bf16", batch=64, hkv=8, g=4, d=128, page=128, lo=1024, hi=32768, chunk=1, prompts=0, window=4096, sink=4),
        # prompt chunks of the 7B-distill layer shape (GQA 7) under a window
        dict(name="sink_prompt_gqa7", kind="attn", dtype="bf16", batch=4, hkv=4, g=7, d=128, page=32, lo=9000, hi=16384, chunk=1024, prompts=4, window=4096, sink=4),
        # weights of three short chunks
        dict(name="weights_small_f32", kind="weights", dtype="f32", batch=3, hkv=2, g=4, d=64, page=16, lo=60, hi=200, chunk=33, prompts=3, window=0, sink=0),
        # weights of the last 2048 tokens of a 16384-token prompt
        dict(name="weights_16k", kind="weights", dtype="bf16", batch=1, hkv=8, g=4, d=128, page=64, lo=16384, hi=16384, chunk=2048, prompts=1, window=0, sink=0),
        # the steps between two eviction events of the tiny fp32 workload
        dict(name="acc_tiny_f32", kind="steps", dtype="f32", batch=1, hkv=2, g=4, d=64, n=128, steps=32),
        # steps of the Qwen3-4B layer shape at the steady state of the protocol
        dict(name="acc_b16", kind="steps", dtype="bf16", batch=16, hkv=8, g=4, d=128, n=2112, steps=8),
        # an eviction event of the same shape
        dict(name="evict_b16", kind="evict", dtype="bf16", batch=16, hkv=8, g=4, d=128, n=2176, budget=2048, recent=128),
        # four prompts of up to 32768 tokens, 2048 pairs of each row are kept
        dict(name="compress_32k", kind="compress", dtype="bf16", batch=4, hkv=8, g=4, d=128, page=64, lo=24000, hi=32768, budget=2048, recent=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["step", "mixed", "prompt", "sink_step", "sink_prompt", "weights", "weights", "steps", "steps", "evict", "compress"])
    c = dict(kind="attn", dtype="bf16", batch=1, hkv=rng.choice([1, 2, 4, 8]), g=rng.choice([1, 2, 4, 4, 5, 7, 8]), d=rng.choice([64, 128, 128]))
    if kind in ("steps", "evict"):
        c.update(kind=kind, batch=_log(rng, 1, 32))
        rows = c["batch"] * c["hkv"]
        if kind == "steps":
            c.update(dtype=rng.choice(["f32", "bf16", "bf16"]), steps=rng.choice([4, 8, 16]))
            row = rows * c["steps"] * 2 * c["d"] * (4 if c["dtype"] == "f32" else 2)   # bytes of a pair of every row
            c.update(n=_log(rng, 100, max(100, min(16384, (1 << 30) // row - 32))))
        else:
            n, r = _log(rng, 100, max(100, min(16384, (1 << 18) // rows))), rng.choice([16, 64, 128])
            c.update(n=n + r + rng.choice([0, _log(rng, 1, 200)]), budget=n, recent=min(r, n))
        return c
    c.update(page=rng.choice([16, 32, 64, 128, 256]))
    if kind == "compress":
        c.update(kind=kind, batch=rng.choice([1, 2, 4, 8]), budget=_log(rng, 300, 4000), recent=rng.choice([32, 128]))
        hi = _log(rng, c["budget"] + 100, max(c["budget"] + 200, min(65536, (1 << 20) // (c["batch"] * c["hkv"]))))
        c.update(hi=hi, lo=max(1, int(hi * rng.uniform(0.3, 1.0))))
        return c
    c.update(window=0, sink=0)
    if kind in ("step", "sink_step"):
        c.update(dtype=rng.choice(["f32", "bf16", "bf16"]), batch=_log(rng, 1, 64), chunk=1, prompts=0)
        hi = _log(rng, 50, max(50, min(32768, (1 << 20) // (c["batch"] * c["hkv"]))))
    elif kind == "mixed":
        c.update(batch=rng.randint(4, 32), chunk=_log(rng, 2, 256))
        c.update(prompts=rng.randint(1, c["batch"]))
        hi = _log(rng, 300, max(300, min(8192, (1 << 28) // (c["batch"] * c["hkv"] * c["g"] * c["chunk"]))))
    else:   # prompt chunks
        f32 = rng.random() < 0.25
        c.update(dtype="f32" if f32 else "bf16", batch=rng.choice([1, 1, 2, 4]), chunk=_log(rng, 17, 1024 if f32 else 2048))
        c.update(prompts=c["batch"])
        hi = _log(rng, 64, max(64, min(16384, (1 << (25 if f32 else 29)) // (c["batch"] * c["hkv"] * c["g"] * c["chunk"]))))
        if kind == "weights":
            c.update(kind="weights")
    if kind in ("sink_step", "sink_prompt") or (kind == "weights" and rng.random() < 0.3):
        c.update(window=_log(rng, 16, 8192), sink=rng.choice([0, 1, 4, 4, 64]))
    c.update(hi=max(hi, c["chunk"]))
    c.update(lo=max(1, int(c["hi"] * rng.uniform(0.1, 1.0))))
    return c


# ---- inputs -------------------------------------------------------------------------------------------------------

def _lengths(c):
    """Chunk lengths and lengths with the chunk, of every sequence; they follow from the case alone."""
    r = random.Random("%d %d %d %d" % (c["lo"], c["hi"], c["batch"], c["hkv"]))
    chunks = [r.randint((c["chunk"] + 1) // 2, c["chunk"]) if c["batch"] > 1 and b < c["prompts"] else c["chunk"] if b < c["prompts"] else 1
              for b in range(c["batch"])]
    r.shuffle(chunks)
    return chunks, [max(n, r.randint(c["lo"], c["hi"])) for n in chunks]


def _prompt_lengths(c):
    r = random.Random("%d %d %d" % (c["lo"], c["hi"], c["batch"]))
    return [r.randint(c["lo"], c["hi"]) for _ in range(c["batch"])]


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _randn(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)


def _heavy(gen, K):
    """One pair in a hundred with a key three times as long."""
    K *= 1.0 + 2.0 * (torch.rand(K.shape[:-1] + (1,), generator=gen, device="cuda") < 0.01).to(K.dtype)
    return K


def _pages(c, gen, lens):
    """A pool with spare pages, and every sequence's pages in it in random order; -1 behind a sequence's end."""
    used = [-(-n // c["page"]) for n in lens]
    pages = sum(used) + 3
    order = torch.randperm(pages, generator=gen, device="cuda", dtype=torch.int32)[:sum(used)]
    rows = [torch.nn.functional.pad(o, (0, max(used) - o.numel()), value=-1) for o in order.split(used)]
    shape = (pages, c["hkv"], c["page"], c["d"])
    return _heavy(gen, _randn(gen, shape, _dtype(c))), _randn(gen, shape, _dtype(c)), torch.stack(rows).contiguous()


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(c, seed):
    gen, kind = torch.Generator(device="cuda").manual_seed(int(seed)), c["kind"]
    B, H, g, d, dt = c["batch"], c["hkv"], c["g"], c["d"], _dtype(c)
    s = dict(kind=kind, g=g, scale=1.0 / math.sqrt(d))
    if kind in ("attn", "weights"):
        chunks, lens = _lengths(c)
        K, V, table = _pages(c, gen, lens)
        n = sum(chunks)
        s.update(K=K, V=V, table=table, chunk=max(chunks), max_len=max(lens), kv_len=_ints(lens), window=c["window"], sink=c["sink"],
                 q_start=_ints([sum(chunks[:b]) for b in range(B + 1)]), q=_randn(gen, (n, H * g, d), dt),
                 stats=torch.empty((n, H * g, 2), dtype=torch.float32, device="cuda"))
        if kind == "attn":
            s.update(k_new=_heavy(gen, _randn(gen, (n, H, d), dt)), v_new=_randn(gen, (n, H, d), dt), out=torch.empty_like(s["q"]))
        else:
            s["stats"].copy_(_attend(s)[1])
            s.update(acc0=torch.rand((B, H, table.shape[1] * c["page"]), generator=gen, device="cuda"))
            s.update(acc=s["acc0"].clone())
    elif kind == "compress":
        lens = _prompt_lengths(c)
        K, V, table = _pages(c, gen, lens)
        # weights of a prompt: a few pairs have most
        acc = torch.randn((B, H, table.shape[1] * c["page"]), generator=gen, device="cuda").exp_()
        cap = (c["budget"] + 127) // 64 * 64
        s.update(K=K, V=V, table=table, kv_len=_ints(lens), row_len=_ints(lens)[:, None].repeat(1, H).contiguous(), acc=acc, max_len=max(lens),
                 budget=c["budget"], recent=c["recent"], keep=torch.zeros((B, H, c["budget"]), dtype=torch.int32, device="cuda"),
                 Kc=torch.zeros((B, H, cap, d), dtype=dt, device="cuda"), Vc=torch.zeros((B, H, cap, d), dtype=dt, device="cuda"),
                 pos=torch.zeros((B, H, cap), dtype=torch.int32, device="cuda"), acc_c=torch.zeros((B, H, cap), device="cuda"),
                 len=torch.zeros((B, H), dtype=torch.int32, device="cuda"))
    else:
        T = c.get("steps", 0)
        cap = (c["n"] + T + 63) // 64 * 64
        s.update(K=_heavy(gen, _randn(gen, (B, H, cap, d), dt)), V=_randn(gen, (B, H, cap, d), dt), len0=_ints([[c["n"]] * H] * B), n=c["n"],
                 pos=torch.arange(cap, dtype=torch.int32, device="cuda").expand(B, H, cap).contiguous(),
                 acc0=torch.randn((B, H, cap), generator=gen, device="cuda").exp_())
        s.update(len=s["len0"].clone(), acc=s["acc0"].clone())
        if kind == "steps":
            s.update(q=_randn(gen, (T, B, H * g, d), dt), k=_randn(gen, (T, B, H, d), dt), v=_randn(gen, (T, B, H, d), dt), T=T,
                     pos_new=(c["n"] + torch.arange(T, dtype=torch.int32, device="cuda"))[:, None].repeat(1, B).contiguous())
            s.update(out=torch.empty_like(s["q"]))
        else:
            s.update(budget=c["budget"], recent=c["recent"], keep=torch.zeros((B, H, c["budget"]), dtype=torch.int32, device="cuda"))
    if own:
        s["calls"] = _calls(c, s)
    return s


def _calls(c, s):
    """The framework's calls of one pass with their workspaces, marshalled once as a serving loop does."""
    import paper_2602_03203_amd as fk

    kind, scale = c["kind"], s["scale"]
    if kind in ("steps", "evict"):
        desc = fk.CacheDesc(c["batch"], c["hkv"] * c["g"], c["hkv"], c["d"], s["K"].shape[2], c["dtype"])
        cache = (s["K"], s["V"], s["pos"])
        if kind == "steps":
            ws = s["ws"] = fk.new_acc_workspace(desc)
            return [fk.prepare(fk.fk_decode_step_acc, desc, s["q"][t], *cache, s["len"], s["k"][t], s["v"][t], s["pos_new"][t], c["n"] + t + 1, scale,
                               s["acc"], s["out"][t], ws) for t in range(s["T"])]
        return [fk.prepare(fk.fk_select_keep, desc, s["acc"], s["pos"], s["len"], c["n"], c["budget"], c["recent"], s["keep"]),
                fk.prepare(fk.fk_compact_acc, desc, *cache, s["acc"], s["len"], s["keep"], c["budget"])]
    paged = fk.PagedDesc(c["batch"], c["hkv"] * c["g"], c["hkv"], c["d"], c["page"], s["K"].shape[0], s["table"].shape[1], c["dtype"])
    if kind == "compress":
        long = fk.CacheDesc(c["batch"], c["hkv"] * c["g"], c["hkv"], c["d"], s["acc"].shape[2], c["dtype"])
        rows = fk.CacheDesc(c["batch"], c["hkv"] * c["g"], c["hkv"], c["d"], s["Kc"].shape[2], c["dtype"])
        need = fk.fk_select_keep_workspace(long, s["max_len"], c["budget"], c["recent"])
        ws = s["ws"] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        return [fk.prepare(fk.fk_select_keep_ws, long, s["acc"], None, s["row_len"], s["max_len"], c["budget"], c["recent"], s["keep"], ws),
                fk.prepare(fk.fk_paged_compress, paged, s["K"], s["V"], s["table"], s["kv_len"], s["acc"], s["keep"], c["budget"], rows, s["Kc"], s["Vc"],
                           s["pos"], s["len"], s["acc_c"])]
    view = (s["table"], s["kv_len"], s["q_start"])
    if kind == "weights":
        ws = s["ws"] = fk.new_paged_weights_workspace(paged, s["q"].shape[0], s["chunk"], s["max_len"])
        return [fk.prepare(fk.fk_paged_weights, paged, s["q"], s["K"], *view, s["chunk"], s["max_len"], s["window"], s["sink"], scale, s["stats"], s["acc"], ws)]
    ws = s["ws"] = fk.new_paged_attn_workspace(paged, s["q"].shape[0], s["chunk"], s["max_len"])
    return [fk.prepare(fk.fk_paged_append, paged, s["K"], s["V"], *view, s["k_new"], s["v_new"]),
            fk.prepare(fk.fk_paged_attn, paged, s["q"], s["K"], s["V"], *view, s["chunk"], s["max_len"], s["window"], s["sink"], scale, s["out"], s["stats"], ws)]


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(s):
    kind = s["kind"]
    if kind in ("steps", "evict"):   # every pass starts from the same lengths and weights
        s["len"].copy_(s["len0"])
    if kind in ("steps", "evict", "weights"):
        s["acc"].copy_(s["acc0"])
    if own:
        for call in s["calls"]:
            call()
    else:
        _plain(s)
    if kind == "attn":
        return dict(out=s["out"], stats=s["stats"], K=s["K"], V=s["V"])
    if kind == "weights":
        return dict(acc=s["acc"])
    if kind == "steps":
        return dict(out=s["out"], acc=s["acc"], K=s["K"], V=s["V"], pos=s["pos"], len=s["len"])
    if kind == "evict":
        return dict(keep=s["keep"], K=s["K"], V=s["V"], pos=s["pos"], acc=s["acc"], len=s["len"])
    return dict(keep=s["keep"], K=s["Kc"], V=s["Vc"], pos=s["pos"], acc=s["acc_c"], len=s["len"])


def _plain(s):
    kind = s["kind"]
    if kind == "attn":
        b, i, p = _tokens(s)
        page, slot = s["table"][b, p // s["K"].shape[2]].long(), p % s["K"].shape[2]
        s["K"][page, :, slot] = s["k_new"]
        s["V"][page, :, slot] = s["v_new"]
        out, stats = _attend(s)
        s["out"].copy_(out)
        s["stats"].copy_(stats)
    elif kind == "weights":
        _weigh(s)
    elif kind == "steps":
        for t in range(s["T"]):   # a step needs the one before
            _step(s, t)
    else:
        acc = s["acc"]
        lens = s["len"] if kind == "evict" else s["row_len"]
        keep = _select(acc, lens, s["budget"], s["recent"])
        s["keep"].copy_(keep)
        if kind == "evict":
            _move(s, keep, lens)
        else:
            _out_of_pages(s, keep, lens)


def _tokens(s):
    """Of every token: its sequence, its place in the chunk, its position."""
    n = s["q_start"].diff().long()
    b = torch.repeat_interleave(torch.arange(n.numel(), device="cuda"), n, output_size=s["q"].shape[0])
    i = torch.arange(s["q"].shape[0], device="cuda") - s["q_start"].long()[b]
    return b, i, s["kv_len"].long()[b] - n[b] + i


def _paged(s, pool):
    """The pairs of every sequence in order, fp32 [batch][heads][max_len][d]."""
    x = pool[s["table"].clamp(min=0).long()].permute(0, 2, 1, 3, 4).flatten(2, 3)
    return x[:, :, :s["max_len"]].float()


def _logits(s):
    """Base-2 logits [batch][heads][chunk][g][max_len], -inf where a query does not see a pair, and where the tokens lie in them."""
    b, i, p = _tokens(s)
    H, g, d, n = s["K"].shape[1], s["g"], s["q"].shape[2], s["max_len"]
    B, C = s["kv_len"].numel(), s["chunk"]
    q = torch.zeros((B, C, H, g, d), device="cuda")
    q[b, i] = s["q"].float().reshape(-1, H, g, d)
    z = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(B, H, C * g, d), _paged(s, s["K"]).transpose(2, 3).contiguous())
    z = z.mul_(s["scale"] * LOG2E).reshape(B, H, C, g, n)
    at = torch.full((B, C), -1, dtype=torch.long, device="cuda")
    at[b, i] = p
    j = torch.arange(n, device="cuda")
    sees = j <= at[:, :, None]
    if s["window"]:
        sees &= (j > at[:, :, None] - s["window"]) | (j < s["sink"])
    return z.masked_fill_(~sees[:, None, :, None, :], float("-inf")), b, i


def _attend(s):
    z, b, i = _logits(s)
    B, H, C, g, n = z.shape
    top = z.amax(-1, keepdim=True)
    e = torch.exp2(z.sub_(top.nan_to_num(neginf=0.0)))
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e.reshape(B, H, C * g, n), _paged(s, s["V"])).reshape(B, H, C, g, -1) / total
    stats = torch.cat([top, total], -1)
    pick = lambda x: x.permute(0, 2, 1, 3, 4)[b, i].flatten(1, 2)   # noqa: E731
    return pick(o).to(s["q"].dtype), pick(stats)


def _weigh(s):
    z, b, i = _logits(s)
    B, H, C, g, n = z.shape
    st = torch.zeros((B, C, H, g, 2), device="cuda")
    st[..., 1] = 1.0
    st[b, i] = s["stats"].reshape(-1, H, g, 2)
    st = st.permute(0, 2, 1, 3, 4)
    w = torch.exp2(z.sub_(st[..., :1])).div_(st[..., 1:]).sum((2, 3))
    j = torch.arange(n, device="cuda")
    old = j < (s["kv_len"] - s["q_start"].diff())[:, None, None]
    live = j < s["kv_len"][:, None, None]
    a = s["acc"][:, :, :n]
    a.copy_(torch.where(live, torch.where(old, a, 0.0) + w, a))


def _step(s, t):
    B, H, g, n = s["K"].shape[0], s["K"].shape[1], s["g"], s["n"] + t + 1
    s["K"][:, :, n - 1], s["V"][:, :, n - 1] = s["k"][t], s["v"][t]
    s["pos"][:, :, n - 1] = s["pos_new"][t][:, None]
    s["len"] += 1
    K, V = s["K"][:, :, :n].float(), s["V"][:, :, :n].float()
    z = torch.matmul(s["q"][t].reshape(B, H, g, -1).float(), K.transpose(2, 3).contiguous()) * s["scale"]
    e = torch.exp(z - z.amax(-1, keepdim=True))
    w = e / e.sum(-1, keepdim=True)
    s["out"][t] = torch.matmul(w, V).reshape(B, H * g, -1).to(s["out"].dtype)
    s["acc"][:, :, n - 1] = 0
    s["acc"][:, :, :n] += w.sum(2)


def _select(scores, lens, budget, recent):
    """The slots kept of every row, ascending: the newest, then the largest scores, equal ones by the lower slot."""
    j = torch.arange(scores.shape[2], device="cuda")
    n = lens[:, :, None]
    x = torch.where(j < n, torch.where(j >= n - recent, float("inf"), scores), float("-inf"))
    best = x.sort(dim=2, descending=True, stable=True).indices[:, :, :budget].sort(dim=2).values
    return torch.where(n > budget, best, j[:budget]).int()


def _move(s, keep, lens):
    k = keep.long()
    full = (lens > s["budget"])[:, :, None]
    m = s["budget"]
    rows = k[..., None].expand(-1, -1, -1, s["K"].shape[3])
    s["K"][:, :, :m] = torch.where(full[..., None], s["K"].gather(2, rows), s["K"][:, :, :m])
    s["V"][:, :, :m] = torch.where(full[..., None], s["V"].gather(2, rows), s["V"][:, :, :m])
    s["pos"][:, :, :m] = torch.where(full, s["pos"].gather(2, k), s["pos"][:, :, :m])
    s["acc"][:, :, :m] = torch.where(full, s["acc"].gather(2, k), s["acc"][:, :, :m])
    lens.clamp_(max=m)


def _out_of_pages(s, keep, lens):
    B, H, m = keep.shape
    n, k = lens.clamp(max=m), keep.long()
    live = torch.arange(m, device="cuda") < n[:, :, None]
    src = k.minimum(lens[:, :, None].long() - 1)
    page = s["table"].clamp(min=0).long()[torch.arange(B, device="cuda")[:, None, None], src // s["K"].shape[2]]
    at = (page, torch.arange(H, device="cuda")[:, None], src % s["K"].shape[2])
    s["Kc"][:, :, :m] = torch.where(live[..., None], s["K"][at], s["Kc"][:, :, :m])
    s["Vc"][:, :, :m] = torch.where(live[..., None], s["V"][at], s["Vc"][:, :, :m])
    s["pos"][:, :, :m] = torch.where(live, keep, s["pos"][:, :, :m])
    s["acc_c"][:, :, :m] = torch.where(live, s["acc"].gather(2, src), s["acc_c"][:, :, :m])
    s["len"].copy_(n)


# ---- the least a pass has to do -------------------------------------------------------------------------------------

def work(c):
    e = 4 if c["dtype"] == "f32" else 2
    B, H, g, d = c["batch"], c["hkv"], c["g"], c["d"]
    pair = 2 * d * e
    if c["kind"] == "steps":
        lens = [c["n"] + t + 1 for t in range(c["steps"])]
        return dict(bytes=sum(B * H * (n * (pair + 8) + 2 * pair + 2 * g * d * e) for n in lens), flops=sum(4.0 * B * H * g * d * n for n in lens))
    if c["kind"] == "evict":
        return dict(bytes=B * H * (c["n"] * 4 + c["budget"] * (2 * (pair + 8) + 4)), flops=B * H * c["n"])
    if c["kind"] == "compress":
        lens = _prompt_lengths(c)
        kept = sum(min(n, c["budget"]) for n in lens)
        return dict(bytes=H * (sum(lens) * 4 + kept * (2 * (pair + 4) + 4 + 4)), flops=H * sum(lens))
    chunks, lens = _lengths(c)
    W, S = c["window"] or max(lens), c["sink"]
    seen, read = 0, 0   # (query, pair) with one seeing the other; pairs that any query sees
    for m, n in zip(chunks, lens):
        seen += sum(min(p + 1, W) + min(S, max(0, p + 1 - W)) for p in range(n - m, n))
        first = max(0, n - m - W + 1)
        read += n - first + min(S, first)
    tokens = sum(chunks)
    q = tokens * H * g * d * e
    if c["kind"] == "weights":
        return dict(bytes=read * H * (pair / 2 + 8) + q + tokens * H * g * 8, flops=seen * H * g * (2.0 * d + 3))
    return dict(bytes=read * H * pair + 2 * tokens * H * pair + 2 * q + tokens * H * g * 8, flops=seen * H * g * 4.0 * d)


# ---- the same in 64 bits ------------------------------------------------------------------------------------------

def exact(c, seed):
    kind = c["kind"]
    if kind in ("evict", "compress"):
        return None   # copies and whole numbers
    s = prepare(c, seed)
    H, g, d, scale = c["hkv"], c["g"], c["d"], s["scale"]
    if kind == "steps":
        n, T = c["n"], c["steps"]
        out, acc = s["out"].double(), s["acc0"].double()
        acc[:, :, n:n + T] = 0
        for b in range(c["batch"]):
            for h in range(H):
                K = torch.cat([s["K"][b, h, :n], s["k"][:, b, h]]).double()
                V = torch.cat([s["V"][b, h, :n], s["v"][:, b, h]]).double()
                z = (s["q"][:, b, h * g:(h + 1) * g].double().reshape(T * g, d) @ K.T).reshape(T, g, n + T) * scale
                late = torch.arange(n + T, device="cuda") > n + torch.arange(T, device="cuda")[:, None]
                w = torch.softmax(z.masked_fill_(late[:, None], float("-inf")), -1)
                out[:, b, h * g:(h + 1) * g] = (w.reshape(T * g, -1) @ V).reshape(T, g, d)
                acc[b, h, :n + T] += w.sum((0, 1))
        return dict(out=out, acc=acc, K=None, V=None, pos=None, len=None)
    chunks, lens = _lengths(c)
    page, first = c["page"], 0
    out, stats = s["q"].double(), s["stats"].double()
    acc = s["acc0"].double() if kind == "weights" else None
    for b, (m, n) in enumerate(zip(chunks, lens)):
        own_pages = s["table"][b, :-(-n // page)].long()
        j, p = torch.arange(n, device="cuda"), n - m + torch.arange(m, device="cuda")[:, None]
        hidden = j > p
        if c["window"]:
            hidden |= (j <= p - c["window"]) & (j >= c["sink"])
        for h in range(H):
            K = s["K"][own_pages, h].reshape(-1, d)[:n].double()
            heads, tokens = slice(h * g, (h + 1) * g), slice(first, first + m)
            if kind == "attn":
                K[n - m:] = s["k_new"][tokens, h].double()
            z = (s["q"][tokens, heads].double().reshape(m * g, d) @ K.T).reshape(m, g, n) * (scale / math.log(2.0))
            z.masked_fill_(hidden[:, None], float("-inf"))
            if kind == "weights":
                st = s["stats"][tokens, heads].double()
                acc[b, h, n - m:n] = 0
                acc[b, h, :n] += (torch.exp2(z - st[..., :1]) / st[..., 1:]).sum((0, 1))
                continue
            V = s["V"][own_pages, h].reshape(-1, d)[:n].double()
            V[n - m:] = s["v_new"][tokens, h].double()
            top = z.amax(-1, keepdim=True)
            e = torch.exp2(z - top)
            stats[tokens, heads] = torch.cat([top, e.sum(-1, keepdim=True)], -1)
            out[tokens, heads] = (e.reshape(m * g, n) @ V).reshape(m, g, d) / e.sum(-1, keepdim=True)
        first += m
    return dict(acc=acc) if kind == "weights" else dict(out=out, stats=stats, K=None, V=None)
