"""Refusals of the calls on drafted tokens: bad arguments end as status codes before any launch (no GPU); frequencies of rotary positions."""
import ctypes
import os

import numpy as np
import pytest


@pytest.fixture(scope="module")
def fklib():
    from paper_2602_03203_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2602_03203_amd import build
        build.build()
    return binding


p = 4096   # a pointer that is never followed
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3


def rope(L, F, **other):
    d = dict(n_q_heads=8, n_kv_heads=2, head_dim=128, rotary_dim=64, layout=0, dtype=F.FK_BF16, inverse=0, magnitude=1.0, q_stride=0, k_stride=0, q_out_stride=0, k_out_stride=0)
    a = dict(q=p, k=p, pos=p, freq=p, n=0, qo=p, ko=p)
    for k, v in other.items():
        (d if k in d else a)[k] = v
    return L.fk_rope(ctypes.byref(F.fk_rope_desc(*d.values())), a["q"], a["k"], a["pos"], a["freq"], a["n"], a["qo"], a["ko"], 0)


@pytest.mark.parametrize("change, code", [
    (dict(n_q_heads=-1), INVALID), (dict(n_kv_heads=-1), INVALID), (dict(n_q_heads=0, n_kv_heads=0), INVALID), (dict(head_dim=0), INVALID), (dict(head_dim=96), UNSUPPORTED),
    (dict(rotary_dim=0), INVALID), (dict(rotary_dim=63), INVALID), (dict(rotary_dim=130), INVALID), (dict(rotary_dim=-2), INVALID), (dict(layout=2), UNSUPPORTED),
    (dict(dtype=2), UNSUPPORTED), (dict(magnitude=float("nan")), INVALID), (dict(magnitude=float("inf")), INVALID), (dict(n_q_heads=1 << 16), UNSUPPORTED),
    (dict(q_stride=1016), INVALID), (dict(k_stride=-256), INVALID), (dict(q_out_stride=1023), INVALID), (dict(k_out_stride=260), INVALID), (dict(n=-1), INVALID),
    (dict(n=4, q=0), INVALID), (dict(n=4, k=0), INVALID), (dict(n=4, qo=0), INVALID), (dict(n=4, ko=0), INVALID), (dict(n=4, pos=0), INVALID), (dict(n=4, freq=0), INVALID),
    (dict(q=p + 8), INVALID), (dict(ko=p + 2), INVALID), (dict(freq=p + 4), INVALID), (dict(n=4, q_stride=2048), INVALID)])   # (the last: in place, with different strides)
def test_rope(fklib, change, code):
    assert rope(fklib.lib(), fklib, **change) == code
    assert rope(fklib.lib(), fklib) == 0 and rope(fklib.lib(), fklib, n_q_heads=0, q=0, qo=0) == 0   # (no tokens: nothing is launched)
    assert fklib.lib().fk_rope(None, p, p, p, p, 0, p, p, 0) == INVALID


def test_strides_in_place_are_each_tensors_own(fklib):
    """Strides of heads that a call has none of do not matter; of those it has, each in place keeps its own."""
    L, F = fklib.lib(), fklib
    assert rope(L, F, n_q_heads=0, q=0, qo=0, q_stride=128) == 0 and rope(L, F, n_q_heads=0, q_out_stride=128) == 0     # keys in place, no queries
    assert rope(L, F, n_kv_heads=0, k=0, ko=0, k_stride=128) == 0 and rope(L, F, n_kv_heads=0, k_out_stride=128) == 0   # the other way round
    assert rope(L, F, q_stride=2048, qo=2 * p) == 0 and rope(L, F, k_stride=2048, ko=2 * p) == 0                        # keys in place, queries elsewhere
    assert rope(L, F, q_stride=2048) == INVALID and rope(L, F, k_out_stride=2048) == INVALID
    assert rope(L, F, q_stride=2048, q_out_stride=2048, k_stride=512, k_out_stride=512) == 0


def test_frequencies(fklib):
    import paper_2602_03203_amd as fk
    r, base = 128, 1e6
    f = base ** (-np.arange(0, r, 2) / r)
    close = lambda a, b: np.allclose(a.numpy(), b, rtol=1e-13, atol=0)   # noqa: E731
    assert close(fk.rope_frequencies(r, base), f)
    assert close(fk.rope_frequencies(r, base, "linear", 8.0), f / 8)
    b = fk.rope_frequencies(r, base, "base", 4.0)
    assert b[0] == 1 and np.isclose(b[-1].item(), f[-1] / 4, rtol=1e-12)
    turns = 32768 * f / (2 * np.pi)
    keep = np.clip((turns - 1) / 31, 0, 1)
    got = fk.rope_frequencies(r, base, "parts", 4.0, context=32768, low=1, high=32)
    assert close(got, f * (keep + (1 - keep) / 4)) and (got.numpy() == f)[:5].all() and close(got[-5:], f[-5:] / 4)
    assert fk.rope_frequencies(2, base, "base", 4.0).tolist() == [1.0]
    for bad in (dict(rotary_dim=0), dict(rotary_dim=5), dict(rotary_dim=8, base=0.0), dict(rotary_dim=8, base=float("nan")), dict(rotary_dim=8, scaling="linear", factor=0.0),
                dict(rotary_dim=8, scaling="parts", factor=4.0), dict(rotary_dim=8, scaling="parts", factor=4.0, context=100, low=4, high=4),
                dict(rotary_dim=8, scaling="parts", factor=4.0, context=100, low=-1, high=4)):
        with pytest.raises(fk.FkError):
            fk.rope_frequencies(**bad)
    L = fklib.lib()
    buf = (ctypes.c_double * 4)()
    assert L.fk_rope_frequencies(8, 1e4, 4, 1.0, 0.0, 0.0, 0.0, buf) == UNSUPPORTED and L.fk_rope_frequencies(8, 1e4, 0, 1.0, 0.0, 0.0, 0.0, None) == INVALID


def trees(F, **other):
    """Both attention calls with good arguments but for those named in `other`, and without a workspace unless it is named."""
    L = F.lib()
    a = dict(q=p, K=p, V=p, len=p, table=p, kt=p, vt=p, parent=p, q_start=p, n=8, max_tree=4, max_len=64, window=0, sink=0, out=p, stats=p, ws=p, bytes=0)
    rows, pages = F.fk_cache_desc(2, 8, 2, 128, 512, F.FK_BF16), F.fk_paged_desc(2, 8, 2, 128, 16, 100, 40, F.FK_BF16)
    for k, v in other.items():
        if k in a:
            a[k] = v
        for d in (rows, pages):
            if hasattr(d, k):
                setattr(d, k, v)
    R, P = ctypes.byref(rows), ctypes.byref(pages)
    mid, end = (a["kt"], a["vt"], a["parent"], a["q_start"], a["n"], a["max_tree"], a["max_len"]), (a["out"], a["stats"], a["ws"], a["bytes"], 0)
    return dict(rows=L.fk_tree_attn(R, a["q"], a["K"], a["V"], a["len"], *mid, 1.0, *end),
                pages=L.fk_paged_tree_attn(P, a["q"], a["K"], a["V"], a["table"], a["len"], *mid, a["window"], a["sink"], 1.0, *end),
                rows_ws=L.fk_tree_attn_workspace(R, a["n"], a["max_tree"], a["max_len"]), pages_ws=L.fk_paged_tree_attn_workspace(P, a["n"], a["max_tree"], a["max_len"]))


@pytest.mark.parametrize("change, code", [
    (dict(batch=0), INVALID), (dict(n_q_heads=7), INVALID), (dict(n_kv_heads=0), INVALID), (dict(head_dim=96), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED),
    (dict(n_q_heads=18), UNSUPPORTED), (dict(n=-1), INVALID), (dict(max_tree=0), INVALID), (dict(max_tree=257), UNSUPPORTED), (dict(max_len=0), INVALID),
    (dict(max_len=641), INVALID), (dict(n=1 << 25), UNSUPPORTED), (dict(n_q_heads=1 << 16, n_kv_heads=1 << 16), UNSUPPORTED)])
def test_sizes_of_trees(fklib, change, code):
    got = trees(fklib, bytes=1 << 50, **change)
    assert got == dict(rows=code, pages=code, rows_ws=0, pages_ws=0)


@pytest.mark.parametrize("change", [dict(q=0), dict(K=0), dict(V=0), dict(len=0), dict(kt=0), dict(vt=0), dict(parent=0), dict(q_start=0), dict(out=0), dict(q=p + 8), dict(K=p + 4),
                                    dict(V=p + 2), dict(kt=p + 8), dict(vt=p + 8), dict(out=p + 8), dict(stats=p + 4)])
def test_arguments_of_trees(fklib, change):
    got = trees(fklib, **change)
    assert got["rows"] == got["pages"] == INVALID


@pytest.mark.parametrize("change", [dict(table=0), dict(window=-1), dict(sink=-1), dict(page_size=8), dict(page_size=48), dict(max_pages=0), dict(n_pages=0)])
def test_arguments_of_pages(fklib, change):
    assert trees(fklib, **change)["pages"] in (INVALID, UNSUPPORTED)


def test_workspaces_of_trees(fklib):
    good = trees(fklib)
    assert good["rows"] == good["pages"] == WORKSPACE and good["rows_ws"] > 0 and good["pages_ws"] > 0
    for name in ("rows", "pages"):
        for change in (dict(ws=0, bytes=1 << 40), dict(bytes=good[name + "_ws"] - 1), dict(ws=p + 8, bytes=1 << 40)):
            assert trees(fklib, **change)[name] == WORKSPACE
    none = trees(fklib, n=0, q=0, kt=0, vt=0, parent=0, out=0, bytes=1 << 30)
    assert none["rows"] == none["pages"] == 0   # no tokens: nothing to do


@pytest.mark.parametrize("batch, g, hkv, D, dtype", [(16, 4, 8, 128, "bf16"), (16, 7, 4, 64, "bf16"), (1, 8, 1, 128, "bf16"), (64, 1, 1, 128, "bf16"), (5, 3, 2, 64, "f32"), (90, 4, 1, 128, "f32"),
                                                     (3, 5, 40, 128, "bf16"), (200, 2, 8, 64, "bf16")])
def test_a_workspace_serves_smaller_calls(fklib, batch, g, hkv, D, dtype):
    """Fewer tiles are split more often and go to other kernels: what serves a call serves every one with fewer tokens, smaller trees, shorter rows."""
    import random
    rng = random.Random(batch)
    rows, pages = fklib.CacheDesc(batch, g * hkv, hkv, D, 40000, dtype), fklib.PagedDesc(batch, g * hkv, hkv, D, 64, 1000, 625, dtype)
    log = lambda lo, hi: int(round(lo * (hi / lo) ** rng.random()))   # noqa: E731
    for size, desc in ((fklib.fk_tree_attn_workspace, rows), (fklib.fk_paged_tree_attn_workspace, pages)):
        needs = {}
        for _ in range(12):
            tree = log(1, 256)
            n, length = log(tree, tree * batch), log(1, 40000)
            whole = size(desc, n, tree, length)
            for _ in range(120):
                t, m, k = log(1, tree), log(1, n), log(1, length)
                needs[m, t, k] = size(desc, m, t, k)
                assert needs[m, t, k] <= whole, f"{(m, t, k)} needs {needs[m, t, k]}, {(n, tree, length)} has {whole}"
        assert len(set(needs.values())) > 3 or batch * hkv > 1024   # (sizes do differ, but where so many tiles are never split)
    if (batch, g, hkv, D, dtype) == (16, 4, 8, 128, "bf16"):
        assert fklib.fk_tree_attn_workspace(rows, 4096, 256, 4096) >= fklib.fk_tree_attn_workspace(rows, 1024, 64, 4096) > 1 << 20


def verify(F, **other):
    a = dict(batch=2, vocab=1000, target=p, draft=p, tokens=p, parent=p, q_start=p, n=8, uniform=p, path=p, accepted=p, next=p, ws=p, bytes=0)
    a.update(other)
    return F.lib().fk_verify_drafts(a["batch"], a["vocab"], a["target"], a["draft"], a["tokens"], a["parent"], a["q_start"], a["n"], a["uniform"], a["path"], a["accepted"],
                                    a["next"], a["ws"], a["bytes"], 0)


@pytest.mark.parametrize("change, code", [(dict(batch=0), INVALID), (dict(vocab=0), INVALID), (dict(n=-1), INVALID), (dict(vocab=1 << 30), UNSUPPORTED), (dict(batch=65536), UNSUPPORTED),
                                          (dict(target=0), INVALID), (dict(tokens=0), INVALID), (dict(parent=0), INVALID), (dict(q_start=0), INVALID), (dict(uniform=0), INVALID),
                                          (dict(path=0), INVALID), (dict(accepted=0), INVALID), (dict(next=0), INVALID), (dict(), WORKSPACE), (dict(ws=0, bytes=1 << 40), WORKSPACE),
                                          (dict(ws=p + 4, bytes=1 << 40), WORKSPACE)])
def test_verify(fklib, change, code):
    assert verify(fklib, **change) == code
    need = fklib.lib().fk_verify_drafts_workspace(2, 1000)
    assert need > 0 and verify(fklib, bytes=need - 1) == WORKSPACE
    assert fklib.lib().fk_verify_drafts_workspace(0, 1000) == 0 and fklib.lib().fk_verify_drafts_workspace(2, 0) == 0


def test_a_workspace_of_verification_serves_smaller_calls(fklib):
    """Fewer sequences are cut into more chunks."""
    size = fklib.fk_verify_drafts_workspace
    for batch in (1, 2, 7, 16, 64, 255, 256, 257, 512, 513, 65535):
        for vocab in (1, 2048, 4095, 4096, 32000, 131072, (1 << 30) - 1):
            whole = size(batch, vocab)
            assert all(size(b, v) <= whole for b in (1, 3, 8, 100, 256, 500, batch) for v in (5, 4096, 50257, 131072, vocab) if b <= batch and v <= vocab), (batch, vocab)
    assert size(512, 131072) >= 256 + 512 * 16   # (eight sequences of 64 chunks at least have a place for a sum each)


@pytest.mark.parametrize("change, code", [(dict(K=0), INVALID), (dict(V=0), INVALID), (dict(pos=0), INVALID), (dict(len=0), INVALID), (dict(kt=0), INVALID), (dict(vt=0), INVALID),
                                          (dict(q_start=0), INVALID), (dict(n=-1), INVALID), (dict(path=0), INVALID), (dict(accepted=0), INVALID), (dict(first=0), INVALID),
                                          (dict(table=0), INVALID), (dict(K=p + 8), INVALID), (dict(vt=p + 8), INVALID), (dict(head_dim=96), UNSUPPORTED), (dict(dtype=5), UNSUPPORTED),
                                          (dict(batch=0), INVALID), (dict(n_kv_heads=3), INVALID), (dict(page_size=24), UNSUPPORTED), (dict(capacity=0), INVALID)])
def test_commit(fklib, change, code):
    L = fklib.lib()

    def calls(n, **other):
        a = dict(K=p, V=p, pos=p, len=p, acc=p, table=p, kt=p, vt=p, q_start=p, n=n, path=p, accepted=p, first=p)
        rows, pages = fklib.fk_cache_desc(2, 8, 2, 128, 512, fklib.FK_BF16), fklib.fk_paged_desc(2, 8, 2, 128, 16, 100, 40, fklib.FK_BF16)
        for k, v in other.items():
            if k in a:
                a[k] = v
            for d in (rows, pages):
                if hasattr(d, k):
                    setattr(d, k, v)
        return (L.fk_commit_drafts(ctypes.byref(rows), a["K"], a["V"], a["pos"], a["len"], a["acc"], a["kt"], a["vt"], a["q_start"], a["n"], a["path"], a["accepted"], a["first"], 0),
                L.fk_paged_commit_drafts(ctypes.byref(pages), a["K"], a["V"], a["table"], a["len"], a["kt"], a["vt"], a["q_start"], a["n"], a["path"], a["accepted"], 0))
    only_rows, only_pages = {"pos", "first", "capacity"} & set(change), {"table", "page_size"} & set(change)
    tokens = 4 if {"kt", "vt", "path"} & set(change) and 0 in change.values() else 0   # (without tokens these may be null, and nothing is launched)
    got = calls(**{"n": tokens, **change}) if "n" not in change else calls(change["n"])
    if not only_pages:
        assert got[0] == code
    if not only_rows:
        assert got[1] == code
    assert calls(0) == (0, 0)


def _wrapped(F, name, change):
    """Runs the wrapper of a call, which must not get as far as the library, on buffers of the right types and sizes but for those in `change`."""
    import torch

    class Device(torch.Tensor):   # (host memory that nothing follows)
        is_cuda = True
    B, H, g, D, n, vocab, cap, page = 2, 2, 4, 64, 5, 11, 32, 16
    bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    z = lambda *s, dtype=i32: torch.zeros(s, dtype=dtype).as_subclass(Device)   # noqa: E731
    rows, pages = F.CacheDesc(B, H * g, H, D, cap, "bf16"), F.PagedDesc(B, H * g, H, D, page, 3, 2, "bf16")
    in_rows = dict(K=z(B, H, cap, D, dtype=bf), V=z(B, H, cap, D, dtype=bf))
    in_pages = dict(K=z(3, H, page, D, dtype=bf), V=z(3, H, page, D, dtype=bf), page_table=z(B, 2), kv_len=z(B))
    tree = dict(k_tree=z(n, H, D, dtype=bf), v_tree=z(n, H, D, dtype=bf))
    nodes, paths = dict(parent=z(n), q_start=z(B + 1)), dict(q_start=z(B + 1), path=z(n), n_accepted=z(B))
    attend = dict(q=z(n, H * g, D, dtype=bf), out=z(n, H * g, D, dtype=bf), stats=z(n, H * g, 2, dtype=f32), workspace=None, max_tree=3, max_len=16, softmax_scale=1.0)
    calls = dict(
        fk_rope=dict(desc=F.RopeDesc(H * g, H, D, D, "half", "bf16"), q=attend["q"], k=tree["k_tree"], pos=z(n), freq=z(D // 2, dtype=torch.float64), q_out=attend["out"],
                     k_out=tree["v_tree"]),
        fk_tree_attn=dict(desc=rows, length=z(B, H), **in_rows, **tree, **nodes, **attend),
        fk_paged_tree_attn=dict(desc=pages, window=0, n_sink=0, **in_pages, **tree, **nodes, **attend),
        fk_verify_drafts=dict(target=z(n, vocab, dtype=f32), draft=z(n, vocab, dtype=f32), tokens=z(n), uniform=z(n, dtype=f32), path=z(n), n_accepted=z(B), next_token=z(B),
                              workspace=None, **nodes),
        fk_commit_drafts=dict(desc=rows, pos=z(B, H, cap), length=z(B, H), acc=z(B, H, cap, dtype=f32), pos_first=z(B), **in_rows, **tree, **paths),
        fk_paged_commit_drafts=dict(desc=pages, **in_pages, **tree, **paths))
    a = calls[name]
    for k, make in change.items():
        assert k in a
        a[k] = make(a[k])
    getattr(F, name)(**a, stream=type("Stream", (), dict(cuda_stream=0)))


SHORT = dict(fk_rope=["k", "pos", "q_out", "k_out"], fk_tree_attn=["K", "V", "length", "k_tree", "v_tree", "parent", "q_start", "out", "stats"],
             fk_paged_tree_attn=["K", "V", "page_table", "kv_len", "k_tree", "v_tree", "parent", "q_start", "out", "stats"],
             fk_verify_drafts=["draft", "tokens", "parent", "uniform", "path", "n_accepted", "next_token"],
             fk_commit_drafts=["K", "V", "pos", "length", "acc", "v_tree", "q_start", "path", "n_accepted", "pos_first"],
             fk_paged_commit_drafts=["K", "V", "page_table", "kv_len", "v_tree", "q_start", "path", "n_accepted"])
ONLY_TYPE = dict(fk_rope=["q"], fk_tree_attn=["q"], fk_paged_tree_attn=["q"], fk_verify_drafts=["target", "q_start"], fk_commit_drafts=["k_tree"], fk_paged_commit_drafts=["k_tree"])


@pytest.mark.parametrize("name", sorted(SHORT))
def test_buffers_of_another_type_or_too_few_are_refused(fklib, name, monkeypatch):
    """What torch gives by itself - tokens and positions in 64 bits, probabilities in bf16 - and rows too few are named, not misread."""
    import torch
    import paper_2602_03203_amd as F
    reached = []
    monkeypatch.setattr(fklib, "_call", lambda call, *args: reached.append(call))
    _wrapped(F, name, {})
    assert reached == [name]
    other = {torch.int32: torch.int64, torch.float32: torch.bfloat16, torch.bfloat16: torch.float16}
    for what in SHORT[name] + ONLY_TYPE[name]:
        with pytest.raises(AssertionError, match="not torch"):
            _wrapped(F, name, {what: lambda x: x.to(other[x.dtype])})
    for what in SHORT[name]:
        with pytest.raises(AssertionError, match="not"):
            _wrapped(F, name, {what: lambda x: x[:-1].contiguous()})
    assert reached == [name]
