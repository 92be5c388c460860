"""Refusals of the paged prompt cache and of the accumulated weights: bad arguments end as status codes before any launch (no GPU)."""
import ctypes
import os

import pytest


@pytest.fixture(scope="module")
def fklib():
    from paper_2602_03203_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2602_03203_amd import build
        build.build()
    return binding


p = 4096   # a pointer that is never followed


def calls(L, d, rows, **other):
    """Every call on the descriptor with good arguments but for those named in `other`."""
    a = dict(K=p, V=p, table=p, kv_len=p, q_start=p, n=8, k_new=p, v_new=p, q=p, out=p, stats=p, acc=p, chunk=4, len=64, window=0, sink=0, ws=p, bytes=0,
             keep=p, budget=64, Kr=p, Vr=p, pos=p, rlen=p, acc_rows=p)
    a.update(other)
    D, R = ctypes.byref(d), ctypes.byref(rows)
    return dict(
        append=L.fk_paged_append(D, a["K"], a["V"], a["table"], a["kv_len"], a["q_start"], a["n"], a["k_new"], a["v_new"], 0) if not other.get("skip_append") else None,
        attn=L.fk_paged_attn(D, a["q"], a["K"], a["V"], a["table"], a["kv_len"], a["q_start"], a["n"], a["chunk"], a["len"], a["window"], a["sink"], 1.0,
                             a["out"], a["stats"], a["ws"], a["bytes"], 0),
        weights=L.fk_paged_weights(D, a["q"], a["K"], a["table"], a["kv_len"], a["q_start"], a["n"], a["chunk"], a["len"], a["window"], a["sink"], 1.0,
                                   a["stats"], a["acc"], a["ws"], a["bytes"], 0))


@pytest.mark.parametrize("field, value, code", [("batch", 0, 1), ("n_q_heads", 7, 1), ("n_kv_heads", 0, 1), ("head_dim", 96, 2), ("dtype", 2, 2),
                                                ("page_size", 0, 1), ("page_size", 8, 2), ("page_size", 48, 2), ("page_size", 2048, 2),
                                                ("n_pages", 0, 1), ("max_pages", 0, 1), ("max_pages", 1 << 20, 2), ("n_q_heads", 18, 2)])
def test_descriptors(fklib, field, value, code):
    L = fklib.lib()
    d = fklib.fk_paged_desc(2, 8, 2, 128, 16, 100, 40, fklib.FK_BF16)
    setattr(d, field, value)
    rows = fklib.fk_cache_desc(2, 8, 2, 128, 512, fklib.FK_BF16)
    got = calls(L, d, rows, bytes=1 << 40)
    assert set(got.values()) == {code}, got
    assert L.fk_paged_attn_workspace(ctypes.byref(d), 8, 4, 64) == 0 and L.fk_paged_weights_workspace(ctypes.byref(d), 8, 4, 64) == 0
    assert L.fk_paged_compress(ctypes.byref(d), p, p, p, p, p, p, 64, ctypes.byref(rows), p, p, p, p, p, 0) == code


@pytest.mark.parametrize("arg, value", [("K", 0), ("table", 0), ("kv_len", 0), ("q_start", 0), ("q", 0), ("V", 0), ("out", 0), ("K", p + 4), ("q", p + 8),
                                        ("out", p + 2), ("stats", p + 4), ("chunk", 0), ("len", 0), ("len", 641), ("n", -1), ("window", -1), ("sink", -1)])
def test_arguments_of_attention_and_weights(fklib, arg, value):
    L = fklib.lib()
    d, rows = fklib.fk_paged_desc(2, 8, 2, 128, 16, 100, 40, fklib.FK_BF16), fklib.fk_cache_desc(2, 8, 2, 128, 512, fklib.FK_BF16)
    got = calls(L, d, rows, bytes=0, skip_append=True, **{arg: value})     # (without a workspace nothing can be launched)
    only = {"V": ("attn",), "out": ("attn",)}.get(arg, ("attn", "weights"))
    for name in only:
        assert got[name] == fklib.FK_ERR_INVALID_ARG, (name, got)


def test_workspaces(fklib):
    L = fklib.lib()
    d, rows = fklib.fk_paged_desc(2, 8, 2, 128, 16, 100, 40, fklib.FK_BF16), fklib.fk_cache_desc(2, 8, 2, 128, 512, fklib.FK_BF16)
    D = ctypes.byref(d)
    need = L.fk_paged_attn_workspace(D, 8, 4, 64), L.fk_paged_weights_workspace(D, 8, 4, 64)
    assert min(need) > 0
    got = calls(L, d, rows, ws=0, bytes=1 << 40, skip_append=True)
    assert got["attn"] == got["weights"] == fklib.FK_ERR_WORKSPACE
    got = calls(L, d, rows, bytes=min(need) - 1, skip_append=True)
    assert got["attn"] == fklib.FK_ERR_WORKSPACE or need[0] > min(need)
    assert got["weights"] == fklib.FK_ERR_WORKSPACE or need[1] > min(need)
    assert L.fk_paged_attn_workspace(D, 1 << 26, 4, 64) == 0               # more query rows than 32-bit counts hold
    got = calls(L, d, rows, n=1 << 26, bytes=1 << 40, skip_append=True)
    assert got["attn"] == got["weights"] == fklib.FK_ERR_UNSUPPORTED
    got = calls(L, d, rows, n=0, bytes=1 << 40)                            # no token: nothing to do
    assert set(got.values()) == {fklib.FK_OK}


def test_append_refuses(fklib):
    L = fklib.lib()
    D = ctypes.byref(fklib.fk_paged_desc(2, 8, 2, 128, 16, 100, 40, fklib.FK_BF16))
    good = [p, p, p, p, p, 8, p, p]
    for i in (0, 1, 2, 3, 4, 6, 7):
        assert L.fk_paged_append(D, *good[:i], 0, *good[i + 1:], 0) == fklib.FK_ERR_INVALID_ARG
    for i in (0, 1, 6, 7):
        assert L.fk_paged_append(D, *good[:i], p + 8, *good[i + 1:], 0) == fklib.FK_ERR_INVALID_ARG
    assert L.fk_paged_append(D, p, p, p, p, p, -1, p, p, 0) == fklib.FK_ERR_INVALID_ARG
    assert L.fk_paged_append(None, *good, 0) == fklib.FK_ERR_INVALID_ARG


def test_compress_refuses(fklib):
    L = fklib.lib()
    D = ctypes.byref(fklib.fk_paged_desc(2, 8, 2, 128, 16, 100, 40, fklib.FK_BF16))
    R = fklib.fk_cache_desc
    good, rows = [p, p, p, p, p, p, 64], R(2, 8, 2, 128, 512, fklib.FK_BF16)
    tail = [p, p, p, p, p]
    for i in range(6):
        assert L.fk_paged_compress(D, *good[:i], 0, *good[i + 1:], ctypes.byref(rows), *tail, 0) == fklib.FK_ERR_INVALID_ARG, i
    for i in range(5):
        assert L.fk_paged_compress(D, *good, ctypes.byref(rows), *tail[:i], 0, *tail[i + 1:], 0) == fklib.FK_ERR_INVALID_ARG, i
    for budget in (0, 513):
        assert L.fk_paged_compress(D, *good[:6], budget, ctypes.byref(rows), *tail, 0) == fklib.FK_ERR_INVALID_ARG
    for other in (R(1, 8, 2, 128, 512, 1), R(2, 4, 2, 128, 512, 1), R(2, 8, 4, 128, 512, 1), R(2, 8, 2, 64, 512, 1), R(2, 8, 2, 128, 512, 0)):
        assert L.fk_paged_compress(D, *good, ctypes.byref(other), *tail, 0) == fklib.FK_ERR_INVALID_ARG
    assert L.fk_paged_compress(D, *good, ctypes.byref(R(2, 8, 2, 96, 512, 1)), *tail, 0) == fklib.FK_ERR_UNSUPPORTED


def test_accumulated_weights_refuse(fklib):
    L = fklib.lib()
    R = fklib.fk_cache_desc
    d = R(2, 8, 2, 128, 512, fklib.FK_BF16)
    need = L.fk_decode_step_acc_workspace(ctypes.byref(d))
    assert need > 0 and L.fk_decode_step_acc_workspace(ctypes.byref(R(2, 7, 2, 128, 512, 1))) == 0
    args = [p] * 8 + [512, 1.0, p, p, p, need, 0]
    for i in [j for j in range(12) if j not in (8, 9)]:
        assert L.fk_decode_step_acc(ctypes.byref(d), *args[:i], 0, *args[i + 1:]) == fklib.FK_ERR_INVALID_ARG, i
    for i in (0, 1, 2, 5, 6, 10, 11):                    # q, K, V, k_new, v_new, acc, out off their alignment
        assert L.fk_decode_step_acc(ctypes.byref(d), *args[:i], p + 4, *args[i + 1:]) == fklib.FK_ERR_INVALID_ARG, i
    for n in (0, 513):
        assert L.fk_decode_step_acc(ctypes.byref(d), *args[:8], n, *args[9:]) == fklib.FK_ERR_INVALID_ARG
    assert L.fk_decode_step_acc(ctypes.byref(d), *args[:13], need - 1, 0) == fklib.FK_ERR_WORKSPACE
    assert L.fk_decode_step_acc(ctypes.byref(d), *args[:12], 0, need, 0) == fklib.FK_ERR_WORKSPACE
    good = [p, p, p, p, p, p]
    for i in range(6):
        assert L.fk_compact_acc(ctypes.byref(d), *good[:i], 0, *good[i + 1:], 256, 0) == fklib.FK_ERR_INVALID_ARG
    for budget in (0, 513):
        assert L.fk_compact_acc(ctypes.byref(d), *good, budget, 0) == fklib.FK_ERR_INVALID_ARG
    assert L.fk_compact_acc(ctypes.byref(R(2, 8, 2, 96, 512, 1)), *good, 256, 0) == fklib.FK_ERR_UNSUPPORTED


def test_no_tokens_and_no_buffers(fklib):
    """A call without tokens, whose token buffers are empty, has nothing to do."""
    L = fklib.lib()
    d, rows = fklib.fk_paged_desc(2, 8, 2, 128, 16, 100, 40, fklib.FK_BF16), fklib.fk_cache_desc(2, 8, 2, 128, 512, fklib.FK_BF16)
    got = calls(L, d, rows, n=0, bytes=1 << 40, q=0, out=0, stats=0, k_new=0, v_new=0)
    assert set(got.values()) == {fklib.FK_OK}


def test_each_workspace_a_byte_short(fklib):
    """Each call on its own: a byte less than it asks for is refused."""
    L = fklib.lib()
    for d in (fklib.fk_paged_desc(2, 8, 2, 128, 16, 100, 40, fklib.FK_BF16), fklib.fk_paged_desc(1, 8, 2, 64, 64, 300, 256, fklib.FK_F32)):
        D = ctypes.byref(d)
        rows = fklib.fk_cache_desc(2, 8, 2, 128, 512, fklib.FK_BF16)
        for n, chunk, length in ((8, 4, 64), (200, 100, 640)):
            need = dict(attn=L.fk_paged_attn_workspace(D, n, chunk, length), weights=L.fk_paged_weights_workspace(D, n, chunk, length))
            for name, size in need.items():
                assert size > 0
                got = L.fk_paged_attn(D, p, p, p, p, p, p, n, chunk, length, 0, 0, 1.0, p, p, p, size - 1, 0) if name == "attn" else \
                    L.fk_paged_weights(D, p, p, p, p, p, n, chunk, length, 0, 0, 1.0, p, p, p, size - 1, 0)
                assert got == fklib.FK_ERR_WORKSPACE, (name, size, got)
        assert calls(L, d, rows, n=8, bytes=0, skip_append=True) == dict(append=None, attn=fklib.FK_ERR_WORKSPACE, weights=fklib.FK_ERR_WORKSPACE)
