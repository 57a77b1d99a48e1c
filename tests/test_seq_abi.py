"""Refusals of the entry points over packed sequences: every call here fails validation (or has nothing to
do), so none of them enqueues a kernel; the fake pointers are never dereferenced."""
import ctypes

import pytest
import torch

from paper_2605_31158_amd import la

cpu_only = pytest.mark.skipif(torch.cuda.is_available(), reason="fake-pointer validation tests run on CPU hosts only")
P = ctypes.c_void_p(4096)
ODD = ctypes.c_void_p(4104)


def seqs(**kw):
    f = dict(S=2, Tq=100, Tk=120, Hq=8, Hkv=2, d=128, causal=1, q_token=1024, q_head=128, o_token=1024, o_head=128,
             k_token=256, k_head=128, v_token=256, v_head=128)
    f.update(kw)
    return la.Seqs(*[f[n] for n, _ in la.Seqs._fields_])


def prompt(s, q=P, k=P, v=P, cu_q=P, cu_k=P, scale=0.0, o=P, lse=None, ws=P, nbytes=1 << 40):
    return la.lib().la_prompt_attn(None if s is None else ctypes.byref(s), q, k, v, cu_q, cu_k, ctypes.c_float(scale), o,
                                   lse, ws, nbytes, None)


@cpu_only
@pytest.mark.parametrize("bad", [dict(S=-1), dict(Tq=-1), dict(Tk=-1), dict(Hq=0), dict(Hkv=0), dict(Hq=9), dict(Hq=65536),
                                 dict(d=96), dict(d=0), dict(causal=2), dict(q_token=64), dict(q_token=1025),
                                 dict(q_head=4), dict(k_token=1 << 24), dict(v_token=127), dict(v_head=-8),
                                 dict(o_head=0), dict(o_token=-1024)], ids=str)
def test_prompt_shapes_refused(bad):
    assert prompt(seqs(**bad)) == la.LA_ERR_SHAPE


@cpu_only
def test_prompt_arguments_refused():
    s = seqs(Tk=2000)
    assert prompt(None) == la.LA_ERR_ARG
    for name in ("q", "k", "v", "o", "cu_q", "cu_k"):
        assert prompt(s, **{name: None}) == la.LA_ERR_ARG, name
    for name in ("q", "k", "v", "o"):
        assert prompt(s, **{name: ODD}) == la.LA_ERR_ARG, name
    for name in ("cu_q", "cu_k", "lse"):
        assert prompt(s, **{name: ctypes.c_void_p(4098)}) == la.LA_ERR_ARG, name
    assert prompt(s, scale=float("nan")) == la.LA_ERR_ARG
    assert prompt(s, scale=float("inf")) == la.LA_ERR_ARG
    need = la.lib().la_prompt_ws_bytes(ctypes.byref(s))
    assert need > 0
    assert prompt(s, ws=None) == la.LA_ERR_WORKSPACE
    assert prompt(s, nbytes=need - 1) == la.LA_ERR_WORKSPACE
    assert prompt(s, ws=ctypes.c_void_p(4096 + 16)) == la.LA_ERR_WORKSPACE


@cpu_only
def test_prompt_with_nothing_to_do():
    for empty in (dict(S=0), dict(Tq=0)):
        s = seqs(**empty)
        assert la.lib().la_prompt_ws_bytes(ctypes.byref(s)) == 0
        assert prompt(s, q=None, k=None, v=None, o=None, ws=None, nbytes=0) == la.LA_OK
    assert la.lib().la_prompt_ws_bytes(ctypes.byref(seqs(d=96))) == 0
    # scratch stops growing with the work: partials of 256 workgroups
    most = la.lib().la_prompt_ws_bytes(ctypes.byref(seqs(Tq=1 << 20, Tk=1 << 20)))
    assert 2 * 256 * 256 * 128 * 4 <= most < 2 * 256 * 256 * 131 * 4
    assert la.lib().la_prompt_ws_bytes(ctypes.byref(seqs(S=1, Tq=1, Tk=2000))) < 1 << 23
    assert la.lib().la_prompt_ws_bytes(ctypes.byref(seqs(S=1, Tq=1, Tk=64))) == 0      # nothing is split


def test_binding_refuses_cpu_tensors():
    q = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    cu = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        la.prompt_attn(q, q, q, cu)


def kv4(**kw):
    f = dict(n_pages=10, page=64, max_pages=4)
    f.update(kw)
    return la.Kv4(f["n_pages"], f["page"], f["max_pages"])


def append(s, c, k=P, v=P, cu=P, lens=P, table=P, cache=P):
    return la.lib().la_kv4_append(None if s is None else ctypes.byref(s), None if c is None else ctypes.byref(c), k, v, cu,
                                  lens, table, cache, None)


def read(s, c, k=P, v=P, cu=P, lens=P, table=P, cache=P):
    return la.lib().la_kv4_read(None if s is None else ctypes.byref(s), None if c is None else ctypes.byref(c), cache, cu,
                                lens, table, k, v, None)


def attn(s, c, max_q=1, q=P, cache=P, cu=P, lens=P, table=P, scale=0.0, o=P, lse=None, ws=P, nbytes=1 << 40):
    return la.lib().la_kv4_attn(None if s is None else ctypes.byref(s), None if c is None else ctypes.byref(c), max_q, q,
                                cache, cu, lens, table, ctypes.c_float(scale), o, lse, ws, nbytes, None)


BAD_KV4 = [dict(n_pages=0), dict(page=8), dict(page=48), dict(page=2048), dict(page=0), dict(max_pages=0)]


@cpu_only
@pytest.mark.parametrize("bad", BAD_KV4, ids=str)
def test_kv4_shapes_refused(bad):
    for call in (append, read, attn):
        assert call(seqs(), kv4(**bad)) == la.LA_ERR_SHAPE, call
    assert la.lib().la_kv4_ws_bytes(ctypes.byref(seqs()), ctypes.byref(kv4(**bad)), 1) == 0


@cpu_only
def test_kv4_arguments_refused():
    s, c = seqs(), kv4()
    for call in (append, read, attn):
        assert call(None, c) == la.LA_ERR_ARG
        assert call(s, None) == la.LA_ERR_ARG
        assert call(seqs(d=96), c) == la.LA_ERR_SHAPE
        assert call(seqs(Hkv=3), c) == la.LA_ERR_SHAPE
        for name in ("cu", "lens", "table", "cache"):
            assert call(s, c, **{name: None}) == la.LA_ERR_ARG, (call, name)
        assert call(s, c, cache=ODD) == la.LA_ERR_ARG
        for name in ("cu", "lens", "table"):
            assert call(s, c, **{name: ctypes.c_void_p(4098)}) == la.LA_ERR_ARG, (call, name)
    for call in (append, read):
        for name in ("k", "v"):
            assert call(s, c, **{name: None}) == la.LA_ERR_ARG
            assert call(s, c, **{name: ODD}) == la.LA_ERR_ARG
        assert call(seqs(k_token=64), c) == la.LA_ERR_SHAPE
        assert call(seqs(v_head=4), c) == la.LA_ERR_SHAPE
        assert call(seqs(Tk=0), c, k=None, v=None) == la.LA_OK
        assert call(seqs(S=0), c, k=None, v=None) == la.LA_OK
    assert read(seqs(v_head=0), c) == la.LA_ERR_SHAPE            # rows that are written lie apart
    for name in ("q", "o"):
        assert attn(s, c, **{name: None}) == la.LA_ERR_ARG
        assert attn(s, c, **{name: ODD}) == la.LA_ERR_ARG
    assert attn(seqs(q_token=64), c) == la.LA_ERR_SHAPE
    assert attn(seqs(o_head=0), c) == la.LA_ERR_SHAPE
    assert attn(s, c, max_q=-1) == la.LA_ERR_ARG
    assert attn(s, c, scale=float("nan")) == la.LA_ERR_ARG
    assert attn(s, c, lse=ctypes.c_void_p(4097)) == la.LA_ERR_ARG
    assert la.lib().la_kv4_ws_bytes(ctypes.byref(s), ctypes.byref(c), 1) == 0           # 256 tokens: nothing is split
    c = kv4(max_pages=100)
    for max_q in (1, 17, 100):
        need = la.lib().la_kv4_ws_bytes(ctypes.byref(s), ctypes.byref(c), max_q)
        assert need > 0
        assert attn(s, c, max_q, ws=None) == la.LA_ERR_WORKSPACE
        assert attn(s, c, max_q, nbytes=need - 1) == la.LA_ERR_WORKSPACE
        assert attn(s, c, max_q, ws=ctypes.c_void_p(4096 + 64)) == la.LA_ERR_WORKSPACE
    for empty in (dict(S=0), dict(Tq=0)):
        assert attn(seqs(**empty), c, q=None, o=None, ws=None, nbytes=0) == la.LA_OK
    assert attn(s, c, max_q=0, ws=None, nbytes=0) == la.LA_OK


def test_kv4_page_bytes():
    f = la.lib().la_kv4_page_bytes
    assert f(128, 16) == 16 * 136 and f(64, 1024) == 1024 * 68
    assert f(96, 64) == 0 and f(128, 24) == 0 and f(128, 8) == 0 and f(128, 2048) == 0
    with pytest.raises(ValueError):
        la.kv4_cache(1, 1, 80, 64, device="cpu")
    with pytest.raises(TypeError):
        la.kv4_read(la.kv4_cache(1, 1, 64, 64, device="cpu"), torch.zeros(2, dtype=torch.int32),
                    torch.zeros(1, dtype=torch.int32), torch.zeros((1, 1), dtype=torch.int32), 1, 64)


@cpu_only
def test_sizes_past_the_limits_refused():
    most = (1 << 31) - 4096
    for big in (dict(Tq=most + 1), dict(Tk=most + 1), dict(S=most + 1), dict(Tq=(1 << 31) - 1)):
        assert prompt(seqs(**big)) == la.LA_ERR_SHAPE, big
        assert attn(seqs(**big), kv4()) == la.LA_ERR_SHAPE, big
        assert la.lib().la_prompt_ws_bytes(ctypes.byref(seqs(**big))) == 0
    for call in (append, read):
        assert call(seqs(Tk=(1 << 28) - 31), kv4()) == la.LA_ERR_SHAPE, call
    # the widest tables are of one size: a sequence ends before 2^31 tokens
    need = [la.lib().la_kv4_ws_bytes(ctypes.byref(seqs()), ctypes.byref(kv4(page=1024, max_pages=n)), 1)
            for n in (1 << 21, (1 << 31) - 1)]
    assert 0 < need[0] == need[1]
