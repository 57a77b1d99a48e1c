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
    s = seqs()
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
    assert la.lib().la_prompt_ws_bytes(ctypes.byref(seqs(S=1, Tq=1, Tk=64))) < 1 << 23


def test_binding_refuses_cpu_tensors():
    q = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    cu = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        la.prompt_attn(q, q, q, cu)
