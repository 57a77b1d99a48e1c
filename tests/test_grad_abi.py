"""Refusals of the relative bias and of the attention's gradients, and the buckets of distances: every call here fails
validation (or has nothing to do), so none of them enqueues a kernel; the fake pointers are never dereferenced."""
import ctypes
import math

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


def grads(**kw):
    f = dict(do_token=1024, do_head=128, dq_token=1024, dq_head=128, dk_token=256, dk_head=128, dv_token=256, dv_head=128)
    f.update(kw)
    return la.PromptGrads(*[f[n] for n, _ in la.PromptGrads._fields_])


def rel(**kw):
    f = dict(lo=-128, hi=128, buckets=32, dtype=0)
    f.update(kw)
    return la.RelBias(*[f[n] for n, _ in la.RelBias._fields_])


def ref(x):
    return None if x is None else ctypes.byref(x)


def fwd(s, b, q=P, k=P, v=P, cu_q=P, cu_k=P, bucket=P, weight=P, scale=0.0, o=P, lse=None, ws=P, nbytes=1 << 40):
    return la.lib().la_prompt_attn_bias(ref(s), ref(b), q, k, v, cu_q, cu_k, bucket, weight, ctypes.c_float(scale), o, lse,
                                        ws, nbytes, None)


def bwd(s, g, b=None, do=P, q=P, k=P, v=P, o=P, lse=P, dlse=None, cu_q=P, cu_k=P, bucket=P, weight=P, scale=0.0, dq=P,
        dk=P, dv=P, dw=P, ws=P, nbytes=1 << 40):
    return la.lib().la_prompt_attn_bwd(ref(s), ref(g), ref(b), do, q, k, v, o, lse, dlse, cu_q, cu_k, bucket, weight,
                                       ctypes.c_float(scale), dq, dk, dv, dw, ws, nbytes, None)


BAD_BIAS = [dict(lo=1, hi=0), dict(lo=-256, hi=257), dict(lo=-(1 << 20) - 1, hi=-(1 << 20)), dict(lo=1 << 20, hi=(1 << 20) + 1),
            dict(buckets=0), dict(buckets=(1 << 20) + 1), dict(lo=-(1 << 31), hi=(1 << 31) - 1)]


@cpu_only
@pytest.mark.parametrize("bad", BAD_BIAS, ids=str)
def test_bias_refused(bad):
    assert fwd(seqs(), rel(**bad)) == la.LA_ERR_SHAPE
    assert bwd(seqs(), grads(), rel(**bad)) == la.LA_ERR_SHAPE
    assert la.lib().la_prompt_bias_ws_bytes(ref(seqs(Tk=20000)), ref(rel(**bad))) == 0
    assert la.lib().la_prompt_bwd_ws_bytes(ref(seqs()), ref(rel(**bad))) == 0


@cpu_only
def test_bias_scratch():
    # none where no unit is cut: few keys, or up to 4096 in short sequences that fill the GPU with whole units
    need = lambda **kw: la.lib().la_prompt_bias_ws_bytes(ref(seqs(**kw)), ref(rel()))   # noqa: E731
    assert need(S=1, Tq=1024, Tk=1024) == 0 < need(S=1, Tq=1025, Tk=1025)
    assert need(S=16, Tq=100, Tk=4096) == 0 < need(S=16, Tq=100, Tk=4097)
    assert need(S=8, Tq=4096, Tk=4096, Hq=16, Hkv=16) == 0 < need(S=8, Tq=4096, Tk=4096, Hq=2, Hkv=2)
    assert need(S=7, Tq=4096, Tk=4096, Hq=16, Hkv=16) > 0


@cpu_only
def test_bias_arguments_refused():
    for dtype, word in ((0, 2), (1, 1)):
        for call in (lambda **kw: fwd(seqs(), rel(dtype=dtype), **kw), lambda **kw: bwd(seqs(), grads(), rel(dtype=dtype), **kw)):
            for name in ("bucket", "weight"):
                assert call(**{name: None}) == la.LA_ERR_ARG, name
            assert call(bucket=ctypes.c_void_p(4098)) == la.LA_ERR_ARG
            assert call(weight=ctypes.c_void_p(4096 + word)) == la.LA_ERR_ARG
    assert fwd(seqs(), rel(), scale=1e-20) == la.LA_ERR_ARG and bwd(seqs(), grads(), rel(), scale=1e-20) == la.LA_ERR_ARG
    for call in (lambda b: fwd(seqs(), b), lambda b: bwd(seqs(), grads(), b)):
        assert call(rel(dtype=2)) == la.LA_ERR_ARG and call(rel(dtype=-1)) == la.LA_ERR_ARG
    assert bwd(seqs(), grads(), rel(), dw=None) == la.LA_ERR_ARG
    assert bwd(seqs(), grads(), rel(), dw=ctypes.c_void_p(4098)) == la.LA_ERR_ARG
    s = seqs(Tk=20000)
    need = la.lib().la_prompt_bias_ws_bytes(ref(s), ref(rel()))
    assert need > 0
    assert fwd(s, rel(), ws=None) == la.LA_ERR_WORKSPACE and fwd(s, rel(), nbytes=need - 1) == la.LA_ERR_WORKSPACE
    # without a bias the call is la_prompt_attn
    assert la.lib().la_prompt_bias_ws_bytes(ref(s), None) == la.lib().la_prompt_ws_bytes(ref(s)) > 0
    assert fwd(seqs(d=96), None) == la.LA_ERR_SHAPE and fwd(s, None, q=None) == la.LA_ERR_ARG


@cpu_only
@pytest.mark.parametrize("bad", [dict(S=-1), dict(Tq=-1), dict(Tk=-1), dict(Hq=0), dict(Hkv=0), dict(Hq=9), dict(Hq=65536),
                                 dict(d=96), dict(causal=2), dict(q_token=64), dict(q_head=4), dict(k_token=1 << 24),
                                 dict(v_token=127), dict(v_head=-8), dict(o_token=-1024), dict(o_head=-128),
                                 dict(S=(1 << 31) - 4095)], ids=str)
def test_bwd_shapes_refused(bad):
    assert bwd(seqs(**bad), grads()) == la.LA_ERR_SHAPE


@cpu_only
@pytest.mark.parametrize("bad", [dict(do_token=64), dict(do_head=-128), dict(do_token=1025), dict(dq_head=0), dict(dq_token=64),
                                 dict(dk_head=0), dict(dk_token=1 << 24), dict(dv_head=4), dict(dv_token=0)], ids=str)
def test_bwd_strides_refused(bad):
    assert bwd(seqs(), grads(**bad)) == la.LA_ERR_SHAPE


@cpu_only
def test_bwd_arguments_refused():
    s, g = seqs(), grads()
    assert bwd(None, g) == la.LA_ERR_ARG and bwd(s, None) == la.LA_ERR_ARG
    for name in ("do", "q", "k", "v", "o", "dq", "dk", "dv"):
        assert bwd(s, g, **{name: None}) == la.LA_ERR_ARG, name
        assert bwd(s, g, **{name: ODD}) == la.LA_ERR_ARG, name
    for name in ("lse", "cu_q", "cu_k"):
        assert bwd(s, g, **{name: None}) == la.LA_ERR_ARG, name
    for name in ("lse", "dlse", "cu_q", "cu_k"):
        assert bwd(s, g, **{name: ctypes.c_void_p(4098)}) == la.LA_ERR_ARG, name
    assert bwd(s, g, scale=float("nan")) == la.LA_ERR_ARG and bwd(s, g, scale=float("inf")) == la.LA_ERR_ARG
    for b in (None, rel()):
        need = la.lib().la_prompt_bwd_ws_bytes(ref(s), ref(b))
        assert need >= 100 * 8 * 8
        assert bwd(s, g, b, ws=None) == la.LA_ERR_WORKSPACE
        assert bwd(s, g, b, nbytes=need - 1) == la.LA_ERR_WORKSPACE
        assert bwd(s, g, b, ws=ctypes.c_void_p(4096 + 16)) == la.LA_ERR_WORKSPACE


@cpu_only
def test_bwd_with_nothing_to_do():
    none = dict(do=None, q=None, k=None, v=None, o=None, lse=None, cu_q=None, cu_k=None, dq=None, dk=None, dv=None, ws=None, nbytes=0)
    for empty in (dict(S=0), dict(Tq=0, Tk=0)):
        assert bwd(seqs(**empty), grads(), **none) == la.LA_OK
    # keys without queries have gradients of zeros to write
    assert bwd(seqs(Tq=0), grads(), **none) == la.LA_ERR_ARG
    # scratch stops growing with the work, but for the rows' statistics
    a, b = (la.lib().la_prompt_bwd_ws_bytes(ref(seqs(Tq=n, Tk=n)), None) for n in (1 << 18, 1 << 19))
    assert b - a == (1 << 18) * 8 * 8


def test_binding_refuses():
    q = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    cu = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        la.prompt_attn_bwd(q, q, q, q, q, torch.zeros(4, 2), cu)


@pytest.mark.parametrize("form", [(32, 128, True), (32, 128, False), (8, 16, True), (20, 250, True), (64, 256, True),
                                  (128, 512, False), (4, 3, True), (2, 2, False), (3, 9, False)], ids=str)
def test_relative_buckets(form):
    buckets, reach, both = form
    to, lo = la.relative_buckets(buckets, reach, both, device="cpu")
    assert lo == -reach and to.numel() == reach + 1 + (reach if both else 0) and to.dtype is torch.int32
    n = buckets // 2 if both else buckets
    one = n // 2
    past = to[: reach + 1].flip(0).tolist()
    assert past[0] == 0 and past[-1] == n - 1 and past == sorted(past)
    assert past[:one] == list(range(one))
    for m, b in enumerate(past):
        if m >= one:
            x = math.log(m / one) / math.log(reach / one) * (n - one)
            assert b == min(n - 1, one + math.floor(x)) or abs(x - round(x)) < 1e-9, (m, b, x)
            if abs(x - round(x)) < 1e-9:
                assert b == min(n - 1, one + round(x))                     # a border belongs to the bucket behind it
    if both:
        assert to[reach + 1:].tolist() == [n + b for b in past[1:]]


def test_relative_buckets_refused():
    for bad in ((1, 16, False), (2, 16, True), (32, 8, True), (32, 257, True), (32, 513, False), (0, 4, False), (-4, 4, False)):
        with pytest.raises(ValueError):
            la.relative_buckets(*bad, device="cpu")
