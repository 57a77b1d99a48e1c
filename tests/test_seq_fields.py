"""Which fields of a la_seqs the calls over a 4-bit cache look at.  Every call here ends in validation or
has nothing to do; the fake pointers are never dereferenced."""
import ctypes

import pytest
import torch

from paper_2605_31158_amd import la

cpu_only = pytest.mark.skipif(torch.cuda.is_available(), reason="fake-pointer validation tests run on CPU hosts only")
P = ctypes.c_void_p(4096)
CACHE = la.Kv4(10, 64, 4)


def rows(**kw):
    """A zeroed la_seqs with the fields that entering and reading rows uses."""
    s = la.Seqs()
    f = dict(S=2, Tk=120, Hkv=2, d=128, k_token=256, k_head=128, v_token=256, v_head=128)
    f.update(kw)
    for n, x in f.items():
        setattr(s, n, x)
    return s


def append(s, cu=P):
    return la.lib().la_kv4_append(ctypes.byref(s), ctypes.byref(CACHE), P, P, cu, P, P, P, None)


def read(s, cu=P):
    return la.lib().la_kv4_read(ctypes.byref(s), ctypes.byref(CACHE), P, cu, P, P, P, P, None)


UNUSED = [dict(), dict(Tq=-1), dict(Tq=(1 << 31) - 1), dict(causal=7), dict(causal=-1),
          dict(q_token=3, q_head=-5, o_token=1, o_head=0), dict(Hq=0), dict(Hq=6)]


@cpu_only
@pytest.mark.parametrize("unused", UNUSED, ids=str)
@pytest.mark.parametrize("call", [append, read])
def test_rows_need_only_their_fields(call, unused):
    # the first check behind the fields is that of the pointers
    assert call(rows(**unused), cu=None) == la.LA_ERR_ARG
    assert call(rows(Tk=0, **unused)) == la.LA_OK
    assert call(rows(S=0, **unused)) == la.LA_OK


@cpu_only
@pytest.mark.parametrize("call", [append, read])
def test_rows_fields_refused(call):
    for bad in (dict(S=-1), dict(Tk=-1), dict(Hkv=0), dict(Hkv=-2), dict(Hkv=65536), dict(d=96), dict(Hq=-2), dict(Hq=3),
                dict(Hq=65536), dict(k_token=64), dict(v_head=4)):
        assert call(rows(**bad)) == la.LA_ERR_SHAPE, bad


@cpu_only
def test_attention_takes_a_zeroed_rest():
    s = la.Seqs()
    for n, x in dict(S=2, Tq=100, Hq=8, Hkv=2, d=128, q_token=1024, q_head=128, o_token=1024, o_head=128).items():
        setattr(s, n, x)
    for n in ("k_token", "k_head", "v_token", "v_head"):
        setattr(s, n, -7)
    call = lambda cu: la.lib().la_kv4_attn(ctypes.byref(s), ctypes.byref(CACHE), 1, P, P, cu, P, P, ctypes.c_float(0),  # noqa: E731
                                           P, None, P, 1 << 40, None)
    assert call(None) == la.LA_ERR_ARG
    s.Hq = 0
    assert call(None) == la.LA_ERR_SHAPE
