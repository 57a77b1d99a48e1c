"""Rows of rotary positions that are written lie apart: a stride of 0 is refused for an output on every axis
that has more than one entry, and taken for an input (a broadcast)."""
import ctypes

import pytest
import torch

from paper_2605_31158_amd import la

cpu_only = pytest.mark.skipif(torch.cuda.is_available(), reason="fake-pointer validation tests run on CPU hosts only")
P = ctypes.c_void_p(4096)


def call(pos=P, **kw):
    f = dict(B=2, L=10, Hq=4, Hk=2, d=128, rot=128, interleaved=0, dtype=la.LA_DTYPE_BF16, axes=1)
    for t, h in (("q", 4), ("qo", 4), ("k", 2), ("ko", 2)):
        f.update({f"{t}_batch": 10 * h * 128, f"{t}_token": h * 128, f"{t}_head": 128})
    f.update(kw)
    s = la.RopeShape()
    for n, x in f.items():
        setattr(s, n, x)
    s.section[0] = 64
    return la.lib().la_rope(ctypes.byref(s), P, P, P, P, pos, P, ctypes.c_float(1.0), None)


@cpu_only
@pytest.mark.parametrize("axis", ["batch", "token", "head"])
@pytest.mark.parametrize("name", ["qo", "ko"])
def test_shared_output_rows_refused(name, axis):
    assert call(**{f"{name}_{axis}": 0}) == la.LA_ERR_SHAPE


@cpu_only
def test_broadcast_inputs_and_single_entries_taken():
    # the last check is that of the positions' pointer
    for name in ("q", "k"):
        for axis in ("batch", "token", "head"):
            assert call(pos=None, **{f"{name}_{axis}": 0}) == la.LA_ERR_ARG
    assert call(pos=None, B=1, qo_batch=0, ko_batch=0) == la.LA_ERR_ARG


@pytest.mark.gpu
def test_binding_refuses_an_expanded_output():
    q = torch.randn((3, 2, 5, 64), device="cuda").to(torch.bfloat16)
    pos = torch.arange(5, dtype=torch.int32, device="cuda")
    freqs = la.rope_frequencies(64)
    one = torch.zeros((1, 2, 5, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(la.LaError):
        la.rope(q, pos, freqs, out=one.expand(3, 2, 5, 64))
    with pytest.raises(la.LaError):
        la.rope(q, pos, freqs, k=q, k_out=one.expand(3, 2, 5, 64))
    torch.cuda.synchronize()
    assert bool((one == 0).all())
    # a broadcast input is turned as its copies are
    x = q[:1].expand(3, 2, 5, 64)
    assert torch.equal(la.rope(x, pos, freqs), la.rope(x.contiguous(), pos, freqs))
    assert torch.equal(la.rope(q[:1], pos, freqs, out=one.expand(1, 2, 5, 64)), la.rope(q[:1], pos, freqs))
