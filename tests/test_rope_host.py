"""Host side of the rotary positions: frequency tables, positions of a grid, refusals."""
import ctypes
import math

import pytest
import torch

from paper_2605_31158_amd import la

cpu_only = pytest.mark.skipif(torch.cuda.is_available(), reason="fake-pointer validation tests run on CPU hosts only")


def freqs(*a, **kw):
    return la.rope_frequencies(*a, device="cpu", **kw)


def test_plain_ladder_and_sections():
    f = freqs(64, base=10000.0)
    assert f.dtype == torch.float64 and f.shape == (32,)
    for j in (0, 1, 31):
        assert float(f[j]) == pytest.approx(10000.0 ** (-2 * j / 64), rel=1e-14)
    f = freqs(128, sections=(22, 21, 21))
    assert f.shape == (64,) and float(f[0]) == float(f[22]) == float(f[43]) == 1.0
    assert float(f[21]) == pytest.approx(10000.0 ** (-21 / 22), rel=1e-14)
    assert float(f[63]) == pytest.approx(10000.0 ** (-20 / 21), rel=1e-14)
    assert freqs(64, sections=(0, 32)).shape == (32,)


def test_scalings():
    plain = freqs(128)
    assert torch.allclose(freqs(128, scaling="linear", factor=8.0), plain / 8, rtol=1e-14, atol=0)
    f = freqs(128, scaling="base", factor=8.0)
    assert float(f[0]) == 1.0 and float(f[-1]) == pytest.approx(float(plain[-1]) / 8, rel=1e-12)
    f = freqs(128, scaling="ramp", factor=32.0, trained=4096, turns=(1.0, 32.0))
    for j in range(64):
        n = 4096 * float(plain[j]) / (2 * math.pi)
        keep = min(1.0, max(0.0, (n - 1) / 31))
        assert float(f[j]) == pytest.approx(float(plain[j]) * (keep + (1 - keep) / 32), rel=1e-12)
    assert float(f[0]) == 1.0 and float(f[-1]) == pytest.approx(float(plain[-1]) / 32, rel=1e-12)


@pytest.mark.parametrize("kw", [dict(rot=3), dict(rot=0), dict(rot=64, base=0.0), dict(rot=64, factor=0.0),
                                dict(rot=64, scaling="x"), dict(rot=64, scaling="ramp"),
                                dict(rot=64, scaling="ramp", trained=10, turns=(3.0, 3.0)),
                                dict(rot=64, sections=(10, 10)), dict(rot=64, sections=(40, -8)),
                                dict(rot=64, sections=(16, 16), scaling="base"), dict(rot=2, scaling="base")], ids=str)
def test_frequencies_refused(kw):
    with pytest.raises(ValueError):
        freqs(**kw)


def test_grid_positions():
    g = la.grid3d(1, 2, 64, 5, 2, 1, 3, 4, 1, 2, 2, 64)
    q, k = la.grid3d_positions(g, device="cpu")
    assert q.shape == (3, 12) and k.shape == (3, 5 + 36) and q.dtype == torch.int32
    assert bool((k[:, :5] == 0).all())
    for n, (t, y, x) in enumerate((t, y, x) for t in range(3) for y in range(3) for x in range(4)):
        assert k[:, 5 + n].tolist() == [t, y, x]
    assert torch.equal(q, k[:, 5 + 24:])
    q, k = la.grid3d_positions(g, frames=[7, 30, 31], device="cpu")
    assert k[0, 5].item() == 7 and k[0, 5 + 12].item() == 30 and q[0, 0].item() == 31
    with pytest.raises(ValueError):
        la.grid3d_positions(g, frames=[1, 2])


P = ctypes.c_void_p(4096)
ODD = ctypes.c_void_p(4100)


def call(q=P, qo=P, k=P, ko=P, pos=P, fr=P, amp=1.0, section=(64, 0, 0), none=False, **kw):
    f = dict(B=1, L=10, Hq=4, Hk=2, d=128, rot=128, interleaved=0, dtype=la.LA_DTYPE_BF16, axes=1)
    for t, h in (("q", 4), ("qo", 4), ("k", 2), ("ko", 2)):
        f.update({f"{t}_batch": 10 * h * 128, f"{t}_token": h * 128, f"{t}_head": 128})
    f.update(kw)
    names = [n for n, _ in la.RopeShape._fields_]
    s = la.RopeShape(*[(ctypes.c_int32 * 3)(*section) if n == "section" else f[n] for n in names])
    return la.lib().la_rope(None if none else ctypes.byref(s), q, qo, k, ko, pos, fr, ctypes.c_float(amp), None)


@cpu_only
@pytest.mark.parametrize("bad", [dict(B=-1), dict(L=-1), dict(Hq=-1), dict(Hk=-1), dict(d=96), dict(rot=0), dict(rot=24),
                                 dict(rot=144), dict(interleaved=2), dict(axes=0), dict(axes=4), dict(B=65536),
                                 dict(section=(60, 0, 0)), dict(section=(60, 4, 0)), dict(axes=2, section=(70, -6, 0)),
                                 dict(q_token=12), dict(k_head=-8), dict(qo_head=0), dict(ko_token=0), dict(q_batch=4)],
                         ids=str)
def test_rope_shapes_refused(bad):
    assert call(**bad) == la.LA_ERR_SHAPE


@cpu_only
def test_rope_arguments_refused():
    assert call(none=True) == la.LA_ERR_ARG
    for name in ("q", "qo", "k", "ko", "pos", "fr"):
        assert call(**{name: None}) == la.LA_ERR_ARG, name
    for name in ("q", "qo", "k", "ko"):
        assert call(**{name: ODD}) == la.LA_ERR_ARG, name
    assert call(pos=ctypes.c_void_p(4098)) == la.LA_ERR_ARG
    assert call(fr=ODD) == la.LA_ERR_ARG
    assert call(dtype=7) == la.LA_ERR_ARG
    assert call(amp=float("nan")) == la.LA_ERR_ARG and call(amp=float("inf")) == la.LA_ERR_ARG
    for empty in (dict(B=0), dict(L=0), dict(Hq=0, Hk=0)):
        assert call(q=None, qo=None, k=None, ko=None, pos=None, fr=None, **empty) == la.LA_OK


def test_binding_refuses_cpu_tensors():
    with pytest.raises(TypeError):
        la.rope(torch.zeros(4, 2, 64), torch.zeros(4, dtype=torch.int32), torch.zeros(32, dtype=torch.float64))


@cpu_only
def test_rope_sizes_past_the_limit_refused():
    assert call(L=(1 << 26) - 3) == la.LA_ERR_SHAPE
    assert call(L=(1 << 31) - 1) == la.LA_ERR_SHAPE
