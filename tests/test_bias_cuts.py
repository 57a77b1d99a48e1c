"""Which calls with a relative bias work on whole units, without pieces and their join (and so without scratch): those
whose lengths cannot leave most of the work to few workgroups.  Sizes alone decide; nothing here enqueues a kernel."""
import ctypes

import pytest

from paper_2605_31158_amd import la


def scratch(S, Tq, Tk, Hq, Hkv, d):
    s = la.Seqs(**dict(S=S, Tq=Tq, Tk=Tk, Hq=Hq, Hkv=Hkv, d=d, causal=0, q_token=Hq * d, q_head=d, o_token=Hq * d, o_head=d,
                       k_token=Hkv * d, k_head=d, v_token=Hkv * d, v_head=d))
    b = la.RelBias(-128, 128, 32, 0)
    return la.lib().la_prompt_bias_ws_bytes(ctypes.byref(s), ctypes.byref(b))


@pytest.mark.parametrize("call", [
    # batches that may hold one long sequence, whose few units would be walked by as many workgroups
    (16, 3950, 3950, 1, 1, 64), (16, 3950, 3950, 4, 4, 64), (16, 4095, 4095, 4, 1, 128), (16, 3950, 3950, 7, 7, 64),
    # single tokens, and few queries over many keys
    (16, 16, 4095, 2, 2, 64), (16, 16, 4095, 16, 4, 128), (16, 16, 4095, 32, 32, 64), (16, 320, 4095, 16, 16, 64),
    (16, 1600, 3900, 16, 16, 64),
    # many keys
    (20, 4199, 4199, 16, 16, 64), (8, 16, 6000, 16, 16, 64),
], ids=str)
def test_cut(call):
    assert scratch(*call) > 0


@pytest.mark.parametrize("call", [
    (1, 1024, 1024, 1, 1, 64), (20, 2000, 2000, 2, 2, 64), (30, 30, 2040, 16, 16, 64), (16, 3344, 3344, 16, 16, 64),
    (16, 3344, 3344, 8, 8, 64), (16, 3344, 3344, 16, 4, 64), (8, 4096, 4096, 16, 16, 128), (8, 4096, 4096, 8, 8, 128),
    (16, 3950, 3950, 16, 16, 64),
], ids=str)
def test_whole(call):
    assert scratch(*call) == 0
