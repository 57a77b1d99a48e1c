"""la_kv4_attn's max_q where both of its kernels, or the one for many query rows alone, have the work:
sequences of more query rows are left as they are, the others are those of a call that takes all."""
import ctypes

import pytest
import torch

from paper_2605_31158_amd import la
import seq_reference as R
from test_kv4_gpu import filled

pytestmark = pytest.mark.gpu

CASES = [
    # (queries, lengths, max_q)
    ([210, 300, 3], [400, 350, 90], 300),          # both kernels, nothing left out
    ([210, 300, 3], [400, 350, 90], 250),          # a sequence of the second kernel left out
    ([210, 300, 3], [400, 350, 90], 209),          # all but those of the first
    ([300, 1, 0, 220, 251], [310, 40, 7, 100, 700], 250),
    ([300], [500], 300),                           # a single sequence: the second kernel alone
    ([240], [500], 250),
    ([300], [500], 250),                           # and nothing to do
    ([100], [500], 250),                           # a single short one, with rows of no sequence behind it
]


@pytest.mark.parametrize("wide", [True, False], ids=["wide", "narrow"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", CASES, ids=[f"{c[0]} max {c[2]}" for c in CASES])
def test_longer_sequences_are_left_out(case, d, wide):
    lq, lens, max_q = case
    Hq, Hkv, page, spare = 4, 2, 16, 160 if lq == [100] else 2
    T = sum(lq)
    print(f"[kv4 max_q] {lq} over {lens} d {d} max_q {max_q} wide {wide}", flush=True)
    cache, table, L, k, v = filled(lens, Hkv, d, page, 11)
    if wide:
        # more columns, none of them of a page: the second kernel's work by the rule on the most there can be
        table = torch.cat([table, torch.full((len(lens), 10 ** 8 // (T * Hq * page)), -1, dtype=torch.int32,
                                             device="cuda")], 1).contiguous()
        seqs = la.Seqs(len(lens), T + spare, 0, Hq, Hkv, d, 1, Hq * d, d, Hq * d, d, 0, 0, 0, 0)
        kv = la.Kv4(cache.shape[0], page, table.shape[1])
        # its partials of 256 rows take more than all of the first kernel's
        assert la.lib().la_kv4_ws_bytes(ctypes.byref(seqs), ctypes.byref(kv), max_q) > 2 * 512 * 32 * (d + 2) * 4 + 65536
    q = (torch.randn((T + spare, Hq, d), device="cuda") * 1.5).to(torch.bfloat16)
    at = [sum(lens[:s]) for s in range(len(lens))]
    want = R.attention(q[:T], lambda s, h: (k[at[s]: at[s] + lens[s], h // 2], v[at[s]: at[s] + lens[s], h // 2]), lq, lens,
                       True)
    out, lse = torch.full_like(q, 7.0), torch.full((T + spare, Hq), 7.0, device="cuda")
    la.kv4_attn(q, cache, R.starts(lq), L, table, max_q, out=out, lse_out=lse)
    torch.cuda.synchronize()
    row = 0
    for s, n in enumerate(lq):
        rows = slice(row, row + n)
        row += n
        if n > max_q:
            assert bool((out[rows] == 7).all()) and bool((lse[rows] == 7).all()), s
        else:
            R.check(out[rows], lse[rows], [x[rows] for x in want], f"sequence {s}")
    assert bool((out[T:] == 7).all()) and bool((lse[T:] == 7).all())
