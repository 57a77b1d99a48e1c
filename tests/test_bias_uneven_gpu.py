"""A relative bias over batches in which one sequence has nearly all keys, in units that are cut, against 64 bits."""
import pytest
import torch

from paper_2605_31158_amd import la
import grad_reference as G
import seq_reference as R
from test_prompt_bias_gpu import make, rel

pytestmark = pytest.mark.gpu

CASES = [
    # (query lengths, key lengths or None for the same, Hq, Hkv, d, causal)
    ([10] * 7 + [3800] + [10] * 8, None, 4, 4, 64, False),
    ([3800] + [10] * 15, None, 2, 1, 128, True),
    ([1] * 16, [13] * 15 + [3900], 8, 2, 64, True),
    ([1] * 16, [3900] + [13] * 15, 16, 16, 128, True),
    ([20] * 16, [13] * 3 + [3900] + [13] * 12, 5, 5, 64, False),
    ([100] * 16, [2400] + [100] * 15, 3, 3, 128, True),
    ([2000] + [6] * 15, None, 2, 2, 64, False),               # whole units
]


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_one_long_sequence(case):
    lq, lk, Hq, Hkv, d, causal = case
    lk = lq if lk is None else lk
    print(f"[uneven] {str(lq)[:40]} over {str(lk)[:40]} {case[2:]}", flush=True)
    q, k, v = make(lq, lk, Hq, Hkv, d, 181)
    bias = rel(Hq, 182, both=not causal)
    cu_q, cu_k = R.starts(lq), R.starts(lk)
    o, lse = la.prompt_attn(q, k, v, cu_q, cu_k, causal=causal, want_lse=True, bias=bias)
    torch.cuda.synchronize()
    R.check(o, lse, G.forward(q, k, v, lq, lk, causal, bias=bias), str(case)[:80])
    again, lse2 = la.prompt_attn(q, k, v, cu_q, cu_k, causal=causal, want_lse=True, bias=bias)
    assert torch.equal(o, again) and torch.equal(lse, lse2)
