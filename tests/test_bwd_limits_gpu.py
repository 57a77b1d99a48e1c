"""Calls of la_prompt_attn_bwd at the ends of what it takes: starts that do not fit the rows, and far more buckets than
distances."""
import pytest
import torch

from paper_2605_31158_amd import la
import grad_reference as G
import seq_reference as R
from test_prompt_bias_gpu import make, rel
from test_prompt_bwd_gpu import grad_of, left

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("biased", [False, True], ids=["plain", "bias"])
@pytest.mark.parametrize("starts,lengths", [([0, 60, 60, 4000, 2 ** 31 - 1, -5], [60, 40]), ([-7, 30, 10, 10], [30]),
                                            ([90, 2 ** 31 - 1], [10])], ids=str)
def test_starts_held_to_the_rows(starts, lengths, d, biased):
    # starts past the rows, before them, or before the one in front: held to what is there, and nothing else is written
    T, first = 100, max(starts[0], 0)
    q, k, v = make([T], [T], 4, 2, d, 191)
    bias = rel(4, 192) if biased else None
    rows = slice(first, first + sum(lengths))
    o, lse = torch.zeros_like(q), torch.zeros((T, 4), device="cuda")
    o[rows], lse[rows] = left(q[rows], k[rows], v[rows], lengths, lengths, True, bias=bias)
    do = grad_of(q, 193)
    want = G.backward(do[rows], q[rows], k[rows], v[rows], o[rows], lse[rows], lengths, lengths, True, bias=bias)
    cu = torch.tensor(starts, dtype=torch.int32, device="cuda")
    held = [torch.full((T + 40, x.shape[1], d), 7.0, dtype=torch.bfloat16, device="cuda") for x in (q, k, v)]
    outs = tuple(x[20: 20 + T] for x in held) + ((torch.full_like(bias.weight, 7.0),) if biased else ())
    la.prompt_attn_bwd(do, q, k, v, o, lse, cu, bias=bias, out=outs)
    G.check([x[rows] for x in outs[:3]] + list(outs[3:]), want, f"{starts} {d} {biased}")
    for x in held:
        x[20 + rows.start: 20 + rows.stop] = 7.0
        assert bool((x == 7).all())
