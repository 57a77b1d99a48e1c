"""Queries that see no key, behind a mask or weights of -inf: they have no gradients and give none, whatever their rows of
q, do and dlse hold (la_prompt_attn_bwd)."""
import pytest
import torch

from paper_2605_31158_amd import la
import grad_reference as G
import seq_reference as R
from test_prompt_bias_gpu import make, rel
from test_prompt_bwd_gpu import grad_of, left

pytestmark = pytest.mark.gpu

FORMS = [
    # (query lengths, key lengths, Hq, Hkv): causal, the first lq - lk queries of a sequence see nothing
    ([150, 40], [100, 90], 4, 2),
    ([40, 3, 70], [37, 0, 5], 6, 2),
    ([700, 65], [600, 64], 2, 2),
    ([131], [130], 8, 1),
]


@pytest.mark.parametrize("form", FORMS, ids=str)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("biased", [False, True], ids=["plain", "bias"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")], ids=str)
def test_behind_the_mask(form, d, biased, value):
    lq, lk, Hq, Hkv = form
    print(f"[empty] {form} {d} {biased} {value}", flush=True)
    q, k, v = make(lq, lk, Hq, Hkv, d, 171)
    bias = rel(Hq, 172, both=False) if biased else None
    cu_q, cu_k = R.starts(lq), R.starts(lk)
    o, lse = left(q, k, v, lq, lk, True, bias=bias)
    do = grad_of(q, 173)
    dlse = torch.randn(lse.shape, generator=torch.Generator(device="cuda").manual_seed(174), device="cuda")
    none = lse == -torch.inf
    assert bool(none.any())
    q[none] = do[none] = 0.0
    dlse[none] = 0.0
    want = la.prompt_attn_bwd(do, q, k, v, o, lse, cu_q, cu_k, bias=bias, dlse=dlse)
    G.check(want, G.backward(do, q, k, v, o, lse, lq, lk, True, bias=bias, dlse=dlse), "zeros")
    assert bool((want[0][none] == 0).all())
    q[none] = do[none] = value
    dlse[none] = value
    got = la.prompt_attn_bwd(do, q, k, v, o, lse, cu_q, cu_k, bias=bias, dlse=dlse)
    for x, y in zip(got, want):
        assert torch.equal(x, y)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_behind_weights_that_hide(d, causal):
    # head 0 sees nothing at all, of head 1 the rows that only reach what is hidden; q stays finite: a logit of NaN is no
    # hidden one
    lq, lk = [90, 200, 3], [40, 260, 3]
    q, k, v = make(lq, lk, 4, 2, d, 175)
    bias = rel(4, 176)
    bias.weight[:, 0] = -torch.inf
    bias.weight[:8, 1] = -torch.inf
    cu_q, cu_k = R.starts(lq), R.starts(lk)
    o, lse = left(q, k, v, lq, lk, causal, bias=bias)
    do = grad_of(q, 177)
    none = lse == -torch.inf
    do[none] = 0.0
    want = la.prompt_attn_bwd(do, q, k, v, o, lse, cu_q, cu_k, causal=causal, bias=bias)
    G.check(want, G.backward(do, q, k, v, o, lse, lq, lk, causal, bias=bias), "zeros")
    do[none] = float("nan")
    got = la.prompt_attn_bwd(do, q, k, v, o, lse, cu_q, cu_k, causal=causal, bias=bias)
    for x, y in zip(got, want):
        assert torch.equal(x, y)
