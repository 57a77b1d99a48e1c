"""Seeded random packed batches through the attention with and without a relative bias and its gradients, against 64
bits: lengths from none to thousands, so that units are whole, cut once and cut often, and borders move; grouped heads,
masks, reaches and types."""
import random

import pytest
import torch

from paper_2605_31158_amd import la
import grad_reference as G
import seq_reference as R
from test_prompt_bias_gpu import make, rel

pytestmark = pytest.mark.gpu


def problem(seed):
    r = random.Random(seed)
    most = r.choice([3, 40, 130, 600, 1500, 2600])
    S = max(1, min(r.choice([1, 2, 5, 17, 70]), 5000 // most))
    length = lambda: 0 if r.random() < 0.1 else r.randint(1, most)            # noqa: E731
    lq = [length() for _ in range(S)]
    form = r.choice(["same", "more", "any"])
    lk = [n if form == "same" else n + r.randint(0, 300) if form == "more" else length() for n in lq]
    Hkv = r.choice([1, 1, 2, 3])
    Hq = Hkv * r.choice([1, 1, 2, 3, 5])
    both = r.random() < 0.5
    bias = None if r.random() < 0.3 else (r.choice([4, 8, 32, 64]), r.randint(33, 256 if both else 512), both,
                                          r.choice([torch.float32, torch.bfloat16]))
    return lq, lk, Hq, Hkv, r.choice([64, 128]), r.random() < 0.5, bias


@pytest.mark.parametrize("seed", range(32))
def test_random(seed):
    lq, lk, Hq, Hkv, d, causal, form = problem(seed)
    what = f"seed {seed}: {len(lq)} of up to {max(lq)} over {max(lk)}, {Hq} over {Hkv}, d {d}, causal {causal}, bias {form}"
    print(f"[random] {what}", flush=True)
    q, k, v = make(lq, lk, Hq, Hkv, d, 100 + seed)
    bias = None if form is None else rel(Hq, 200 + seed, *form)
    cu_q, cu_k = R.starts(lq), R.starts(lk)
    o, lse = la.prompt_attn(q, k, v, cu_q, cu_k, causal=causal, want_lse=True, bias=bias)
    R.check(o, lse, G.forward(q, k, v, lq, lk, causal, bias=bias), what)
    do = torch.randn(q.shape, generator=torch.Generator(device="cuda").manual_seed(300 + seed), device="cuda").to(torch.bfloat16)
    got = la.prompt_attn_bwd(do, q, k, v, o, lse, cu_q, cu_k, causal=causal, bias=bias)
    G.check(got, G.backward(do, q, k, v, o, lse, lq, lk, causal, bias=bias), what)
