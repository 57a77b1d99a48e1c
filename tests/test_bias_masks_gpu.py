"""Rows whose visible keys all carry a large finite weight as a mask (la_rel_bias): forward and gradients against the
softmax in 64 bits, in which such a weight cancels."""
import pytest
import torch

from paper_2605_31158_amd import la
import grad_reference as G
import seq_reference as R
from test_prompt_bias_gpu import make, rel

pytestmark = pytest.mark.gpu

MOST = 2.0 ** 14                     # what finite weights are held to


def reference(do, q, k, v, o, lq, lk, causal, bias):
    """{name: (value, bound)} of o, lse and the gradients, delta from the o that is given.

    Roundings of a logit beside those of grad_reference, in F32 of |b|: the table in base 2 over the scale 3, the
    accumulators that start from it 8 (4 products, twice a rounding's half step where one truncates), the exponent 2.
    lse repeats them and adds its maximum, its sum and the change of base, 3 of |lse|; P in the backward call has lse's
    error for a whole row, lse's change of base and the difference, 2 of |lse|, and its own logit's, 4 of |x| + |b|."""
    T, Hq, d = q.shape
    G_, U, F = Hq // k.shape[1], G.U, G.F32
    scale = d ** -0.5
    z = lambda x, n=1: [torch.zeros(x, dtype=torch.float64, device=q.device) for _ in range(2 * n)]   # noqa: E731
    out = {"o": z(q.shape), "lse": z((T, Hq)), "dq": z(q.shape), "dk": z(k.shape), "dv": z(v.shape),
           "dw": z(bias[0].shape)}
    chain = 64 + sum((m / 64 + 2) * (n / 128 + 2) for n, m in zip(lq, lk))
    a = c = 0
    for n, m in zip(lq, lk):
        rows, keys = slice(a, a + n), slice(c, c + m)
        a, c = a + n, c + m
        see = G.seen(n, m, causal, q.device)
        for h in range(Hq):
            qh, kh, vh, g = (x.double() for x in (q[rows, h], k[keys, h // G_], v[keys, h // G_], do[rows, h]))
            w, to = G.biased(*bias, h, n, m)
            w = torch.where(torch.isinf(w), w, w.clamp(-MOST, MOST))
            x = torch.where(see, qh @ kh.T * scale + w, -torch.inf)
            lse = torch.logsumexp(x, -1)
            p = torch.exp(x - lse[:, None])
            out["lse"][0][rows, h] = lse
            out["o"][0][rows, h] = p @ vh
            # of the pairs that carry a weight: the others' logits have no part in the row
            size = (qh.abs() @ kh.abs().T) * scale
            heavy = torch.where(p > 0, w.abs(), 0.0).amax(-1)
            e_f = ((d + 4) * F * size.amax(-1) + (m / 64 + 64) * F + 13 * F * heavy)[:, None]
            t = (U + 2 * e_f) * (p @ vh.abs())
            out["o"][1][rows, h] = t + U * ((p @ vh).abs() + t)
            out["lse"][1][rows, h] = e_f[:, 0] + 3 * F * lse.abs()
            e = e_f + 5 * F * lse.abs()[:, None] + (d + 4) * F * size + 4 * F * (
                torch.where(p > 0, x.abs() + w.abs(), 0.0) + 2)
            oh = o[rows, h].double()
            ds = p * (g @ vh.T - (g * oh).sum(-1)[:, None])
            r = (d + 4) * F * (g.abs() @ vh.abs().T + (g * oh).abs().sum(-1)[:, None])
            w_ds = 2 * e * ds.abs() + p * r
            s = F * (max(n, m) / 16 + 64)
            r_ds = (U + s) * ds.abs() + 2 * w_ds
            for name, at, y, b in (("dq", (rows, h), scale * (ds @ kh), scale * (r_ds @ kh.abs())),
                                   ("dk", (keys, h // G_), scale * (ds.T @ qh), scale * (r_ds.T @ qh.abs())),
                                   ("dv", (keys, h // G_), p.T @ g, ((U + s + 2 * e) * p).T @ g.abs())):
                out[name][0][at] += y
                out[name][1][at] += b
            t = w_ds + chain * F * ds.abs()
            for i in to.unique().tolist():
                if i >= 0:
                    out["dw"][0][i, h] += ds[to == i].sum()
                    out["dw"][1][i, h] += t[to == i].sum()
    last = {"o": 0.0, "lse": G.F32, "dw": U if bias[0].dtype is torch.bfloat16 else G.F32}
    return {n: (x, t + last.get(n, U) * (x.abs() + t)) for n, (x, t) in out.items()}


@pytest.mark.parametrize("low", [-1e4, -1e6, -1e9, None, 1e9], ids=["-1e4", "-1e6", "-1e9", "lowest", "1e9"])
@pytest.mark.parametrize("form", [(64, [1, 40, 200], True, torch.float32), (128, [1, 40, 200], True, torch.bfloat16),
                                  (64, [1100], True, torch.bfloat16), (128, [1100], False, torch.float32),
                                  (64, [130, 77], False, torch.float32)], ids=str)
def test_rows_of_masked_keys_alone(form, low):
    d, lq, causal, dtype = form
    print(f"[masks] {form} {low}", flush=True)
    q, k, v = make(lq, lq, 4, 2, d, 71)
    cu = R.starts(lq)
    bias = rel(4, 72, dtype=dtype, both=not causal)
    value = torch.finfo(dtype).min if low is None else low
    # head 0: its own place, so that the first token of a causal text sees nothing else; head 1: everything; head 2: all
    # beyond the one before
    bias.weight[0, 0] = bias.weight[:, 1] = bias.weight[2:, 2] = value
    do = torch.randn(q.shape, generator=torch.Generator(device="cuda").manual_seed(73), device="cuda").to(torch.bfloat16)
    o, lse = la.prompt_attn(q, k, v, cu, causal=causal, want_lse=True, bias=bias)
    got = (o, lse, *la.prompt_attn_bwd(do, q, k, v, o, lse, cu, causal=causal, bias=bias))
    G.check(got, reference(do, q, k, v, o, lq, lq, causal, bias), f"{form} {low}")
