"""64-bit reference of the operators over packed sequences, and the bounds that their outputs are held to.

U: half a step of bf16.  The kernels' weights are rounded to bf16 before they meet the values, and the
output is rounded once: with A = sum_j w_j |v_j| an output element is within U A of the first rounding
and U |o| of the second.  The logits are sums of d products in fp32, off by at most
E = (d + 4) 2^-24 scale sum |q k|, which moves a weight (and their sum) by at most E of itself, and the
exponentials and sums of n keys in fp32 add (n / 64 + 64) 2^-24: partial sums run over 64-key tiles.
"""
import torch

U = 2.0 ** -8
F32 = 2.0 ** -24


def starts(lengths, device="cuda"):
    c = [0]
    for n in lengths:
        c.append(c[-1] + n)
    return torch.tensor(c, dtype=torch.int32, device=device)


def attention(q, keys, lq, lk, causal, scale=None):
    """q [T, Hq, d]; keys(s, h) -> K and V [lk[s], d] of sequence s and key head h; lq, lk per sequence.
    Returns o, lse, and the bounds of both, [T, Hq, d] and [T, Hq] in float64."""
    T, Hq, d = q.shape
    scale = d ** -0.5 if scale is None else scale
    dev = q.device
    o, lse, tol, ltol = (torch.zeros(s, dtype=torch.float64, device=dev) for s in ((T, Hq, d), (T, Hq), (T, Hq, d), (T, Hq)))
    q = q.double()
    t0 = 0
    for s, (n, m) in enumerate(zip(lq, lk)):
        rows = slice(t0, t0 + n)
        t0 += n
        if n == 0:
            continue
        last = torch.full((n,), m - 1, device=dev)
        if causal:
            last = torch.arange(n, device=dev) + (m - n)
        seen = torch.arange(m, device=dev)[None] <= last[:, None]
        none = ~seen.any(-1) if m else torch.ones(n, dtype=torch.bool, device=dev)
        for h in range(Hq):
            if m == 0:
                lse[rows, h] = -torch.inf
                continue
            k, v = (x.double() for x in keys(s, h))
            # a key or value that no weight belongs to is never touched
            x = (q[rows, h] @ k.T) * scale
            x = torch.where(seen, x, -torch.inf)
            top = torch.where(none, 0.0, x.amax(-1))
            w = torch.where(seen, torch.exp(x - top[:, None]), 0.0)
            total = w.sum(-1)
            w = w / torch.where(none, 1.0, total)[:, None]
            o[rows, h] = w @ v
            lse[rows, h] = torch.where(none, -torch.inf, top + torch.log(total))
            size = (q[rows, h].abs() @ k.abs().T) * scale
            e = (d + 4) * F32 * torch.where(seen, size, 0.0).amax(-1) + (m / 64 + 64) * F32
            tol[rows, h] = (U + 2 * e[:, None]) * (w @ v.abs()) * (1 + U) + U * o[rows, h].abs()
            ltol[rows, h] = e + 2 * F32 * lse[rows, h].abs().nan_to_num(posinf=0.0)
    return o, lse, tol, ltol


def check(got, lse, want, what=""):
    """Outputs against attention()'s; prints the largest share of the bound that is used."""
    o_ref, lse_ref, tol, ltol = want
    err = (got.double() - o_ref).abs()
    assert torch.isfinite(got).all(), f"{what}: outputs that are not finite"
    used = float((err / tol.clamp(min=1e-30)).max()) if err.numel() else 0.0
    lused = 0.0
    if lse is not None:
        fin = torch.isfinite(lse_ref)
        assert torch.equal(fin, torch.isfinite(lse)) and bool((lse[~fin] == -torch.inf).all()), f"{what}: lse of empty rows"
        d = (lse.double() - lse_ref).abs()[fin] / ltol[fin]
        lused = float(d.max()) if d.numel() else 0.0
    print(f"[seq] {what}: {used:.3f} of the bound (lse {lused:.3f})", flush=True)
    assert used <= 1.0 and lused <= 1.0, (what, used, lused)
