"""64-bit reference of the relative bias and of the attention's gradients, and the bounds that the kernels' outputs
are held to.

U is half a step of bf16, F32 of fp32 (relative).  With x = scale q.k + b, P = exp(x - lse), dP = do.v,
delta = do.o - dlse and dS = P (dP - delta):
  x       is a sum of d products in fp32, off by (d + 4) F32 scale sum |q k|, and x, b and lse are each rounded
          a few times on their way to the exponential: e = that + 4 F32 (|x| + |b| + |lse| + 2) moves P by e of itself.
  dP, delta  are off by (d + 4) F32 of the sums of their products' magnitudes, r together.
  dS      is off by w = 2 e |dS| + P r.
  dv      sums P do with P rounded to bf16: (U + 2 e) P |do|;  dq and dk sum dS with dS rounded: U |dS| + 2 w,
          times |k| and |q|; sums of n fp32 terms over MFMAs of 32 add n / 16 + 64 roundings at most.
  dweight sums dS in fp32: 32 of a lane and tile, then a chain of the tiles and units, then 64 bits.
The results are rounded once: U (bf16) or F32 (fp32) of themselves.
"""
import torch

U = 2.0 ** -8
F32 = 2.0 ** -24


def biased(weight, bucket, lo, h, n, m):
    """(bias [n, m], bucket index [n, m]) of head h in float64; a bucket outside the weights' rows: 0, -1."""
    place = torch.arange(n, device=weight.device)[:, None] + (m - n)
    at = (torch.arange(m, device=weight.device)[None] - place).clamp(lo, lo + bucket.numel() - 1) - lo
    to = bucket.long()[at]
    ok = (to >= 0) & (to < weight.shape[0])
    to = torch.where(ok, to, -1)
    return torch.where(ok, weight.double()[to.clamp(min=0), h], 0.0), to


def seen(n, m, causal, dev):
    last = torch.full((n,), m - 1, device=dev)
    if causal:
        last = torch.arange(n, device=dev) + (m - n)
    return torch.arange(m, device=dev)[None] <= last[:, None]


def forward(q, k, v, lq, lk, causal, scale=None, bias=None):
    """o, lse and their bounds, as seq_reference.attention, with a bias (weight, bucket, lo)."""
    T, Hq, d = q.shape
    G = Hq // k.shape[1]
    scale = d ** -0.5 if scale is None else scale
    dev = q.device
    o, tol = (torch.zeros((T, Hq, d), dtype=torch.float64, device=dev) for _ in range(2))
    lse, ltol = (torch.zeros((T, Hq), dtype=torch.float64, device=dev) for _ in range(2))
    a = b = 0
    for n, m in zip(lq, lk):
        rows, keys = slice(a, a + n), slice(b, b + m)
        a, b = a + n, b + m
        if n == 0:
            continue
        see = seen(n, m, causal, dev)
        for h in range(Hq):
            if m == 0:
                lse[rows, h] = -torch.inf
                continue
            qh, kh, vh = q[rows, h].double(), k[keys, h // G].double(), v[keys, h // G].double()
            x = (qh @ kh.T) * scale
            extra = 0.0
            if bias is not None:
                w = biased(*bias, h, n, m)[0]
                x = x + w
                extra = torch.where(see & torch.isfinite(w), w.abs(), 0.0).amax(-1)
            x = torch.where(see, x, -torch.inf)
            top = x.amax(-1)
            none = top == -torch.inf
            p = torch.exp(x - torch.where(none, 0.0, top)[:, None])
            total = p.sum(-1)
            p = p / torch.where(none, 1.0, total)[:, None]
            o[rows, h] = p @ vh
            lse[rows, h] = torch.where(none, -torch.inf, top + torch.log(total))
            size = torch.where(see, (qh.abs() @ kh.abs().T) * scale, 0.0).amax(-1)
            e = (d + 4) * F32 * size + (m / 64 + 64) * F32 + 4 * F32 * extra
            tol[rows, h] = (U + 2 * e[:, None]) * (p @ vh.abs()) * (1 + U) + U * o[rows, h].abs()
            ltol[rows, h] = e + 2 * F32 * lse[rows, h].abs().nan_to_num(posinf=0.0)
    return o, lse, tol, ltol


def backward(do, q, k, v, o, lse, lq, lk, causal, scale=None, bias=None, dlse=None):
    """{name: (gradient, bound)} for dq, dk, dv and, with a bias, dw."""
    T, Hq, d = q.shape
    G = Hq // k.shape[1]
    scale = d ** -0.5 if scale is None else scale
    dev = q.device
    z = lambda x: torch.zeros(x.shape, dtype=torch.float64, device=dev)   # noqa: E731
    out = {n: (z(x), z(x)) for n, x in (("dq", q), ("dk", k), ("dv", v))}
    chain = 64 + sum((m / 64 + 2) * (n / 128 + 2) for n, m in zip(lq, lk))
    if bias is not None:
        out["dw"] = (z(bias[0]), z(bias[0]))
    a = b = 0
    for n, m in zip(lq, lk):
        rows, keys = slice(a, a + n), slice(b, b + m)
        a, b = a + n, b + m
        if n == 0 or m == 0:
            continue
        see = seen(n, m, causal, dev)
        for h in range(Hq):
            qh, kh, vh = q[rows, h].double(), k[keys, h // G].double(), v[keys, h // G].double()
            g, oh, ls = do[rows, h].double(), o[rows, h].double(), lse[rows, h].double()
            none = ls == -torch.inf
            x = (qh @ kh.T) * scale
            size = torch.zeros_like(x)
            if bias is not None:
                w, to = biased(*bias, h, n, m)
                x = x + w
                size = torch.where(torch.isfinite(w), w.abs(), 0.0)
            p = torch.where(see & ~none[:, None], torch.exp(x - torch.where(none, 0.0, ls)[:, None]), 0.0)
            dp = g @ vh.T
            delta = (g * oh).sum(-1)
            if dlse is not None:
                delta = delta - dlse[rows, h].double()
            ds = p * (dp - torch.where(none, 0.0, delta)[:, None])
            finite = torch.where(torch.isfinite(x), x.abs(), 0.0)
            e = (d + 4) * F32 * scale * (qh.abs() @ kh.abs().T) + 4 * F32 * (
                finite + size + torch.where(none, 0.0, ls.abs())[:, None] + 2)
            r = (d + 4) * F32 * (g.abs() @ vh.abs().T + (g * oh).abs().sum(-1)[:, None])
            if dlse is not None:
                r = r + 2 * F32 * torch.where(none, 0.0, dlse[rows, h].double().abs())[:, None]
            w_ds = 2 * e * ds.abs() + p * r
            s = F32 * (max(n, m) / 16 + 64)
            r_ds = (U + s) * ds.abs() + 2 * w_ds
            add = lambda name, at, x, t: (out[name][0][at].add_(x), out[name][1][at].add_(t))   # noqa: E731
            add("dq", (rows, h), scale * (ds @ kh), scale * (r_ds @ kh.abs()))
            add("dk", (keys, h // G), scale * (ds.T @ qh), scale * (r_ds.T @ qh.abs()))
            add("dv", (keys, h // G), p.T @ g, ((U + s + 2 * e) * p).T @ g.abs())
            if bias is not None:
                t = w_ds + chain * F32 * ds.abs()
                for i in to.unique().tolist():
                    if i >= 0:
                        add("dw", (i, h), ds[to == i].sum(), t[to == i].sum())
    last = {"dw": U if bias is not None and bias[0].dtype is torch.bfloat16 else F32}
    return {n: (x, t + last.get(n, U) * (x.abs() + t)) for n, (x, t) in out.items()}


def check(got, want, what=""):
    """Tensors against backward()'s by name; prints the largest share of each bound that is used."""
    used = {}
    for (name, (x, t)), y in zip(want.items(), got):
        assert y.shape == x.shape and torch.isfinite(y).all(), f"{what}: {name} is not finite"
        err = (y.double() - x).abs()
        used[name] = float((err / t.clamp(min=1e-30)).max()) if err.numel() else 0.0
    print(f"[grad] {what}: " + ", ".join(f"{n} {u:.3f}" for n, u in used.items()) + " of the bounds", flush=True)
    assert len(got) == len(want) and all(u <= 1.0 for u in used.values()), (what, used)
