"""The cases that the training side of the packed sequences of `paper_2605_31158_amd.la` is measured on: attention
with a learned bias by relative position, and attention's gradients without and with that bias.

A case is a dict of plain values; `what` names the operator that one pass calls:

  bias       prompt_attn with bias: every bucket of distances has a learned number for each head
  back       prompt_attn_bwd: the gradients of q, k and v, from the forward's o and log-sum-exp
  back_bias  prompt_attn_bwd with bias: the same, and the gradient of the bias' weights

Where `own` is false, `run` computes the same in elementary torch operations.
"""
import math

import torch

own = False

F480 = 30 * 52                       # tokens of a latent frame at 480P


# ------------------------------------------------------------------------------------------------
# cases

def _case(name, what, S, lo, hi, Hq, Hk, d, causal, before=0, lse=False, buckets=0, reach=0, both=False, wtype=""):
    """S sequences of lo to hi queries (logarithmic) with before / 2 to `before` keys more than queries.  The bias
    has `buckets` buckets, distances from `reach` on share the last one; both: keys behind a query have their own."""
    c = dict(what=what, S=S, lo=lo, hi=hi, Hq=Hq, Hk=Hk, d=d, causal=causal, before=before, lse=lse, buckets=buckets,
             reach=reach, both=both, wtype=wtype)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # the next token of 8 sequences being generated, one-sided bias: the smallest call, latency
        _case("bias_tokens", "bias", 8, 1, 1, 16, 16, 64, True, before=1000, buckets=32, reach=128, wtype="bf16"),
        # a batch of prompts in a text encoder: both directions, the log-sum-exp for the backward pass
        _case("bias_text", "bias", 16, 60, 512, 16, 16, 64, False, lse=True, buckets=32, reach=128, both=True,
              wtype="bf16"),
        # one long causal text, grouped heads
        _case("bias_long", "bias", 1, 8192, 8192, 16, 4, 128, True, buckets=32, reach=128, wtype="fp32"),
        # one short prompt: the smallest backward call
        _case("back_one", "back", 1, 77, 77, 16, 16, 64, True),
        # many short prompts at once, grouped heads
        _case("back_short", "back", 48, 1, 300, 16, 4, 64, True),
        # one long prompt
        _case("back_long", "back", 1, 8192, 8192, 16, 4, 128, True),
        # prompts of very different lengths that continue earlier text
        _case("back_ragged", "back", 6, 150, 3300, 24, 8, 128, True, before=700),
        # a 480P chunk of 4 frames against itself and the frames before it
        _case("back_480p_chunk", "back", 1, 4 * F480, 4 * F480, 16, 16, 128, False, before=4 * F480),
        # the text encoder's batch, trained
        _case("back_bias_text", "back_bias", 16, 60, 512, 16, 16, 64, False, buckets=32, reach=128, both=True,
              wtype="bf16"),
        # two long causal texts, the weights' gradient in fp32
        _case("back_bias_long", "back_bias", 2, 4096, 4096, 16, 16, 128, True, buckets=32, reach=128, wtype="fp32"),
        # ragged texts with earlier keys, grouped heads, a bias of few buckets that looks to both sides
        _case("back_bias_ragged", "back_bias", 5, 100, 2100, 12, 4, 64, False, before=300, buckets=20, reach=250,
              both=True, wtype="fp32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: no larger than the largest listed one of its operator."""
    what = rng.choice(["bias", "bias", "back", "back", "back_bias"])
    d = rng.choice([64, 128])
    Hk = rng.choice([1, 2, 3, 4, 8, 16])
    G = rng.choice([1, 1, 1, 2, 3, 4, 5, 8])
    while G * Hk > 16:
        G, Hk = max(1, G // 2), max(1, Hk - 1)
    b = {}
    if what != "back":
        both = rng.random() < 0.5
        b = dict(buckets=rng.choice([8, 20, 32, 64]), reach=_log(rng, 34, 256), both=both, wtype=rng.choice(["bf16", "fp32"]))
    causal = rng.random() < 0.6
    if what == "bias" and rng.random() < 0.3:                           # single tokens
        return _case("", what, _log(rng, 1, 64), 1, 1, G * Hk, Hk, d, True, before=_log(rng, 1, 2000),
                     lse=rng.random() < 0.5, **b)
    hi = _log(rng, 8, 4500 if causal else 3200)
    S = max(1, min(_log(rng, 1, 64), 7000 // hi))
    return _case("", what, S, max(1, _log(rng, 1, hi)), hi, G * Hk, Hk, d, causal,
                 before=rng.choice([0, 0, _log(rng, 1, 900)]), lse=what == "bias" and rng.random() < 0.5, **b)


def _lengths(S, lo, hi):
    """S lengths from lo to hi, spread over the logarithm."""
    g = torch.Generator().manual_seed(77)
    at = (torch.arange(S, dtype=torch.float64) + torch.rand(S, generator=g, dtype=torch.float64)) / S
    return torch.exp(math.log(lo) + at * (math.log(hi) - math.log(lo))).round().to(torch.int64).clamp(lo, hi)


def _shape(c, seed=0):
    """(queries, keys) of each sequence: the case's lengths, in an order that the seed gives."""
    S = c["S"]
    lq = _lengths(S, c["lo"], c["hi"])
    lk = lq + torch.randint(c["before"] // 2, c["before"] + 1, (S,), generator=torch.Generator().manual_seed(78))
    order = torch.randperm(S, generator=torch.Generator().manual_seed(seed))
    return lq[order], lk[order]


def work(c):
    lq, lk = _shape(c)
    d, Hq, Hk = c["d"], c["Hq"], c["Hk"]
    # query i sees the keys up to i + lk - lq
    pairs = float((lq * (2 * lk - lq + 1)).sum()) / 2 if c["causal"] else float((lq * lk).sum())
    q, kv, stat = 2 * d * float(lq.sum()) * Hq, 2 * d * float(lk.sum()) * Hk, 4 * float(lq.sum()) * Hq
    bias = c["buckets"] * Hq * (2 if c["wtype"] == "bf16" else 4) + 4 * (2 if c["both"] else 1) * c["reach"]
    if c["what"] == "bias":
        return {"bytes": 2 * q + 2 * kv + (stat if c["lse"] else 0) + bias, "flops": 4.0 * d * Hq * pairs}
    # q, o, do, k, v, the log-sum-exp; dq, dk, dv
    return {"bytes": 4 * q + 4 * kv + stat + 2 * bias, "flops": 10.0 * d * Hq * pairs}


# ------------------------------------------------------------------------------------------------
# inputs

def _starts(n):
    return torch.cat([torch.zeros(1, dtype=torch.int64), n.cumsum(0)]).to(torch.int32)


def _normal(shape, g, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(torch.bfloat16)


def _buckets(c):
    """(bucket of every distance key - query from `lo` on, lo): half of a side's buckets hold one distance each, the
    others ever more, on a logarithm that ends at `reach`."""
    n = c["buckets"] // 2 if c["both"] else c["buckets"]
    one = n // 2

    def side(m):
        if m < one:
            return m
        return min(n - 1, one + int(math.log(m / one) / math.log(c["reach"] / one) * (n - one) + 1e-9))

    lo, hi = -c["reach"], c["reach"] if c["both"] else 0
    return [side(abs(x)) + (n if x > 0 else 0) for x in range(lo, hi + 1)], lo


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    lq, lk = _shape(c, seed)
    d, Hq, Hk = c["d"], c["Hq"], c["Hk"]
    s = {"c": c, "lq": lq.tolist(), "lk": lk.tolist(), "cu_q": _starts(lq).cuda(), "cu_k": _starts(lk).cuda()}
    s["q"] = _normal((int(lq.sum()), Hq, d), g, 1.5)
    s["k"], s["v"] = (_normal((int(lk.sum()), Hk, d), g) for _ in range(2))
    if c["what"] != "back":
        to, s["lo"] = _buckets(c)
        s["bucket"] = torch.tensor(to, dtype=torch.int32, device="cuda")
        s["weight"] = torch.randn((c["buckets"], Hq), generator=g, device="cuda")
        if c["wtype"] == "bf16":
            s["weight"] = s["weight"].to(torch.bfloat16)
    if c["what"] != "bias":
        # what the forward pass left
        s["o"], s["lse"] = _plain_forward(s)
        s["do"] = _normal(s["q"].shape, g)
    return s


# ------------------------------------------------------------------------------------------------
# one pass

def _sequences(s):
    """(rows of q, rows of k, queries, keys) of each sequence."""
    a = b = 0
    for n, m in zip(s["lq"], s["lk"]):
        yield slice(a, a + n), slice(b, b + m), n, m
        a, b = a + n, b + m


def _logits(s, q, k, n, m):
    """Logits [Hk, G, n, m] of q [Hk, G, n, d] over k [Hk, 1, m, d], -inf where a query does not see."""
    c = s["c"]
    x = q @ k.transpose(-1, -2).contiguous() * c["d"] ** -0.5
    away = torch.arange(m, device="cuda") - torch.arange(m - n, m, device="cuda")[:, None]
    if "weight" in s:
        at = s["bucket"].long()[away.clamp(s["lo"], s["lo"] + len(s["bucket"]) - 1) - s["lo"]]
        x += s["weight"].float().T[:, at].unflatten(0, (c["Hk"], -1))
    return x.masked_fill(away > 0, -torch.inf) if c["causal"] else x


def _heads(x, Hk):
    """Rows [n, H, d] as [Hk, H / Hk, n, d] in 32 bits."""
    return x.float().unflatten(1, (Hk, -1)).permute(1, 2, 0, 3).contiguous()


def _rows(x):
    return x.permute(2, 0, 1, 3).flatten(1, 2)


def _plain_forward(s):
    Hk = s["c"]["Hk"]
    o, lse = [], []
    for rq, rk, n, m in _sequences(s):
        k, v = _heads(s["k"][rk], Hk), _heads(s["v"][rk], Hk)
        x = _logits(s, _heads(s["q"][rq], Hk), k, n, m)
        top = x.amax(-1, keepdim=True)
        p = (x - top).exp()
        total = p.sum(-1, keepdim=True)
        o.append(_rows((p @ v) / total))
        lse.append(_rows(top + total.log()).squeeze(-1))
    return torch.cat(o).to(torch.bfloat16), torch.cat(lse)


def _along_diagonals(x, n, m):
    """Sums of x [H, n, m] over the pairs at each distance key - query, from 1 - n to m - 1, in 64 bits."""
    x = torch.nn.functional.pad(x.flip(1), (0, n)).flatten(1)
    return x[:, : n * (n + m - 1)].unflatten(1, (n, n + m - 1)).sum(1, dtype=torch.float64)


def _plain_back(s):
    c, Hk = s["c"], s["c"]["Hk"]
    scale = c["d"] ** -0.5
    dq, dk, dv = [], [], []
    if "weight" in s:
        dw = torch.zeros(c["Hq"], c["buckets"], dtype=torch.float64, device="cuda")
    for rq, rk, n, m in _sequences(s):
        q, do, k, v = _heads(s["q"][rq], Hk), _heads(s["do"][rq], Hk), _heads(s["k"][rk], Hk), _heads(s["v"][rk], Hk)
        delta = (do * _heads(s["o"][rq], Hk)).sum(-1, keepdim=True)
        p = (_logits(s, q, k, n, m) - _heads(s["lse"][rq][..., None], Hk)).exp()
        ds = do @ v.transpose(-1, -2).contiguous()
        ds = (ds - delta) * p
        dq.append(_rows(ds @ k * scale))
        dk.append((ds.transpose(-1, -2).contiguous() @ q).sum(1, keepdim=True) * scale)
        dv.append((p.transpose(-1, -2).contiguous() @ do).sum(1, keepdim=True))
        dk[-1], dv[-1] = _rows(dk[-1]), _rows(dv[-1])
        if "weight" in s:
            away = torch.arange(1 - n, m, device="cuda") - (m - n)
            at = s["bucket"].long()[away.clamp(s["lo"], s["lo"] + len(s["bucket"]) - 1) - s["lo"]]
            dw.index_add_(1, at, _along_diagonals(ds.flatten(0, 1), n, m))
    out = [torch.cat(x).to(torch.bfloat16) for x in (dq, dk, dv)]
    return out + [dw.T.to(s["weight"].dtype).contiguous()] if "weight" in s else out


def _own(s):
    from paper_2605_31158_amd import la
    c = s["c"]
    bias = la.RelativeBias(s["weight"], s["bucket"], s["lo"]) if "weight" in s else None
    if c["what"] == "bias":
        o = la.prompt_attn(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], causal=c["causal"], want_lse=c["lse"], bias=bias)
        return list(o) if c["lse"] else [o]
    return list(la.prompt_attn_bwd(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["cu_q"], s["cu_k"],
                                   causal=c["causal"], bias=bias))


def run(s):
    if own:
        return _own(s)
    if s["c"]["what"] == "bias":
        o, lse = _plain_forward(s)
        return [o, lse] if s["c"]["lse"] else [o]
    return _plain_back(s)


# ------------------------------------------------------------------------------------------------
# the definitions in 64 bits, head by head

def exact(c, seed):
    s = prepare(c, seed)
    G, d = c["Hq"] // c["Hk"], c["d"]
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    back = c["what"] != "bias"
    if back:
        do, o, lse = s["do"].double(), s["o"].double(), s["lse"].double()
        dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    else:
        o, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda")
    if "weight" in s:
        w, to = s["weight"].double(), s["bucket"].tolist()
        dw = torch.zeros_like(w)
    q0 = k0 = 0
    for n, m in zip(s["lq"], s["lk"]):
        # key j is `gap` away from the place of query i among the keys
        gap = torch.arange(m, device="cuda")[None] - (torch.arange(n, device="cuda")[:, None] + (m - n))
        hidden = gap > 0 if c["causal"] else torch.zeros_like(gap, dtype=torch.bool)
        if "weight" in s:
            which = torch.tensor(to, device="cuda")[torch.clamp(gap - s["lo"], 0, len(to) - 1)]
        for h in range(c["Hq"]):
            qh, kh, vh = q[q0: q0 + n, h], k[k0: k0 + m, h // G], v[k0: k0 + m, h // G]
            t = torch.einsum("id,jd->ij", qh, kh) / math.sqrt(d)
            if "weight" in s:
                t = t + w[:, h][which]
            t[hidden] = -math.inf
            if not back:
                lse[q0: q0 + n, h] = torch.logsumexp(t, 1)
                o[q0: q0 + n, h] = torch.softmax(t, 1) @ vh
                continue
            doh = do[q0: q0 + n, h]
            p = torch.exp(t - lse[q0: q0 + n, h, None])
            dv[k0: k0 + m, h // G] += torch.einsum("ij,id->jd", p, doh)
            ds = p * (torch.einsum("id,jd->ij", doh, vh) - torch.einsum("id,id->i", doh, o[q0: q0 + n, h])[:, None])
            dq[q0: q0 + n, h] = torch.einsum("ij,jd->id", ds, kh) / math.sqrt(d)
            dk[k0: k0 + m, h // G] += torch.einsum("ij,id->jd", ds, qh) / math.sqrt(d)
            if "weight" in s:
                for b in range(c["buckets"]):
                    dw[b, h] += ds[which == b].sum()
        q0, k0 = q0 + n, k0 + m
    if not back:
        return [o, lse] if c["lse"] else [o]
    return [dq, dk, dv, dw] if "weight" in s else [dq, dk, dv]
