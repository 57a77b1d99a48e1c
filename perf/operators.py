"""The cases that the sequence operators of `paper_2605_31158_amd.la` are measured on: rotary positions,
attention over whole prompts, and a cache of keys and values in 4 bits with the attention that reads it.

A case is a dict of plain values; `what` names the operator that one pass calls:

  rope    rope: queries and keys of one layer are rotated by their tokens' positions
  prompt  prompt_attn: packed sequences attend to their own keys, causally or not, with grouped heads
  append  kv4_append and kv4_read: new tokens enter the cache, and the values they stand for come back
  cache   kv4_attn: one or more queries of every sequence attend to the sequence's cache

Where `own` is false, `run` computes the same in elementary torch operations.
"""
import math

import torch

own = False

F480 = 30 * 52                       # tokens of a latent frame at 480P


# ------------------------------------------------------------------------------------------------
# cases

def _rope(name, T, Hq, Hk, d, rot, pairs, scaling, far, dtype, chunk=()):
    """chunk: (frames, rows, columns) of a latent grid with a position for each axis, or () for running
    positions that end before `far`."""
    rows, cols = chunk[1:] or (0, 0)
    c = dict(what="rope", T=T, Hq=Hq, Hk=Hk, d=d, rot=rot, pairs=pairs, scaling=scaling, far=far, dtype=dtype,
             rows=rows, cols=cols)
    return dict(name=name, **c) if name else c


def _prompt(name, S, lo, hi, Hq, Hk, d, causal, before=0, lse=False):
    """S sequences of lo to hi tokens (logarithmic); `before`: up to this many keys more than queries."""
    c = dict(what="prompt", S=S, lo=lo, hi=hi, Hq=Hq, Hk=Hk, d=d, causal=causal, before=before, lse=lse)
    return dict(name=name, **c) if name else c


def _append(name, S, new, before, Hk, d, page):
    c = dict(what="append", S=S, new=new, before=before, Hk=Hk, d=d, page=page)
    return dict(name=name, **c) if name else c


def _cache(name, S, lq, lo, hi, Hq, Hk, d, page, causal=True, lse=False):
    """S sequences of lo to hi cached tokens (logarithmic), lq queries each."""
    c = dict(what="cache", S=S, lq=lq, lo=lo, hi=hi, Hq=Hq, Hk=Hk, d=d, page=page, causal=causal, lse=lse)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # one token for each of 8 sequences being generated: the smallest call, latency
        _rope("rope_tokens", 8, 16, 4, 128, 128, "half", "none", 5000, "bf16"),
        # a 480P chunk of 4 frames with positions (t, y, x), neighbours paired
        _rope("rope_480p_chunk", 4 * F480, 16, 16, 128, 128, "neighbours", "none", 0, "bf16", (4, 30, 52)),
        # far positions with a stretched table, half of each head turned, fp32, an odd number of tokens
        _rope("rope_far", 8191, 16, 8, 128, 64, "half", "ramp", 1000000, "fp32"),
        # many short prompts at once, grouped heads
        _prompt("prompt_short", 48, 1, 300, 16, 4, 64, True),
        # one long prompt
        _prompt("prompt_long", 1, 8192, 8192, 16, 4, 128, True),
        # prompts of very different lengths that continue earlier text, with the log-sum-exp
        _prompt("prompt_ragged", 6, 150, 3300, 24, 8, 128, True, before=700, lse=True),
        # the next token of 64 sequences enters the cache
        _append("append_tokens", 64, 1, 4000, 8, 128, 64),
        # a 480P chunk of 4 frames enters the cache of its trajectory
        _append("append_480p_chunk", 1, 4 * F480, 8 * F480, 16, 128, 64),
        # the next token of one short sequence: the smallest attention call
        _cache("token_one", 1, 1, 1000, 1000, 16, 4, 128, 64),
        # the next token of 32 sequences between 1000 and 16000 tokens
        _cache("token_batch", 32, 1, 1000, 16000, 32, 8, 128, 64),
        # five proposed tokens of each of 8 sequences are scored at once, small pages, 64-wide heads
        _cache("tokens_scored", 8, 5, 700, 9000, 32, 4, 64, 16, lse=True),
        # a 480P chunk attends to the 8 frames before it, held in 4 bits; its own keys come from elsewhere
        _cache("chunk_480p", 1, 4 * F480, 8 * F480, 8 * F480, 16, 16, 128, 64, causal=False, lse=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: no larger than the largest listed one of its operator."""
    what = rng.choice(["rope", "prompt", "prompt", "append", "cache", "cache", "cache"])
    d = rng.choice([64, 128, 128])
    Hk = rng.choice([1, 2, 3, 4, 8, 16])
    G = rng.choice([1, 1, 2, 3, 4, 5, 8, 16])
    while G * Hk > 32:
        G, Hk = max(1, G // 2), max(1, Hk - 1)
    if what == "rope":
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        pairs = rng.choice(["half", "neighbours"])
        if rng.random() < 0.3:
            grid = [rng.randint(1, 5), _log(rng, 6, 30), _log(rng, 6, 52)]
            return _rope("", math.prod(grid), G * Hk, Hk, d, d, pairs, "none", 0, dtype, grid)
        T = _log(rng, 1, 8191)
        rot = rng.choice([d, d, d // 2, 32])
        return _rope("", T, G * Hk, Hk, d, rot, pairs, rng.choice(["none", "linear", "ramp"]),
                     T + _log(rng, 1, 1000000), dtype)
    if what == "prompt":
        hi = _log(rng, 8, 4500)
        S = max(1, min(_log(rng, 1, 64), 9000 // hi))
        c = _prompt("", S, max(1, _log(rng, 1, hi)), hi, G * Hk, Hk, d, rng.random() < 0.8,
                    before=rng.choice([0, 0, _log(rng, 1, 900)]), lse=rng.random() < 0.4)
        return c
    page = rng.choice([16, 32, 64, 128])
    if what == "append":
        S = _log(rng, 1, 64)
        new = 1 if rng.random() < 0.5 else _log(rng, 2, max(2, 6000 // S))
        return _append("", S, new, _log(rng, 1, 12000), Hk, d, page)
    if rng.random() < 0.25:                                             # whole chunks
        lq, S = _log(rng, 70, 6000), 1
        hi = lq + _log(rng, 64, 12000)
        while G * Hk > 16:
            G, Hk = max(1, G // 2), max(1, Hk - 1)
        return _cache("", S, lq, hi, hi, G * Hk, Hk, d, page, causal=rng.random() < 0.5, lse=rng.random() < 0.5)
    lq = rng.choice([1, 1, 1, rng.randint(2, 9), _log(rng, 10, 64)])
    S = _log(rng, 1, 32)
    hi = _log(rng, 64, 16000)
    return _cache("", S, lq, max(1, _log(rng, 1, hi)), hi, G * Hk, Hk, d, page, causal=rng.random() < 0.8,
                  lse=rng.random() < 0.4)


def _lengths(S, lo, hi):
    """S lengths from lo to hi, spread over the logarithm."""
    g = torch.Generator().manual_seed(77)
    at = (torch.arange(S, dtype=torch.float64) + torch.rand(S, generator=g, dtype=torch.float64)) / S
    return torch.exp(math.log(lo) + at * (math.log(hi) - math.log(lo))).round().to(torch.int64).clamp(lo, hi)


def _shape(c, seed=0):
    """(queries, keys) of each sequence: the case's lengths, in an order that the seed gives."""
    S, g = c["S"], torch.Generator().manual_seed(78)
    if c["what"] == "prompt":
        lq = _lengths(S, c["lo"], c["hi"])
        lk = lq + torch.randint(0, c["before"] + 1, (S,), generator=g)
    elif c["what"] == "append":
        lq = _lengths(S, (c["new"] + 1) // 2, c["new"])
        lk = lq + torch.randint(c["before"] // 2, c["before"] + 1, (S,), generator=g)
    else:
        lq, lk = torch.full((S,), c["lq"], dtype=torch.int64), _lengths(S, c["lo"], c["hi"])
    order = torch.randperm(S, generator=torch.Generator().manual_seed(seed))
    return lq[order], lk[order]


def _pairs_seen(lq, lk, causal):
    if not causal:
        return float((lq * lk).sum())
    # query i sees the keys up to i + lk - lq
    first = (lk - lq).clamp(min=0) + 1
    rows = torch.minimum(lq, lk)
    return float(((first + lk) * rows).sum()) / 2


def work(c):
    if c["what"] == "rope":
        size = 2 if c["dtype"] == "bf16" else 4
        n = c["T"] * (c["Hq"] + c["Hk"])
        axes = 3 if c["rows"] else 1
        return {"bytes": 2 * n * c["d"] * size + 4 * axes * c["T"] + 4 * c["rot"], "flops": 3.0 * n * c["rot"]}
    lq, lk = _shape(c)
    d, Hk = c["d"], c["Hk"]
    if c["what"] == "append":
        values = 2 * float(lq.sum()) * Hk * d
        return {"bytes": values * (2 + 2 + 2 * 17 / 32), "flops": 4 * values}
    flops = 4.0 * d * c["Hq"] * _pairs_seen(lq, lk, c["causal"])
    rows = float(lq.sum()) * c["Hq"]
    out = rows * (4 * d + (4 if c["lse"] else 0))
    if c["what"] == "prompt":
        return {"bytes": out + 4 * d * float(lk.sum()) * Hk, "flops": flops}
    return {"bytes": out + 2 * d * 17 / 32 * float(lk.sum()) * Hk + 4 * float(lk.sum()) / c["page"], "flops": flops}


# ------------------------------------------------------------------------------------------------
# inputs

def _starts(n):
    return torch.cat([torch.zeros(1, dtype=torch.int64), n.cumsum(0)]).to(torch.int32)


def _normal(shape, g, dtype=torch.bfloat16, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _frequencies(c):
    """Radians that a pair turns by for each position, in 64 bits: base 10000, a ladder of its own for every axis."""
    half = c["rot"] // 2
    if c["rows"]:
        n = _axis_pairs(half)
        return torch.cat([10000.0 ** (-torch.arange(m, dtype=torch.float64) / m) for m in n])
    f = 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
    if c["scaling"] == "linear":
        return f / 8.0
    if c["scaling"] == "ramp":                        # 1 to 32 turns over the 32768 trained positions, 32 times as long
        keep = ((32768.0 * f / (2 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
        return f * (keep + (1.0 - keep) / 32.0)
    return f


def _axis_pairs(half):
    side = half // 3
    return [half - 2 * side, side, side]


# codes of e2m1 in order: 0, 0.5, 1, 1.5, 2, 3, 4, 6
_MIDDLES = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]


def _quantise(x):
    """x [.., d] in bf16 -> (codes 0..15, scale bytes [.., d / 32]): per 32 values the smallest power of two,
    2^(byte - 127), under which the largest is rounded by no more than half a step."""
    x = x.float().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1)
    e = torch.frexp(top).exponent - 3                 # 4 <= top / 2^e < 8
    e = torch.where(top >= 7.0 * torch.ldexp(torch.ones_like(top), e), e + 1, e)
    byte = torch.where(top > 0, e + 127, torch.zeros_like(e)).clamp(2, 252)
    y = torch.ldexp(x, (127 - byte).unsqueeze(-1))
    mag = y.abs()
    code = torch.zeros_like(x, dtype=torch.uint8)
    for n, m in enumerate(_MIDDLES):                  # a value in the middle goes to the even code
        code += (mag > m) if n % 2 == 0 else (mag >= m)
    code |= torch.signbit(y).to(torch.uint8) << 3
    return code.flatten(-2), byte.to(torch.uint8)


def _values(code, byte):
    """What codes and scale bytes stand for, in fp32."""
    step = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=code.device)
    v = step[(code & 7).long()]
    v = torch.where(code > 7, -v, v).unflatten(-1, (-1, 32))
    return torch.ldexp(v, (byte.int() - 127).unsqueeze(-1)).flatten(-2)


def _pack(kc, ks, vc, vs):
    """Pages [n, P, H, ..] of codes and scale bytes -> the cache's bytes [n, H, P (d + d / 16)]: K codes row by
    row, K scales by 32-value block, V codes in quads of 4 tokens (a chunk of d / 16 values of each in turn), V scales."""
    n, P, H, d = kc.shape
    kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)                          # [n, H, P, d]
    ks, vs = ks.permute(0, 2, 3, 1), vs.permute(0, 2, 3, 1)                  # [n, H, d / 32, P]
    two = lambda x: x[..., 0::2] | (x[..., 1::2] << 4)                       # noqa: E731
    quads = two(vc).reshape(n, H, P // 4, 4, 16, d // 32).transpose(3, 4)
    return torch.cat([x.reshape(n, H, -1) for x in (two(kc), ks, quads, vs)], dim=-1).contiguous()


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"c": c}
    if c["what"] == "rope":
        dtype = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
        s["q"] = _normal((c["T"], c["Hq"], c["d"]), g, dtype)
        s["k"] = _normal((c["T"], c["Hk"], c["d"]), g, dtype)
        s["freqs"] = _frequencies(c).cuda()
        t = torch.arange(c["T"])
        if c["rows"]:
            first = torch.randint(0, 200, (1,), generator=g, device="cuda").cpu()
            rows, cols = c["rows"], c["cols"]
            s["positions"] = torch.stack([first + t // (rows * cols), t // cols % rows, t % cols]).to(torch.int32).cuda()
            s["sections"] = tuple(_axis_pairs(c["rot"] // 2))
        else:
            first = torch.randint(0, max(1, c["far"] - c["T"]), (1,), generator=g, device="cuda").cpu()
            s["positions"], s["sections"] = (first + t).to(torch.int32).cuda(), None
        return s
    lq, lk = _shape(c, seed)
    s["cu_q"], s["max_q"] = _starts(lq).cuda(), int(lq.max())
    T, d, Hk = int(lq.sum()), c["d"], c["Hk"]
    if c["what"] == "prompt":
        s["cu_k"] = _starts(lk).cuda()
        s["q"] = _normal((T, c["Hq"], d), g, scale=1.5)
        s["k"], s["v"] = (_normal((int(lk.sum()), Hk, d), g) for _ in range(2))
        return s
    # a pool of pages, handed out in random order
    P = c["page"]
    need = (lk + P - 1) // P
    n = int(need.sum()) + 3
    order = torch.randperm(n, generator=g, device="cuda").to(torch.int32).cpu()
    at = _starts(need)
    table = torch.zeros((c["S"], int(need.max())), dtype=torch.int32)
    for i in range(c["S"]):
        table[i, : int(need[i])] = order[at[i]: at[i + 1]]
    s["table"], s["lens"] = table.cuda(), lk.to(torch.int32).cuda()
    if c["what"] == "append":
        s["k"], s["v"] = (_normal((T, Hk, d), g) for _ in range(2))
        s["cache"] = torch.zeros((n, Hk, P * (d + d // 16)), dtype=torch.uint8, device="cuda")
        return s
    s["q"] = _normal((T, c["Hq"], d), g, scale=1.5)
    kc, ks = _quantise(_normal((n, P, Hk, d), g))
    vc, vs = _quantise(_normal((n, P, Hk, d), g))
    s["cache"] = _pack(kc, ks, vc, vs)
    return s


# ------------------------------------------------------------------------------------------------
# one pass

def _turn(x, cos, sin, half_pairs):
    r = cos.shape[-1]
    y = x.float()
    if half_pairs:
        a, b, rest = y[..., :r], y[..., r: 2 * r], y[..., 2 * r:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1).to(x.dtype)
    a, b, rest = y[..., 0: 2 * r: 2], y[..., 1: 2 * r: 2], y[..., 2 * r:]
    both = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([both, rest], -1).to(x.dtype)


def _plain_rope(s):
    c, p = s["c"], s["positions"].double()
    if s["sections"] is None:
        angle = p[:, None] * s["freqs"]
    else:
        n = torch.tensor(s["sections"], device="cuda")
        angle = p.repeat_interleave(n, dim=0).T * s["freqs"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    return [_turn(s["q"], cos, sin, c["pairs"] == "half"), _turn(s["k"], cos, sin, c["pairs"] == "half")]


def _softmax_product(score, seen, v):
    """(o, log-sum-exp) of scores where `seen`; rows that see nothing give 0 and -inf."""
    score = score.masked_fill(~seen, -torch.inf)
    top = score.amax(-1, keepdim=True)
    p = (score - top.masked_fill(top == -torch.inf, 0.0)).exp()
    total = p.sum(-1, keepdim=True)
    o = (p @ v) / total.masked_fill(total == 0.0, 1.0)
    return o, (top + total.log()).squeeze(-1)


def _plain_prompt(s):
    c, (Tq, Hq, d), Hk = s["c"], s["q"].shape, s["c"]["Hk"]
    q = s["q"].float().reshape(Tq, Hk, Hq // Hk, d).permute(1, 2, 0, 3)
    k, v = (x.float().permute(1, 0, 2)[:, None] for x in (s["k"], s["v"]))
    cq, ck = s["cu_q"].long(), s["cu_k"].long()
    tq, tk = torch.arange(Tq, device="cuda"), torch.arange(k.shape[2], device="cuda")
    iq, ik = (torch.bucketize(t, cu[1:], right=True) for t, cu in ((tq, cq), (tk, ck)))
    seen = iq[:, None] == ik[None]
    if c["causal"]:                                    # the last query sees the last key
        seen &= (tk - ck[1:][ik])[None] <= (tq - cq[1:][iq])[:, None]
    o, lse = _softmax_product(q @ k.transpose(-1, -2).contiguous() * d ** -0.5, seen, v)
    o = o.permute(2, 0, 1, 3).reshape(Tq, Hq, d).to(torch.bfloat16)
    return [o, lse.permute(2, 0, 1).reshape(Tq, Hq).contiguous()] if c["lse"] else [o]


def _plain_append(s):
    out = []
    for x in (s["k"], s["v"]):
        out.append(_values(*_quantise(x)).to(torch.bfloat16))
    return out


def _unpack(pages, P, d):
    """The cache's bytes [.., P (d + d / 16)] -> K and V [.., P, d] in fp32."""
    a, b = P * d // 2, P * d // 32
    kc, ks, vc, vs = pages.split([a, b, a, b], dim=-1)
    kc = kc.unflatten(-1, (P, d // 2))
    vc = vc.unflatten(-1, (P // 4, 16, 4, d // 32)).transpose(-3, -2).flatten(-2).flatten(-3, -2)
    both = lambda x: torch.stack([x & 15, x >> 4], -1).flatten(-2)           # noqa: E731
    scale = lambda x: x.unflatten(-1, (d // 32, P)).transpose(-1, -2)        # noqa: E731
    return _values(both(kc), scale(ks)), _values(both(vc), scale(vs))


def _plain_cache(s):
    c, (T, Hq, d), Hk, S, P = s["c"], s["q"].shape, s["c"]["Hk"], s["c"]["S"], s["c"]["page"]
    k, v = _unpack(s["cache"][s["table"].long()], P, d)                      # [S, pages, Hk, P, d]
    k, v = (x.transpose(1, 2).flatten(2, 3) for x in (k, v))                 # [S, Hk, keys, d]
    q = s["q"].float().reshape(S, c["lq"], Hk, Hq // Hk, d).permute(0, 2, 3, 1, 4).flatten(2, 3)
    tk, lens = torch.arange(k.shape[2], device="cuda"), s["lens"].long()[:, None, None]
    last = lens - 1
    if c["causal"]:
        last = last - (c["lq"] - 1) + torch.arange(c["lq"], device="cuda")[:, None]
    seen = (tk <= last).expand(S, c["lq"], -1).repeat(1, Hq // Hk, 1)[:, None]
    o, lse = _softmax_product(q @ k.transpose(-1, -2).contiguous() * d ** -0.5, seen, v)
    o = o.unflatten(2, (Hq // Hk, c["lq"])).permute(0, 3, 1, 2, 4).reshape(T, Hq, d).to(torch.bfloat16)
    return [o, lse.unflatten(2, (Hq // Hk, c["lq"])).permute(0, 3, 1, 2).reshape(T, Hq)] if c["lse"] else [o]


def _own(s):
    from paper_2605_31158_amd import la
    c = s["c"]
    if c["what"] == "rope":
        return list(la.rope(s["q"], s["positions"], s["freqs"], k=s["k"], interleaved=c["pairs"] == "neighbours",
                            sections=s["sections"]))
    if c["what"] == "append":
        la.kv4_append(s["cache"], s["k"], s["v"], s["cu_q"], s["lens"], s["table"])
        return list(la.kv4_read(s["cache"], s["cu_q"], s["lens"], s["table"], s["k"].shape[0], c["d"]))
    if c["what"] == "prompt":
        o = la.prompt_attn(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], causal=c["causal"], want_lse=c["lse"])
    else:
        o = la.kv4_attn(s["q"], s["cache"], s["cu_q"], s["lens"], s["table"], s["max_q"], causal=c["causal"],
                        want_lse=c["lse"])
    return list(o) if c["lse"] else [o]


def run(s):
    if own:
        return _own(s)
    what = s["c"]["what"]
    if what == "rope":
        return _plain_rope(s)
    if what == "prompt":
        return _plain_prompt(s)
    if what == "append":
        return _plain_append(s)
    return _plain_cache(s)


# ------------------------------------------------------------------------------------------------
# the definitions in 64 bits

def _exact_rope(s):
    c = s["c"]
    f, p = s["freqs"].cpu(), s["positions"].cpu().double()
    axis = torch.zeros(len(f), dtype=torch.long)
    if s["sections"] is not None:
        axis = torch.cat([torch.full((n,), a) for a, n in enumerate(s["sections"])])
    p = p.reshape(-1, p.shape[-1])
    turn = torch.exp(1j * torch.stack([p[axis[j]] * f[j] for j in range(len(f))], -1)).cuda()[:, None]
    out = []
    for x in (s["q"].double(), s["k"].double()):
        i = torch.arange(len(f), device="cuda")
        at, to = (i, i + len(f)) if c["pairs"] == "half" else (2 * i, 2 * i + 1)
        z = torch.complex(x[..., at], x[..., to]) * turn
        y = x.clone()
        y[..., at], y[..., to] = z.real, z.imag
        out.append(y)
    return out


def _exact_rows(q, k, v, seen):
    """Attention of q [n, d] to k, v [m, d]; seen[i] keys at the front of k are visible to row i."""
    t = (q @ k.T) / math.sqrt(q.shape[-1])
    t = torch.where(torch.arange(len(k), device=t.device)[None] < seen[:, None], t, -math.inf)
    lse = torch.logsumexp(t, -1)
    w = torch.exp(t - torch.where(torch.isinf(lse), 0.0, lse)[:, None])
    return w @ v, lse


def _exact_attention(s, keys):
    """keys(i, h) gives K and V of sequence i and key head h in 64 bits."""
    c, cu = s["c"], s["cu_q"].tolist()
    q = s["q"].double()
    G = c["Hq"] // c["Hk"]
    o, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda")
    for i in range(len(cu) - 1):
        n = cu[i + 1] - cu[i]
        for h in range(c["Hk"]):
            k, v = keys(i, h)
            seen = torch.full((n,), len(k), device="cuda")
            if c["causal"]:
                seen = (len(k) - n + 1 + torch.arange(n, device="cuda")).clamp(min=0)
            for j in range(h * G, h * G + G):
                o[cu[i]: cu[i + 1], j], lse[cu[i]: cu[i + 1], j] = _exact_rows(q[cu[i]: cu[i + 1], j], k, v, seen)
    return [o, lse] if c["lse"] else [o]


def _nibbles(row):
    """A cache row's bytes -> its e2m1 values: sign, two exponent bits, one bit of mantissa."""
    code = torch.stack([row % 16, row // 16], -1).flatten(-2).double()
    sign = 1.0 - 2.0 * (code >= 8).double()
    e, m = (code % 8 / 2).floor(), code % 2
    return sign * torch.where(e == 0, m * 0.5, (1.0 + m * 0.5) * 2.0 ** (e - 1))


def exact(c, seed):
    s = prepare(c, seed)
    if c["what"] == "rope":
        return _exact_rope(s)
    if c["what"] == "prompt":
        ck = s["cu_k"].tolist()
        return _exact_attention(s, lambda i, h: (s["k"][ck[i]: ck[i + 1], h].double(), s["v"][ck[i]: ck[i + 1], h].double()))
    if c["what"] == "append":
        out = []
        grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device="cuda")
        for x in (s["k"].double(), s["v"].double()):
            b = x.unflatten(-1, (-1, 32))
            top = b.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -130)
            unit = 2.0 ** torch.ceil(torch.log2(top / 7.0))                   # top / unit in (3.5, 7]
            unit = torch.where(top == 7.0 * unit, 2.0 * unit, unit)
            unit = unit.clamp(2.0 ** -125, 2.0 ** 125)
            far = (b.abs() / unit)[..., None] - grid
            even = torch.tensor([0, 1, 0, 1, 0, 1, 0, 1], device="cuda") * 1e-9   # the even code wins a tie
            pick = (far.abs() + even).argmin(-1)
            out.append((torch.sign(b) * grid[pick] * unit).flatten(-2))
        return out
    P, d = c["page"], c["d"]
    lens, table, raw = s["lens"].tolist(), s["table"].long(), s["cache"]
    a, b = P * d // 2, P * d // 32

    def keys(i, h):
        t = torch.arange(lens[i], device="cuda")
        page, at = raw[table[i][t // P], h], (t % P)[:, None]
        kb = torch.arange(d // 2, device="cuda")[None] + at * (d // 2)
        # V: quad of 4 tokens, chunk of d / 32 bytes, token inside the quad, byte of the chunk
        n = torch.arange(d // 2, device="cuda")[None]
        w = d // 32
        vb = a + b + (at // 4) * (2 * d) + (n // w) * (4 * w) + (at % 4) * w + n % w
        sb = torch.arange(d // 32, device="cuda")[None] * P + at
        unit = lambda o: 2.0 ** (page.gather(1, sb + o).double() - 127).repeat_interleave(32, 1)   # noqa: E731
        return _nibbles(page.gather(1, kb)) * unit(a), _nibbles(page.gather(1, vb)) * unit(2 * a + b)

    return _exact_attention(s, keys)
