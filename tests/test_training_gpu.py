"""A layer's attention forward and backward through the calls as they are used together: rotary positions, packed
sequences with a relative bias, the gradients, and the positions turned back; one step after the other against the
formulas, and the whole against differentiation in 64 bits.  Far strides, and many sequences."""
import pytest
import torch

from paper_2605_31158_amd import la
import grad_reference as G
import seq_reference as R

pytestmark = pytest.mark.gpu


def turned(x, pos, freqs, sign=1):
    """x [T, H, d] in float64 turned by sign * pos, pairs (j, j + d / 2)."""
    a = pos.double()[:, None] * freqs * sign
    c, s = a.cos()[:, None], a.sin()[:, None]
    u, v = x.chunk(2, -1)
    return torch.cat([u * c - v * s, v * c + u * s], -1)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_a_layer_there_and_back(d, causal):
    lq, Hq, Hkv = [130, 1, 300, 64], 8, 2
    T = sum(lq)
    g = torch.Generator(device="cuda").manual_seed(90)
    f = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)   # noqa: E731
    q0, k0, v, do = f(T, Hq, d), f(T, Hkv, d), f(T, Hkv, d), f(T, Hq, d)
    cu = R.starts(lq)
    pos = torch.cat([torch.arange(n, dtype=torch.int32) for n in lq]).cuda()
    freqs = la.rope_frequencies(d)
    bucket, lo = la.relative_buckets(32, 128, not causal)
    bias = la.RelativeBias(torch.randn((32, Hq), generator=g, device="cuda"), bucket, lo)

    q, k = la.rope(q0, pos, freqs, k=k0)
    o, lse = la.prompt_attn(q, k, v, cu, causal=causal, want_lse=True, bias=bias)
    dq, dk, dv, dw = la.prompt_attn_bwd(do, q, k, v, o, lse, cu, causal=causal, bias=bias)
    dq0, dk0 = la.rope(dq, -pos, freqs, k=dk)

    R.check(o, lse, G.forward(q, k, v, lq, lq, causal, bias=bias), "forward")
    G.check((dq, dk, dv, dw), G.backward(do, q, k, v, o, lse, lq, lq, causal, bias=bias), "backward")
    for have, want in ((dq0, turned(dq.double(), pos, freqs, -1)), (dk0, turned(dk.double(), pos, freqs, -1))):
        # one rounding to bf16, and fp32 products of fp32 sines
        size = want.abs() + 8 * G.F32 * have.abs().amax()
        assert bool(((have.double() - want).abs() <= (G.U + 4 * G.F32) * size + 8 * G.F32 * want.abs().amax()).all())

    # the whole in 64 bits from q0, k0, v and the weights.  In 2-norms: seven roundings to bf16 lie between an input
    # and its gradient (q and k turned, o, P, dS, the gradient, the gradient turned back), each at most U of what it
    # rounds; q's and k's move a logit by U sqrt(2 / d) of its size, some 4 here, so P by less than 4 U more.
    xs = [x.double().requires_grad_() for x in (q0, k0, v)] + [bias.weight.double().requires_grad_()]
    qd, kd = turned(xs[0], pos, freqs), turned(xs[1], pos, freqs)
    total = 0.0
    a = 0
    for n in lq:
        rows = slice(a, a + n)
        a += n
        see = G.seen(n, n, causal, q.device)
        for h in range(Hq):
            x = qd[rows, h] @ kd[rows, h // 4].T * d ** -0.5
            away = torch.arange(n, device="cuda")[None] - torch.arange(n, device="cuda")[:, None]
            x = x + xs[3][:, h][bucket.long()[away.clamp(lo, lo + bucket.numel() - 1) - lo]]
            total = total + ((torch.where(see, x, -torch.inf).softmax(-1) @ xs[2][rows, h // 4]) * do[rows, h].double()).sum()
    want = torch.autograd.grad(total, xs)
    for name, x, y in zip(("dq", "dk", "dv", "dw"), (dq0, dk0, dv, dw), want):
        rel = float((x.double() - y).norm() / y.norm())
        print(f"[layer] d {d} causal {causal} {name}: {rel:.5f} of its norm", flush=True)
        assert rel <= (7 + 4) * G.U, (name, rel)


def spread(x, token):
    """x with rows `token` elements apart."""
    T, H, d = x.shape
    buf = torch.empty(T * token, dtype=x.dtype, device=x.device)
    y = buf.as_strided((T, H, d), (token, d, 1))
    y.copy_(x)
    return y


@pytest.mark.parametrize("d", [64, 128])
def test_far_strides(d):
    # rows 32 MB apart: offsets inside a tile reach 2^31, those of a tensor pass 2^32
    far = (1 << 24) - 8
    lq = [67, 70]
    T = sum(lq)
    g = torch.Generator(device="cuda").manual_seed(91)
    q, k, v, do = (torch.randn((T, h, d), generator=g, device="cuda").to(torch.bfloat16) for h in (2, 1, 1, 2))
    cu = R.starts(lq)
    o, lse = la.prompt_attn(q, k, v, cu, want_lse=True)
    want = la.prompt_attn_bwd(do, q, k, v, o, lse, cu)
    for which in range(3):
        wide = [spread(x, far) if which == n else x for n, x in ((0, q), (0, do), (1, k), (1, v), (2, o))]
        outs = tuple(spread(torch.zeros_like(x), far) if which == 2 else torch.zeros_like(x) for x in (q, k, v))
        got = la.prompt_attn_bwd(wide[1], wide[0], wide[2], wide[3], wide[4], lse, cu, out=outs)
        for x, y in zip(got, want):
            assert torch.equal(x, y), which
        del wide, outs, got
        torch.cuda.empty_cache()


def test_many_sequences():
    # 40000 sequences of none to three tokens: every gradient against a batched form of the same in 64 bits
    S, H, d = 40000, 2, 64
    g = torch.Generator().manual_seed(92)
    n = torch.randint(0, 4, (S,), generator=g)
    cu = torch.cat([torch.zeros(1, dtype=torch.int64), n.cumsum(0)]).to(torch.int32)
    T = int(cu[-1])
    gg = torch.Generator(device="cuda").manual_seed(93)
    q, k, v, do = (torch.randn((T, H, d), generator=gg, device="cuda").to(torch.bfloat16) for _ in range(4))
    cu = cu.cuda()
    o, lse = la.prompt_attn(q, k, v, cu, want_lse=True)
    dq, dk, dv = la.prompt_attn_bwd(do, q, k, v, o, lse, cu)
    for m in (1, 2, 3):
        at = cu[:-1].long().cpu()[n == m]
        rows = (at[:, None] + torch.arange(m)).cuda()                       # [sequences, m]
        x = {name: t[rows].double().transpose(1, 2) for name, t in dict(q=q, k=k, v=v, do=do, o=o).items()}
        logit = (x["q"] @ x["k"].transpose(-1, -2).contiguous()) * d ** -0.5
        see = torch.tril(torch.ones(m, m, dtype=torch.bool, device="cuda"))
        p = torch.where(see, (logit - lse[rows].double().transpose(1, 2)[..., None]).exp(), 0.0)
        dp = x["do"] @ x["v"].transpose(-1, -2).contiguous()
        ds = p * (dp - (x["do"] * x["o"]).sum(-1, keepdim=True))
        w = 1e-5 * (p * (dp.abs() + x["do"].abs().sum(-1, keepdim=True) * 5))         # fp32 sums of 64 products
        for have, want, size in ((dv, p.transpose(-1, -2) @ x["do"], p.transpose(-1, -2) @ x["do"].abs()),
                                 (dq, ds @ x["k"] * d ** -0.5, (ds.abs() + w / G.U) @ x["k"].abs() * d ** -0.5),
                                 (dk, ds.transpose(-1, -2) @ x["q"] * d ** -0.5,
                                  (ds.abs() + w / G.U).transpose(-1, -2) @ x["q"].abs() * d ** -0.5)):
            err = (have[rows].double().transpose(1, 2) - want).abs()
            assert bool((err <= G.U * (1.01 * size + want.abs() * 1.01) + 1e-6).all()), m
