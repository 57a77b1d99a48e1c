"""The sequence operators as a serving loop uses them: prompts are turned by their positions, attend to
themselves and enter the 4-bit cache; then tokens come one by one (or a few proposed at once), each turned,
entered and attending to the cache, eagerly and as one captured graph."""
import pytest
import torch

from paper_2605_31158_amd import la
import seq_reference as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,page,G", [(128, 64, 4), (64, 16, 3)])
def test_prompts_then_tokens(d, page, G):
    Hk, lens = 2, [37, 1, 300, 129]
    S, Hq = len(lens), 2 * G
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda n, h: torch.randn((n, h, d), generator=g, device="cuda").to(torch.bfloat16)      # noqa: E731
    freqs = la.rope_frequencies(d)
    room = [n + 24 for n in lens]
    pages = [-(-n // page) for n in room]
    table = torch.full((S, max(pages)), -1, dtype=torch.int32)
    order = torch.randperm(sum(pages), generator=torch.Generator().manual_seed(2)).to(torch.int32)
    at = 0
    for s, n in enumerate(pages):
        table[s, :n] = order[at: at + n]
        at += n
    table = table.cuda()
    cache = la.kv4_cache(sum(pages), Hk, d, page)

    # prompts
    T = sum(lens)
    q, k, v = rnd(T, Hq), rnd(T, Hk), rnd(T, Hk)
    pos = torch.cat([torch.arange(n) for n in lens]).to(torch.int32).cuda()
    cu, L = R.starts(lens), torch.tensor(lens, dtype=torch.int32, device="cuda")
    qr, kr = la.rope(q, pos, freqs, k=k)
    o = la.prompt_attn(qr, kr, v, cu)
    la.kv4_append(cache, kr, v, cu, L, table)
    starts = [sum(lens[:s]) for s in range(S)]
    R.check(o, None, R.attention(qr, lambda s, h: (kr[starts[s]: starts[s] + lens[s], h // G],
                                                   v[starts[s]: starts[s] + lens[s], h // G]), lens, lens, True), "prompts")

    def reference(qt, n_new, now):
        # over what the cache holds, read back
        total = sum(now)
        kc, vc = la.kv4_read(cache, R.starts(now), torch.tensor(now, dtype=torch.int32, device="cuda"), table, total, d)
        b = [sum(now[:s]) for s in range(S)]
        return R.attention(qt, lambda s, h: (kc[b[s]: b[s] + now[s], h // G], vc[b[s]: b[s] + now[s], h // G]),
                           [n_new] * S, now, True)

    # tokens one by one
    one = R.starts([1] * S)
    now = list(lens)
    for step in range(3):
        q, k, v = rnd(S, Hq), rnd(S, Hk), rnd(S, Hk)
        p = L.clone()
        L += 1
        now = [n + 1 for n in now]
        qr, kr = la.rope(q, p, freqs, k=k)
        la.kv4_append(cache, kr, v, one, L, table)
        o = la.kv4_attn(qr, cache, one, L, table, 1)
        R.check(o, None, reference(qr, 1, now), f"token {step}")
    # four proposed tokens at once
    q, k, v = rnd(4 * S, Hq), rnd(4 * S, Hk), rnd(4 * S, Hk)
    p = (L[:, None] + torch.arange(4, device="cuda", dtype=torch.int32)).flatten()
    L += 4
    now = [n + 4 for n in now]
    cu4 = R.starts([4] * S)
    qr, kr = la.rope(q, p, freqs, k=k)
    la.kv4_append(cache, kr, v, cu4, L, table)
    R.check(la.kv4_attn(qr, cache, cu4, L, table, 4), None, reference(qr, 4, now), "four tokens")

    # the same step captured once and replayed: the lengths grow on the device
    sq, sk, sv, so = rnd(S, Hq), rnd(S, Hk), rnd(S, Hk), torch.empty((S, Hq, d), dtype=torch.bfloat16, device="cuda")
    L0, before = L.clone(), cache.clone()

    def step():
        p = L.clone()
        L.add_(1)
        qr, kr = la.rope(sq, p, freqs, k=sk)
        la.kv4_append(cache, kr, sv, one, L, table)
        la.kv4_attn(qr, cache, one, L, table, 1, out=so)

    inputs = [(rnd(S, Hq), rnd(S, Hk), rnd(S, Hk)) for _ in range(4)]
    eager = []
    for a, b, c in inputs:
        sq.copy_(a), sk.copy_(b), sv.copy_(c)
        step()
        eager.append(so.clone())
    after = cache.clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    L.copy_(L0), cache.copy_(before)
    for (a, b, c), want in zip(inputs, eager):
        sq.copy_(a), sk.copy_(b), sv.copy_(c)
        so.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(so, want)
    assert torch.equal(cache, after)


def test_a_chunk_over_context_in_4_bits_and_its_own_keys():
    # the chunk's queries over the context's cache, and over its own rows, joined by their log-sum-exps:
    # the attention over both
    H, d, n, m = 3, 128, 200, 700
    g = torch.Generator(device="cuda").manual_seed(3)
    q, kn, vn = (torch.randn((n, H, d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    kc, vc = (torch.randn((m, H, d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    pages = -(-m // 64)
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    cache, L, cu = la.kv4_cache(pages, H, d, 64), torch.tensor([m], dtype=torch.int32, device="cuda"), R.starts([n])
    la.kv4_append(cache, kc, vc, R.starts([m]), L, table)
    o1, l1 = la.kv4_attn(q, cache, cu, L, table, n, causal=False, want_lse=True)
    o2, l2 = la.prompt_attn(q, kn, vn, cu, causal=False, want_lse=True)
    top = torch.logaddexp(l1, l2)
    o = (o1.double() * (l1 - top).exp()[..., None] + o2.double() * (l2 - top).exp()[..., None])
    kq, vq = la.kv4_read(cache, R.starts([m]), L, table, m, d)
    k, v = torch.cat([kq, kn]), torch.cat([vq, vn])
    want, lse, tol, ltol = R.attention(q, lambda s, h: (k[:, h], v[:, h]), [n], [n + m], False)
    # each part is rounded once more than the whole is
    assert float(((o - want).abs() / (2 * tol + 2 * R.U * (o1.double().abs() + o2.double().abs()))).max()) <= 1.0
    assert float((top.double() - lse).abs().max()) < 1e-5


@pytest.mark.parametrize("d", [64, 128])
def test_far_strides(d):
    # rows 32 MB apart (the largest stride), 4.4 GB in all: q, k, v and the outputs are columns of one buffer
    T, Hq, Hkv, stride = 130, 4, 2, (1 << 24) - 8
    buf = torch.empty((T, stride), dtype=torch.bfloat16, device="cuda")
    at = lambda c, h: buf[:, c: c + h * d].unflatten(1, (h, d))       # noqa: E731
    q, k, v, o, k2, v2 = (at(c, h) for c, h in ((0, Hq), (1 << 20, Hkv), (1 << 23, Hkv), ((1 << 24) - 2048, Hq),
                                                (1 << 21, Hkv), (1 << 22, Hkv)))
    gen = torch.Generator(device="cuda").manual_seed(11)
    for x in (q, k, v):
        x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
    cu, pos, f = R.starts([T]), torch.arange(T, dtype=torch.int32, device="cuda"), la.rope_frequencies(d)
    near = [x.contiguous() for x in (q, k, v)]
    assert torch.equal(la.prompt_attn(q, k, v, cu, out=o), la.prompt_attn(*near, cu))
    assert torch.equal(o, la.prompt_attn(*near, cu))
    assert torch.equal(la.rope(q, pos, f, out=o), la.rope(near[0], pos, f))
    cache, lens = la.kv4_cache(9, Hkv, d, 16), torch.tensor([T], dtype=torch.int32, device="cuda")
    table = torch.arange(9, dtype=torch.int32, device="cuda").view(1, 9)
    la.kv4_append(cache, k, v, cu, lens, table)
    want = la.kv4_read(cache, cu, lens, table, T, d)
    got = la.kv4_read(cache, cu, lens, table, T, d, out=(k2, v2))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    again = torch.zeros_like(cache)
    la.kv4_append(again, near[1], near[2], cu, lens, table)
    read = la.kv4_read(again, cu, lens, table, T, d)
    assert torch.equal(read[0], want[0]) and torch.equal(read[1], want[1])
    for most in (1, T):
        rows, c = (q[-1:], R.starts([1])) if most == 1 else (q, cu)
        assert torch.equal(la.kv4_attn(rows, cache, c, lens, table, most, out=o[-1:] if most == 1 else o),
                           la.kv4_attn(rows.contiguous(), cache, c, lens, table, most))
