"""Attention over packed prompts (la_prompt_attn) against 64 bits: lengths from none to several
workgroups' worth, grouped heads, causal or not, strides, rows behind the last sequence, values that are
not finite next to a sequence, graph capture and two streams."""
import pytest
import torch

from paper_2605_31158_amd import la
import seq_reference as R

pytestmark = pytest.mark.gpu


def make(lq, lk, Hq, Hkv, d, seed, spare=0, qscale=1.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    f = lambda n, h, s: (torch.randn((n, h, d), generator=g, device="cuda") * s).to(torch.bfloat16)   # noqa: E731
    return f(sum(lq) + spare, Hq, qscale), f(sum(lk) + spare, Hkv, 1.0), f(sum(lk) + spare, Hkv, 1.0)


def reference(q, k, v, lq, lk, causal, scale=None):
    G = q.shape[1] // k.shape[1]
    at = [sum(lk[:s]) for s in range(len(lk))]
    return R.attention(q[: sum(lq)], lambda s, h: (k[at[s]: at[s] + lk[s], h // G], v[at[s]: at[s] + lk[s], h // G]),
                       lq, lk, causal, scale)


CASES = [
    # (query lengths, key lengths or None for the same, Hq, Hkv, d, causal)
    ([1], None, 1, 1, 64, True),
    ([1], None, 4, 2, 128, True),
    ([64], None, 2, 2, 128, True),
    ([63, 65, 1, 2], None, 2, 1, 64, True),
    ([255, 256, 257], None, 2, 2, 128, True),
    ([255, 256, 257], None, 2, 2, 64, False),
    ([1000], None, 3, 1, 128, True),                      # a group of 3: 255 of 256 rows used
    ([700, 1, 300], None, 5, 1, 64, True),
    ([333, 90], None, 14, 2, 128, True),
    ([40, 3], None, 40, 2, 64, True),
    ([6, 2], None, 300, 1, 64, True),                     # a group of more heads than a workgroup has rows
    ([0, 5, 0, 0, 70, 0], None, 4, 2, 128, True),         # empty sequences
    ([0, 0], None, 4, 2, 128, True),
    ([5, 7, 9], [0, 3, 200], 4, 2, 64, True),             # no keys; fewer keys than queries; more
    ([5, 7, 9], [0, 3, 200], 4, 2, 128, False),
    ([500], [20], 2, 2, 128, True),                       # most rows see nothing
    ([1, 1, 1], [1000, 1, 64], 8, 2, 128, True),          # one new token each
    ([130], [2100], 6, 2, 64, True),
    ([2500], None, 2, 1, 128, True),
    ([1200] * 3, None, 4, 4, 64, False),
    (list(range(1, 130)), None, 4, 1, 64, True),          # more sequences than lanes of a wave
    ([3] * 1000, None, 2, 2, 128, True),
]


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_against_64_bits(case):
    lq, lk, Hq, Hkv, d, causal = case
    lk = lq if lk is None else lk
    print(f"[prompt] {str(lq)[:60]} over {str(lk)[:60]} Hq {Hq} Hkv {Hkv} d {d} causal {causal}", flush=True)
    q, k, v = make(lq, lk, Hq, Hkv, d, 5)
    cu_q, cu_k = R.starts(lq), R.starts(lk)
    o, lse = la.prompt_attn(q, k, v, cu_q, cu_k, causal=causal, want_lse=True)
    torch.cuda.synchronize()
    R.check(o, lse, reference(q, k, v, lq, lk, causal), str(case)[:80])
    again, lse2 = la.prompt_attn(q, k, v, cu_q, cu_k, causal=causal, want_lse=True)
    assert torch.equal(o, again) and torch.equal(lse, lse2)      # bit for bit
    assert torch.equal(la.prompt_attn(q, k, v, cu_q, cu_k, causal=causal), o)


@pytest.mark.parametrize("scale", [0.02, 1.0])
def test_scales_and_peaks(scale):
    # logits of +-100 at scale 1: one key takes nearly everything, the maximum is raised late
    lq, lk = [200, 77], [300, 77]
    q, k, v = make(lq, lk, 4, 2, 128, 6, qscale=1.0)
    k[250:260] *= 4
    o, lse = la.prompt_attn(q, k, v, R.starts(lq), R.starts(lk), scale=scale, want_lse=True)
    R.check(o, lse, reference(q, k, v, lq, lk, True, scale), f"scale {scale}")


@pytest.mark.parametrize("d", [64, 128])
def test_strides(d):
    lq, Hq, Hkv = [70, 300, 1], 6, 2
    T = sum(lq)
    q, k, v = make(lq, lq, Hq, Hkv, d, 7)
    cu = R.starts(lq)
    want = reference(q, k, v, lq, lq, True)
    # one buffer [T, Hq + 2 Hkv, d], rows of [H, T, d], and a wide buffer's middle; out in place of a strided one
    buf = torch.cat([q, k, v], 1)
    o = la.prompt_attn(buf[:, :Hq], buf[:, Hq: Hq + Hkv], buf[:, Hq + Hkv:], cu)
    R.check(o, None, want, "one buffer")
    ht = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v)]
    out = torch.empty((Hq, T, d), dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    assert torch.equal(la.prompt_attn(*ht, cu, out=out), o) and torch.equal(out, o)
    wide = torch.zeros((T, Hkv, 2, d + 64), dtype=torch.bfloat16, device="cuda")
    wide[:, :, 0, 32: 32 + d], wide[:, :, 1, 32: 32 + d] = k, v
    assert torch.equal(la.prompt_attn(q, wide[:, :, 0, 32: 32 + d], wide[:, :, 1, 32: 32 + d], cu), o)
    # one key head for all, given as a broadcast
    k1, v1 = k[:, :1], v[:, :1]
    a = la.prompt_attn(q, k1, v1, cu)
    b = la.prompt_attn(q, k1.expand(T, Hkv, d), v1.expand(T, Hkv, d), cu)
    R.check(a, None, reference(q, k1, v1, lq, lq, True), "one head")
    R.check(b, None, reference(q, k1, v1, lq, lq, True), "one head, broadcast")


@pytest.mark.parametrize("d", [64, 128])
def test_rows_outside_the_sequences(d):
    # rows behind the last sequence keep what they hold; keys there, and those of the next sequence, are
    # not finite and do not reach the sequences in front of them
    lq, spare = [30, 65, 100], 37
    q, k, v = make(lq, lq, 4, 2, d, 8, spare=spare)
    T = sum(lq)
    want = reference(q, k, v, lq, lq, True)
    nan = float("nan")
    q[T:], k[T:], v[T:] = nan, nan, float("inf")
    out = torch.full_like(q, 7.0)
    lse = torch.full((T + spare, 4), 7.0, device="cuda")
    la.prompt_attn(q, k, v, R.starts(lq), out=out, lse_out=lse)
    R.check(out[:T], lse[:T], want, "spare rows")
    assert bool((out[T:] == 7).all()) and bool((lse[T:] == 7).all())
    # only the middle sequence is finite
    q2, k2, v2 = (x.clone() for x in (q, k, v))
    for x in (k2, v2):
        x[: lq[0]] = nan
        x[lq[0] + lq[1]:] = nan
    o = la.prompt_attn(q2, k2, v2, R.starts(lq))
    rows = slice(lq[0], lq[0] + lq[1])
    assert torch.equal(o[rows], out[rows])
    # starts that run backwards or past the rows are held to the rows there are (rows 20 to 29 belong to two
    # sequences then, and hold the result of either)
    cu = torch.tensor([0, 30, 20, 100000], dtype=torch.int32, device="cuda")
    o = la.prompt_attn(q, k, v, cu)
    torch.cuda.synchronize()
    assert torch.equal(o[:20], out[:20])


def test_graph_and_streams():
    lq = [400, 33, 700]
    q, k, v = make(lq, lq, 8, 2, 128, 9)
    cu = R.starts(lq)
    ref = la.prompt_attn(q, k, v, cu, want_lse=True)
    out, lse = torch.empty_like(q), torch.empty((sum(lq), 8), device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        la.prompt_attn(q, k, v, cu, out=out, lse_out=lse)
    for r in range(4):
        out.zero_(), lse.zero_()
        graph.replay()
        eager = la.prompt_attn(q, k, v, cu)
        torch.cuda.synchronize()
        assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1]) and torch.equal(eager, ref[0]), r
    # the lengths are read when the graph runs
    cu2 = cu.clone()
    cu.copy_(R.starts([100, 33, 600]))
    graph.replay()
    torch.cuda.synchronize()
    want = la.prompt_attn(q, k, v, cu)
    n = 733
    assert torch.equal(out[:n], want[:n])
    cu.copy_(cu2)
    # two calls at once
    q2, k2, v2 = make(lq, lq, 8, 2, 128, 10)
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    outs = []
    for _ in range(3):
        with torch.cuda.stream(a):
            outs.append((la.prompt_attn(q, k, v, cu), 0))
        with torch.cuda.stream(b):
            outs.append((la.prompt_attn(q2, k2, v2, cu), 1))
    torch.cuda.synchronize()
    want = (ref[0], la.prompt_attn(q2, k2, v2, cu))
    assert all(torch.equal(o, want[i]) for o, i in outs)


def test_random_lengths():
    gen = torch.Generator().manual_seed(3)
    for n in range(24):
        S = int(torch.randint(1, 9, (1,), generator=gen))
        lq = torch.randint(0, 400, (S,), generator=gen).tolist()
        lk = [x + int(torch.randint(-20, 300, (1,), generator=gen)) for x in lq]
        lk = [max(0, x) for x in lk]
        Hkv = [1, 2, 3][n % 3]
        G, d, causal = [1, 2, 3, 4, 7][n % 5], [64, 128][n % 2], n % 4 != 3
        print(f"[prompt] random {n}: {lq} over {lk} G {G} Hkv {Hkv} d {d}", flush=True)
        q, k, v = make(lq, lk, G * Hkv, Hkv, d, 100 + n)
        o, lse = la.prompt_attn(q, k, v, R.starts(lq), R.starts(lk), causal=causal, want_lse=True)
        R.check(o, lse, reference(q, k, v, lq, lk, causal), f"random {n}")


def test_without_keys_and_shared_workspace():
    q = torch.randn((5, 4, 64), device="cuda").to(torch.bfloat16)
    none = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    o, lse = la.prompt_attn(q, none, none, R.starts([2, 3]), R.starts([0, 0]), want_lse=True)
    assert bool((o == 0).all()) and bool((lse == -torch.inf).all())
    assert la.prompt_attn(q[:0], none, none, R.starts([0, 0])).shape == (0, 4, 64)
    # one workspace for several calls in turn, and captured ones among them
    ws = torch.empty(1 << 27, dtype=torch.uint8, device="cuda")
    sizes = [([900], 128), ([20, 300], 64), ([5] * 40, 128)]
    made = [(*make(lq, lq, 8, 2, d, 20 + i), R.starts(lq)) for i, (lq, d) in enumerate(sizes)]
    want = [la.prompt_attn(*m) for m in made]
    graphs, outs = [], []
    for m in made:
        out = torch.empty_like(m[0])
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            la.prompt_attn(*m, ws=ws, out=out)
        graphs.append(graph), outs.append(out)
    for r in range(3):
        for graph, out, w, m in zip(graphs, outs, want, made):
            out.zero_()
            graph.replay()
            assert torch.equal(la.prompt_attn(*m, ws=ws), w)
            torch.cuda.synchronize()
            assert torch.equal(out, w), r


def test_wide_strides():
    # a head's rows lie 64 MB apart
    L, H = 1 << 18, 24
    buf = torch.empty((H, L, 128), dtype=torch.bfloat16, device="cuda")
    q = buf[:, :70].transpose(0, 1)
    q.copy_(torch.randn((70, H, 128), device="cuda"))
    k, v = (torch.randn((70, 1, 128), device="cuda").to(torch.bfloat16) for _ in range(2))
    o = la.prompt_attn(q, k, v, R.starts([70]))
    R.check(o, None, reference(q, k, v, [70], [70], True), "wide strides")


@pytest.mark.parametrize("lq,lk", [([512], [512]), ([513], [513]), ([5000], [500]), ([100] * 5, [100] * 5),
                                   ([3] * 700, [0] * 300 + [1] * 300 + [2] * 100), ([300, 800], [500, 12]),
                                   ([300, 800], [500, 13])], ids=lambda x: f"{len(x)}x{x[0]}")
@pytest.mark.parametrize("causal", [True, False])
def test_few_keys(lq, lk, causal):
    # up to 512 keys in all no work is split, whatever the number of queries and sequences
    q, k, v = make(lq, lk, 12, 4, 64, 31)
    o, lse = la.prompt_attn(q, k, v, R.starts(lq), R.starts(lk), causal=causal, want_lse=True)
    R.check(o, lse, reference(q, k, v, lq, lk, causal), "few keys")
