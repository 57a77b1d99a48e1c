"""Gradients of attention over packed prompts (la_prompt_attn_bwd) against 64 bits and against differences: lengths,
grouped heads, masks, a relative bias and its gradient, the gradient of the log-sum-exp, strides, rows and keys
outside the sequences, rows that see nothing, graph capture, two streams."""
import pytest
import torch

from paper_2605_31158_amd import la
import grad_reference as G
import seq_reference as R
from test_prompt_bias_gpu import make, rel

pytestmark = pytest.mark.gpu


def left(q, k, v, lq, lk, causal, scale=None, bias=None):
    """What the forward pass leaves, (o in bf16, lse in fp32), from 64 bits."""
    o, lse, _, _ = G.forward(q, k, v, lq, lk, causal, scale, bias)
    return o.to(torch.bfloat16), lse.float()


def grad_of(q, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(q.shape, generator=g, device="cuda").to(torch.bfloat16)


CASES = [
    # (query lengths, key lengths or None for the same, Hq, Hkv, d, causal)
    ([1], None, 1, 1, 64, True),
    ([1], None, 4, 2, 128, True),
    ([64], None, 2, 2, 128, True),
    ([63, 65, 1, 2], None, 2, 1, 64, True),
    ([127, 128, 129], None, 2, 2, 128, False),
    ([255, 256, 257], None, 2, 2, 64, True),
    ([1000], None, 3, 1, 128, True),                      # units are cut
    ([1000], None, 3, 3, 64, False),
    ([700, 1, 300], None, 5, 1, 64, True),
    ([333, 90], None, 14, 2, 128, True),
    ([40, 3], None, 40, 2, 64, False),
    ([6, 2], None, 300, 1, 64, True),                     # a group of more heads than a unit has rows
    ([0, 5, 0, 0, 70, 0], None, 4, 2, 128, True),         # empty sequences
    ([0, 0], None, 4, 2, 128, True),
    ([5, 7, 9], [0, 3, 200], 4, 2, 64, True),             # no keys; fewer keys than queries; more
    ([5, 7, 9], [0, 3, 200], 4, 2, 128, False),
    ([0, 7, 0], [130, 3, 1], 4, 2, 128, True),            # keys that no query sees
    ([500], [20], 2, 2, 128, True),                       # most rows see nothing
    ([1, 1, 1], [1000, 1, 64], 8, 2, 128, True),
    ([130], [2100], 6, 2, 64, True),
    ([2500], None, 2, 1, 128, True),
    ([1200] * 3, None, 4, 4, 64, False),
    (list(range(1, 130)), None, 4, 1, 64, True),          # more sequences than lanes of a wave
    ([3] * 1000, None, 2, 2, 128, True),
]


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
@pytest.mark.parametrize("biased", [False, True], ids=["plain", "bias"])
def test_against_64_bits(case, biased):
    lq, lk, Hq, Hkv, d, causal = case
    lk = lq if lk is None else lk
    print(f"[bwd] {str(lq)[:60]} over {str(lk)[:60]} {case[2:]} bias {biased}", flush=True)
    q, k, v = make(lq, lk, Hq, Hkv, d, 35)
    bias = rel(Hq, 36, both=len(lq) % 2 == 0, reach=100) if biased else None
    cu_q, cu_k = R.starts(lq), R.starts(lk)
    o, lse = left(q, k, v, lq, lk, causal, bias=bias)
    do = grad_of(q, 37)
    got = la.prompt_attn_bwd(do, q, k, v, o, lse, cu_q, cu_k, causal=causal, bias=bias)
    torch.cuda.synchronize()
    G.check(got, G.backward(do, q, k, v, o, lse, lq, lk, causal, bias=bias), f"{str(case)[:70]} bias {biased}")
    again = la.prompt_attn_bwd(do, q, k, v, o, lse, cu_q, cu_k, causal=causal, bias=bias)
    for x, y in zip(got, again):
        assert torch.equal(x, y)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("form", [([2500], [3000], 16, 16), ([1300, 200], [2300, 900], 32, 16), ([3000, 1], [150, 4000], 18, 9)],
                         ids=str)
@pytest.mark.parametrize("causal", [False, True])
def test_several_units_to_a_workgroup(form, d, causal):
    # more units of 128 rows than workgroups: without a mask a unit's walk starts in the middle and wraps
    lq, lk, Hq, Hkv = form
    q, k, v = make(lq, lk, Hq, Hkv, d, 95)
    cu_q, cu_k = R.starts(lq), R.starts(lk)
    o, lse = left(q, k, v, lq, lk, causal)
    do = grad_of(q, 96)
    got = la.prompt_attn_bwd(do, q, k, v, o, lse, cu_q, cu_k, causal=causal)
    G.check(got, G.backward(do, q, k, v, o, lse, lq, lk, causal), f"{form} d {d} causal {causal}")
    for x, y in zip(got, la.prompt_attn_bwd(do, q, k, v, o, lse, cu_q, cu_k, causal=causal)):
        assert torch.equal(x, y)


BIASES = [
    # (buckets, reach, both, weights)
    (8, 16, False, torch.float32),
    (32, 128, False, torch.bfloat16),
    (64, 256, True, torch.float32),
    (20, 34, True, torch.bfloat16),
    (128, 512, False, torch.float32),
]


@pytest.mark.parametrize("form", BIASES, ids=str)
@pytest.mark.parametrize("d", [64, 128])
def test_bias_forms(form, d):
    buckets, reach, both, dtype = form
    lq, lk = [300, 1, 77], [900, 40, 30]
    q, k, v = make(lq, lk, 6, 2, d, 38)
    bias = rel(6, 39, buckets, reach, both, dtype)
    o, lse = left(q, k, v, lq, lk, False, bias=bias)
    do = grad_of(q, 40)
    got = la.prompt_attn_bwd(do, q, k, v, o, lse, R.starts(lq), R.starts(lk), causal=False, bias=bias)
    assert got[3].dtype is dtype
    G.check(got, G.backward(do, q, k, v, o, lse, lq, lk, False, bias=bias), str(form))


@pytest.mark.parametrize("d", [64, 128])
def test_ranges_to_one_side_and_buckets_that_are_none(d):
    lq, lk = [300, 65], [340, 65]
    q, k, v = make(lq, lk, 4, 2, d, 41)
    cu_q, cu_k = R.starts(lq), R.starts(lk)
    do = grad_of(q, 42)
    g = torch.Generator(device="cuda").manual_seed(4)
    for lo, n in ((-200, 100), (20, 90), (-512, 513), (-1, 3), (0, 1), (400, 7), (-1 << 20, 9)):
        to = torch.arange(n, dtype=torch.int32, device="cuda")
        if n > 50:
            to[::7] = n
            to[3::11] = -1
        b = la.RelativeBias(torch.randn((n, 4), generator=g, device="cuda"), to, lo)
        for causal in (True, False):
            o, lse = left(q, k, v, lq, lk, causal, bias=b)
            got = la.prompt_attn_bwd(do, q, k, v, o, lse, cu_q, cu_k, causal=causal, bias=b)
            G.check(got, G.backward(do, q, k, v, o, lse, lq, lk, causal, bias=b), f"distances from {lo}, {n}")


@pytest.mark.parametrize("d", [64, 128])
def test_weights_that_hide(d):
    lq, lk = [200, 300, 3], [260, 100, 3]
    q, k, v = make(lq, lk, 4, 4, d, 43)
    b = rel(4, 44)
    b.weight[15, 0] = b.weight[31, 0] = -torch.inf
    b.weight[16:, 1] = b.weight[0, 1] = -torch.inf
    b.weight[:, 2] = -torch.inf
    for causal in (True, False):
        o, lse = left(q, k, v, lq, lk, causal, bias=b)
        do = grad_of(q, 45)
        got = la.prompt_attn_bwd(do, q, k, v, o, lse, R.starts(lq), R.starts(lk), causal=causal, bias=b)
        assert bool((got[0][:, 2] == 0).all()) and bool((got[1][:, 2] == 0).all()) and bool((got[3][:, 2] == 0).all())
        G.check(got, G.backward(do, q, k, v, o, lse, lq, lk, causal, bias=b), f"hidden, causal {causal}")


@pytest.mark.parametrize("scale", [0.02, 1.0])
def test_scales_and_peaks(scale):
    lq, lk = [200, 77], [300, 77]
    q, k, v = make(lq, lk, 4, 2, 128, 46, qscale=1.0)
    k[250:260] *= 4
    o, lse = left(q, k, v, lq, lk, True, scale)
    do = grad_of(q, 47)
    got = la.prompt_attn_bwd(do, q, k, v, o, lse, R.starts(lq), R.starts(lk), scale=scale)
    G.check(got, G.backward(do, q, k, v, o, lse, lq, lk, True, scale), f"scale {scale}")


@pytest.mark.parametrize("d", [64, 128])
def test_gradient_of_lse(d):
    # rows that see nothing have an lse of -inf, whose gradient may be anything
    lq, lk = [150, 40], [100, 90]
    q, k, v = make(lq, lk, 4, 2, d, 48)
    o, lse = left(q, k, v, lq, lk, True)
    do = grad_of(q, 49)
    dlse = torch.randn(lse.shape, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    dlse[lse == -torch.inf] = float("nan")
    got = la.prompt_attn_bwd(do, q, k, v, o, lse, R.starts(lq), R.starts(lk), dlse=dlse)
    want = G.backward(do, q, k, v, o, lse, lq, lk, True, dlse=dlse.nan_to_num())
    G.check(got, want, "with the gradient of lse")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("biased", [False, True], ids=["plain", "bias"])
def test_strides(d, biased):
    lq, Hq, Hkv = [70, 300, 1], 6, 2
    T = sum(lq)
    q, k, v = make(lq, lq, Hq, Hkv, d, 50)
    cu = R.starts(lq)
    bias = rel(Hq, 51) if biased else None
    o, lse = left(q, k, v, lq, lq, True, bias=bias)
    do = grad_of(q, 52)
    want = la.prompt_attn_bwd(do, q, k, v, o, lse, cu, bias=bias)
    G.check(want, G.backward(do, q, k, v, o, lse, lq, lq, True, bias=bias), "packed")
    # one buffer [T, Hq + 2 Hkv, d] in and out, o and do as [H, T, d]
    buf = torch.cat([q, k, v], 1)
    grads = torch.empty_like(buf)
    ht = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (o, do)]
    outs = (grads[:, :Hq], grads[:, Hq: Hq + Hkv], grads[:, Hq + Hkv:]) + ((torch.empty_like(bias.weight),) if biased else ())
    got = la.prompt_attn_bwd(ht[1], buf[:, :Hq], buf[:, Hq: Hq + Hkv], buf[:, Hq + Hkv:], ht[0], lse, cu, bias=bias,
                             out=outs)
    for x, y, z in zip(got, want, outs):
        assert torch.equal(x, y) and x.data_ptr() == z.data_ptr()
    # key and value heads given as a broadcast, a gradient of o that is one row for all heads
    k1, v1, d1 = k[:, :1], v[:, :1], do[:, :1].expand(T, Hq, d)
    o1, lse1 = left(q, k1, v1, lq, lq, True, bias=bias)
    got = la.prompt_attn_bwd(d1, q, k1.expand(T, Hkv, d), v1.expand(T, Hkv, d), o1, lse1, cu, bias=bias)
    ks, vs = k1.expand(T, Hkv, d).contiguous(), v1.expand(T, Hkv, d).contiguous()
    G.check(got, G.backward(d1.contiguous(), q, ks, vs, o1, lse1, lq, lq, True, bias=bias), "broadcasts")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("biased", [False, True], ids=["plain", "bias"])
def test_rows_outside_the_sequences(d, biased):
    # rows behind the last sequence keep what they hold, and what their inputs hold reaches nothing
    lq, spare = [30, 65, 100], 37
    q, k, v = make(lq, lq, 4, 2, d, 53, spare=spare)
    T = sum(lq)
    bias = rel(4, 54) if biased else None
    o, lse = (torch.full_like(q, float("nan")), torch.full((T + spare, 4), float("nan"), device="cuda"))
    o[:T], lse[:T] = left(q[:T], k[:T], v[:T], lq, lq, True, bias=bias)
    do = grad_of(q, 55)
    want = G.backward(do[:T], q[:T], k[:T], v[:T], o[:T], lse[:T], lq, lq, True, bias=bias)
    for x in (q, k, v, do):
        x[T:] = float("nan")
    outs = tuple(torch.full_like(x, 7.0) for x in (q, k, v)) + ((torch.empty_like(bias.weight),) if biased else ())
    la.prompt_attn_bwd(do, q, k, v, o, lse, R.starts(lq), bias=bias, out=outs)
    G.check([x[:T] for x in outs[:3]] + list(outs[3:]), want, "spare rows")
    for x in outs[:3]:
        assert bool((x[T:] == 7).all())
    # only the middle sequence is finite
    for x in (q, k, v, do):
        x[:30], x[95:] = float("nan"), float("inf")
    got = la.prompt_attn_bwd(do, q, k, v, o, lse, R.starts(lq), bias=bias)
    for x, y in zip(got[:3], outs):
        assert torch.equal(x[30:95], y[30:95])


def test_starts_that_do_not_fit():
    # starts past the rows and sequences that would end before they start: held to what is there
    q, k, v = make([100], [100], 2, 2, 64, 56)
    o, lse = left(q, k, v, [100], [100], True)
    do = grad_of(q, 57)
    cu = torch.tensor([0, 100, 50, 4000, 2 ** 31 - 1, -5], dtype=torch.int32, device="cuda")
    for bias in (None, rel(2, 58)):
        outs = tuple(torch.full_like(x, 7.0) for x in (q, k, v)) + (() if bias is None else (torch.empty_like(bias.weight),))
        la.prompt_attn_bwd(do, q, k, v, o, lse, cu, bias=bias, out=outs)
        torch.cuda.synchronize()


def test_nothing_to_do():
    z = torch.zeros((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    k = torch.ones((40, 2, 64), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((0, 2), device="cuda")
    bias = rel(2, 59)
    for b in (None, bias):
        got = la.prompt_attn_bwd(z, z, k, k, z, lse, R.starts([0, 0]), R.starts([10, 30]), bias=b)
        assert all(bool((x == 0).all()) for x in got)
        outs = (z, torch.full_like(k, 7.0), torch.full_like(k, 7.0)) + (() if b is None else (torch.ones_like(b.weight),))
        la.prompt_attn_bwd(z, z, k, k, z, lse, R.starts([]), R.starts([]), bias=b, out=outs)
        assert bool((outs[1] == 7).all()) and (b is None or bool((outs[3] == 0).all()))
        got = la.prompt_attn_bwd(k, k, z, z, torch.zeros_like(k), torch.full((40, 2), -torch.inf, device="cuda"),
                                 R.starts([40]), R.starts([0]), bias=b)
        assert bool((got[0] == 0).all()) and (b is None or bool((got[3] == 0).all()))


@pytest.mark.parametrize("biased", [False, True], ids=["plain", "bias"])
def test_against_differences(biased):
    # single inputs moved by +-h: central differences of sum(do o) with the 64-bit forward, off by h^2 of third
    # derivatives (1e-8 times some tens) and 2^-53 / h of the sum.  dlse takes out what the rounding of o to bf16 makes
    # of delta, so that the kernel's values are the true gradients within its bounds.
    lq, lk = [40, 25], [70, 25]
    q, k, v = make(lq, lk, 4, 2, 64, 60)
    bias = rel(4, 61, buckets=16, reach=30) if biased else None
    o, lse = left(q, k, v, lq, lk, True, bias=bias)
    do = grad_of(q, 62)
    true = G.forward(q, k, v, lq, lk, True, bias=bias)[0]
    dlse = (do.double() * (o.double() - true)).sum(-1).float()
    got = la.prompt_attn_bwd(do, q, k, v, o, lse, R.starts(lq), R.starts(lk), bias=bias, dlse=dlse)
    want = G.backward(do, q, k, v, o, lse, lq, lk, True, bias=bias, dlse=dlse)
    xs = [q.double(), k.double(), v.double()] + ([bias.weight.double()] if biased else [])

    def total(ys):
        b = None if not biased else (ys[3], bias.bucket, bias.lo)
        return float((G.forward(*ys[:3], lq, lk, True, bias=b)[0] * do.double()).sum())

    g = torch.Generator().manual_seed(6)
    h = 1e-4
    for i, (x, name) in enumerate(zip(xs, ("dq", "dk", "dv", "dw"))):
        for n in torch.randint(0, x.numel(), (12,), generator=g).tolist():
            step = torch.zeros_like(x).flatten()
            step[n] = h
            up, down = list(xs), list(xs)
            up[i], down[i] = x + step.view_as(x), x - step.view_as(x)
            diff = (total(up) - total(down)) / (2 * h)
            have, bound = float(got[i].flatten()[n]), float(want[name][1].flatten()[n])
            assert abs(have - diff) <= bound + 1e-6, (name, n, have, diff, bound)


@pytest.mark.parametrize("biased", [False, True], ids=["plain", "bias"])
def test_captured_and_replayed(biased):
    lq, lk = [600, 37], [700, 37]
    q, k, v = make(lq, lk, 4, 2, 64, 63)
    cu_q, cu_k = R.starts(lq), R.starts(lk)
    bias = rel(4, 64) if biased else None
    o, lse = left(q, k, v, lq, lk, True, bias=bias)
    do = grad_of(q, 65)
    ws = torch.empty(1 << 27, dtype=torch.uint8, device="cuda")
    outs = tuple(torch.empty_like(x) for x in (q, k, v)) + ((torch.empty_like(bias.weight),) if biased else ())
    st = torch.cuda.Stream()
    call = lambda: la.prompt_attn_bwd(do, q, k, v, o, lse, cu_q, cu_k, bias=bias, ws=ws, out=outs)   # noqa: E731
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        call()
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        call()
    for i in range(4):
        do.copy_(grad_of(q, 70 + i))
        if i == 2:                                            # other lengths, read on the GPU
            cu_q.copy_(R.starts([500, 137]))
        graph.replay()
        torch.cuda.synchronize()
        want = la.prompt_attn_bwd(do, q, k, v, o, lse, cu_q, cu_k, bias=bias)
        torch.cuda.synchronize()
        for x, y in zip(outs, want):
            assert torch.equal(x, y), i


def test_two_streams():
    lq = [900, 70]
    q, k, v = make(lq, lq, 4, 2, 128, 66)
    cu = R.starts(lq)
    o, lse = left(q, k, v, lq, lq, True)
    dos = [grad_of(q, 80), grad_of(q, 81)]
    want = [la.prompt_attn_bwd(x, q, k, v, o, lse, cu) for x in dos]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s, x in zip(streams, dos):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append([la.prompt_attn_bwd(x, q, k, v, o, lse, cu) for _ in range(3)])
    torch.cuda.synchronize()
    for w, runs in zip(want, got):
        for r in runs:
            assert all(torch.equal(x, y) for x, y in zip(w, r))


def test_two_graphs_share_scratch():
    # two captured calls of different sizes and kinds with one scratch, replayed in turn with eager work between
    ws = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    st = torch.cuda.Stream()
    calls = []
    for n, (lq, lk, H, K, d, causal, form) in enumerate([([700, 90], [700, 90], 4, 4, 64, False, (32, 128, True)),
                                                          ([130, 1, 900], [300, 40, 900], 6, 2, 128, True, None)]):
        q, k, v = make(lq, lk, H, K, d, 110 + n)
        bias = None if form is None else rel(H, 120 + n, *form)
        cu_q, cu_k = R.starts(lq), R.starts(lk)
        o, lse = left(q, k, v, lq, lk, causal, bias=bias)
        do = grad_of(q, 130 + n)
        outs = tuple(torch.empty_like(x) for x in (q, k, v)) + (() if bias is None else (torch.empty_like(bias.weight),))

        def call(out=None, ws=None, a=(do, q, k, v, o, lse, cu_q, cu_k), causal=causal, bias=bias):
            return la.prompt_attn_bwd(*a, causal=causal, bias=bias, ws=ws, out=out)

        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            call(outs, ws)
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            call(outs, ws)
        calls.append((graph, call, do, outs))
    for i in range(6):
        graph, call, do, outs = calls[i % 2]
        do.copy_(grad_of(do, 140 + i))
        ws[::4097].fill_(i)                                   # what the other call left there does not matter
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(outs, call()):
            assert torch.equal(x, y), i


@pytest.mark.parametrize("d", [64, 128])
def test_everything_at_once(d):
    # a bias, the gradient of lse, one gradient row for all heads, columns of one buffer, a scale, keys past the queries
    lq, lk, H, K = [90, 3, 200], [300, 50, 200], 6, 3
    q, k, v = make(lq, lk, H, K, d, 150, qscale=1.0)
    bias = rel(H, 151, 32, 200, True, torch.bfloat16)
    o, lse = left(q, k, v, lq, lk, False, 0.2, bias)
    do = grad_of(q, 152)[:, :1].expand(sum(lq), H, d)
    dlse = torch.randn(lse.shape, generator=torch.Generator(device="cuda").manual_seed(8), device="cuda")
    kv = torch.cat([k, v], 1)
    grads = torch.empty_like(kv)
    outs = (torch.empty((H, sum(lq), d), dtype=torch.bfloat16, device="cuda").transpose(0, 1), grads[:, :K], grads[:, K:],
            torch.empty_like(bias.weight))
    got = la.prompt_attn_bwd(do, q, kv[:, :K], kv[:, K:], o, lse, R.starts(lq), R.starts(lk), causal=False, scale=0.2,
                             bias=bias, dlse=dlse, out=outs)
    G.check(got, G.backward(do, q, k, v, o, lse, lq, lk, False, 0.2, bias, dlse), "everything")


def test_refusals():
    q, k, v = make([40], [40], 4, 2, 64, 160)
    cu = R.starts([40])
    o, lse = la.prompt_attn(q, k, v, cu, want_lse=True)
    b = rel(4, 161)
    good = dict(do=q, q=q, k=k, v=v, o=o, lse=lse, cu_q=cu)
    la.prompt_attn_bwd(**good)
    for bad in (dict(do=q[:39]), dict(do=q.float()), dict(o=o[:, :2]), dict(lse=lse[:, :2]), dict(lse=lse.double()),
                dict(lse=lse.t().contiguous().t()), dict(dlse=lse[:20]), dict(k=k[:, :, :32]), dict(v=v[:30]), dict(cu_q=cu.long()),
                dict(do=q[:, :, :1].expand(40, 4, 64)), dict(out=(q, k)), dict(out=(q, k, v[:30])), dict(bias=b, out=(q, k, v)),
                dict(bias=b, out=(q, k, v, b.weight[:4])), dict(bias=b._replace(weight=b.weight[:, :2])),
                dict(bias=b._replace(weight=b.weight.half())), dict(bias=b._replace(weight=b.weight.t())),
                dict(bias=b._replace(bucket=b.bucket.long())), dict(bias=b._replace(bucket=b.bucket.cpu())),
                dict(bias=b._replace(bucket=torch.zeros(514, dtype=torch.int32, device="cuda"))),
                dict(bias=b._replace(lo=1 << 21)), dict(ws=torch.empty(16, dtype=torch.uint8))):
        with pytest.raises((TypeError, ValueError)):
            la.prompt_attn_bwd(**{**good, **bad})
    for bad in (dict(ws=torch.empty(256, dtype=torch.uint8, device="cuda")), dict(scale=float("nan")),
                dict(bias=b._replace(lo=(1 << 20) - 3)), dict(bias=b, scale=1e-30)):
        with pytest.raises(la.LaError):
            la.prompt_attn_bwd(**{**good, **bad})
