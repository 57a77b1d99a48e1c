"""Calls of la_prompt_attn_bwd at the ends of what it takes: starts that do not fit the rows, and far more buckets than
distances."""
import pytest
import torch

from paper_2605_31158_amd import la
import grad_reference as G
import seq_reference as R
from test_prompt_bias_gpu import make, rel
from test_prompt_bwd_gpu import grad_of, left

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("biased", [False, True], ids=["plain", "bias"])
@pytest.mark.parametrize("starts,lengths", [([0, 60, 60, 4000, 2 ** 31 - 1, -5], [60, 40]), ([-7, 30, 10, 10], [30]),
                                            ([90, 2 ** 31 - 1], [10])], ids=str)
def test_starts_held_to_the_rows(starts, lengths, d, biased):
    # starts past the rows, before them, or before the one in front: held to what is there, and nothing else is written
    T, first = 100, max(starts[0], 0)
    q, k, v = make([T], [T], 4, 2, d, 191)
    bias = rel(4, 192) if biased else None
    rows = slice(first, first + sum(lengths))
    o, lse = torch.zeros_like(q), torch.zeros((T, 4), device="cuda")
    o[rows], lse[rows] = left(q[rows], k[rows], v[rows], lengths, lengths, True, bias=bias)
    do = grad_of(q, 193)
    want = G.backward(do[rows], q[rows], k[rows], v[rows], o[rows], lse[rows], lengths, lengths, True, bias=bias)
    cu = torch.tensor(starts, dtype=torch.int32, device="cuda")
    held = [torch.full((T + 40, x.shape[1], d), 7.0, dtype=torch.bfloat16, device="cuda") for x in (q, k, v)]
    outs = tuple(x[20: 20 + T] for x in held) + ((torch.full_like(bias.weight, 7.0),) if biased else ())
    la.prompt_attn_bwd(do, q, k, v, o, lse, cu, bias=bias, out=outs)
    G.check([x[rows] for x in outs[:3]] + list(outs[3:]), want, f"{starts} {d} {biased}")
    for x in held:
        x[20 + rows.start: 20 + rows.stop] = 7.0
        assert bool((x == 7).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("buckets", [64, 65, 513, 514, 5000, 1 << 20])
def test_many_buckets(buckets, dtype):
    # few of them are named by a distance, the same one by several; the others' gradient is 0, written in every call
    lq, lk = [300, 1, 77], [340, 40, 77]
    q, k, v = make(lq, lk, 6, 2, 64, 194)
    g = torch.Generator(device="cuda").manual_seed(195)
    to = torch.randint(0, buckets, (257,), generator=g, device="cuda").to(torch.int32)
    to[100:110], to[0], to[256], to[50], to[51], to[52] = to[7], buckets - 1, 0, -3, buckets, 2 ** 31 - 1
    bias = la.RelativeBias(torch.randn((buckets, 6), generator=g, device="cuda").to(dtype), to, -128)
    cu_q, cu_k = R.starts(lq), R.starts(lk)
    o, lse = left(q, k, v, lq, lk, False, bias=bias)
    do = grad_of(q, 196)
    out = tuple(torch.full_like(x, 7.0) for x in (q, k, v, bias.weight))
    for _ in range(2):
        la.prompt_attn_bwd(do, q, k, v, o, lse, cu_q, cu_k, causal=False, bias=bias, out=out)
    G.check(out, G.backward(do, q, k, v, o, lse, lq, lk, False, bias=bias), f"{buckets} buckets")
    named = torch.zeros(buckets, dtype=torch.bool, device="cuda")
    named[to[(to >= 0) & (to < buckets)].long()] = True
    assert bool((out[3][~named] == 0).all())
    # no queries, and no sequences: zeros alone
    z = torch.zeros((0, 6, 64), dtype=torch.bfloat16, device="cuda")
    for starts in ([0], []):
        out[3].fill_(7.0)
        la.prompt_attn_bwd(z, z, k, v, z, lse[:0], R.starts(starts), R.starts([40] if starts else []), causal=False,
                           bias=bias, out=(z, *out[1:]))
        assert bool((out[3] == 0).all())


def test_many_buckets_captured():
    lq = [200, 70]
    q, k, v = make(lq, lq, 4, 2, 64, 197)
    to = torch.arange(0, 65 * 40, 40, dtype=torch.int32, device="cuda")
    bias = la.RelativeBias(torch.randn((3000, 4), device="cuda"), to, -32)
    cu = R.starts(lq)
    o, lse = left(q, k, v, lq, lq, True, bias=bias)
    do = grad_of(q, 198)
    ws = torch.empty(1 << 27, dtype=torch.uint8, device="cuda")
    out = tuple(torch.empty_like(x) for x in (q, k, v, bias.weight))
    call = lambda: la.prompt_attn_bwd(do, q, k, v, o, lse, cu, bias=bias, ws=ws, out=out)   # noqa: E731
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        call()
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        call()
    for i in range(4):
        do.copy_(grad_of(q, 199 + i))
        out[3].fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(out, la.prompt_attn_bwd(do, q, k, v, o, lse, cu, bias=bias)):
            assert torch.equal(x, y), i
