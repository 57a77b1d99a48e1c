"""The 4-bit cache (la_kv4_append, la_kv4_read) and the attention over it (la_kv4_attn) against 64 bits."""
import numpy as np
import pytest
import torch

from paper_2605_31158_amd import la
import seq_reference as R

pytestmark = pytest.mark.gpu

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantised(x):
    """The definition, in numpy: x float64 [.., d] -> the values that the cache holds."""
    b = x.reshape(*x.shape[:-1], -1, 32)
    top = np.abs(b).max(-1, keepdims=True)
    bad = ~np.isfinite(b).all(-1, keepdims=True)
    safe = np.where(np.isfinite(top) & (top > 0), top, 1.0)
    e = np.floor(np.log2(safe)) - 2
    e = e - (safe < 4 * 2.0 ** e) + (safe >= 8 * 2.0 ** e)           # whatever the logarithm's rounding
    e = np.where(safe >= 7 * 2.0 ** e, e + 1, e)
    e = np.clip(np.where(top > 0, e, -125), -125, 125)
    y = np.abs(np.where(np.isfinite(b), b, 0.0)) / 2.0 ** e
    far = np.abs(y[..., None] - GRID)
    near = far.min(-1, keepdims=True)
    code = np.where(far == near, np.arange(8) + 100 * (np.arange(8) % 2), 1000).argmin(-1)   # ties: the even code
    v = np.where(bad, np.nan, np.sign(np.where(np.isfinite(b), b, 0.0)) * GRID[code] * 2.0 ** e)
    return v.reshape(x.shape)


def pages_for(lens, page, seed, spare=2):
    """(table, number of pages): each sequence's pages, handed out in random order; spare entries hold -1."""
    need = [-(-max(0, n) // page) for n in lens]
    n = sum(need) + spare
    order = torch.randperm(n, generator=torch.Generator().manual_seed(seed)).tolist()
    table = torch.full((len(lens), max(1, max(need) if need else 1) + 1), -1, dtype=torch.int32)
    at = 0
    for s, m in enumerate(need):
        table[s, :m] = torch.tensor(order[at: at + m], dtype=torch.int32)
        at += m
    return table.cuda(), n


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def filled(lens, Hkv, d, page, seed, fill=0xFF, scale=1.0):
    """A cache of sequences of these lengths (the rest of its bytes `fill`): cache, table, lens, and the K and V
    that it stands for, packed."""
    table, n = pages_for(lens, page, seed)
    cache = la.kv4_cache(n, Hkv, d, page)
    cache.fill_(fill)
    g = torch.Generator(device="cuda").manual_seed(seed)
    k, v = ((torch.randn((sum(lens), Hkv, d), generator=g, device="cuda") * scale).to(torch.bfloat16) for _ in range(2))
    cu, L = R.starts(lens), ints(lens)
    la.kv4_append(cache, k, v, cu, L, table)
    kq, vq = la.kv4_read(cache, cu, L, table, sum(lens), d)
    return cache, table, L, kq, vq


@pytest.mark.parametrize("d", [64, 128])
def test_every_value(d):
    # every bf16 value beside others of its size, and alone with a large or small neighbour
    bits = np.arange(65536, dtype=np.uint16)
    x = bits.copy()
    alone = np.zeros((4096, 32), np.uint16)
    alone[:, 0] = bits[::16]
    alone[:, 1] = bits[7::16]
    mixed = np.random.default_rng(1).integers(0, 0x7F80, (4096, 32)).astype(np.uint16)
    rows = np.concatenate([x, alone.ravel(), mixed.ravel()]).reshape(-1, d)
    t = la.bf16_from_bits(rows)[:, None]
    T = t.shape[0]
    table, n = pages_for([T], 64, 1)
    cache = la.kv4_cache(n, 1, d, 64)
    la.kv4_append(cache, t, t.flip(0), R.starts([T]), ints([T]), table)
    k, v = la.kv4_read(cache, R.starts([T]), ints([T]), table, T, d)
    want = quantised(t[:, 0].double().cpu().numpy())
    np.testing.assert_array_equal(k[:, 0].double().cpu().numpy(), want)
    np.testing.assert_array_equal(v[:, 0].double().cpu().numpy(), want[::-1])


CASES = [
    # (tokens entered, length with them, Hkv, d, page)
    ([1], [1], 1, 64, 16),
    ([1, 1, 1], [5, 64, 65], 2, 128, 64),
    ([3, 0, 17, 1], [20, 9, 17, 4], 3, 128, 16),
    ([40, 7], [33, 7], 2, 64, 32),                 # more rows than the sequence is long: the first are dropped
    ([0, 0, 5, 0], [3, 0, 130, 0], 1, 128, 128),
    ([1] * 70, list(range(1, 71)), 1, 64, 16),
    ([1] * 1500, [17] * 1500, 1, 64, 16),          # more starts than the search holds at once
    ([900], [1000], 4, 128, 64),
]


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_append_and_read(case):
    new, lens, Hkv, d, page = case
    print(f"[kv4] {str(new)[:50]} of {str(lens)[:50]} heads {Hkv} d {d} page {page}", flush=True)
    T = sum(new) + 3
    table, n = pages_for(lens, page, 2)
    g = torch.Generator(device="cuda").manual_seed(3)
    buf = torch.randn((T, 2 * Hkv, d), generator=g, device="cuda").to(torch.bfloat16)
    k, v = buf[:, :Hkv], buf[:, Hkv:]                                 # rows with a stride
    cache = la.kv4_cache(n, Hkv, d, page)
    cache.fill_(0xAB)
    cu, L = R.starts(new), ints(lens)
    la.kv4_append(cache, k, v, cu, L, table)
    # reads: every row from its place, rows of no sequence as they were
    out = [torch.full((Hkv, T, d), 9.0, dtype=torch.bfloat16, device="cuda").transpose(0, 1) for _ in range(2)]
    kr, vr = la.kv4_read(cache, cu, L, table, T, d, out=out)
    assert bool((kr[sum(new):] == 9).all()) and bool((vr[sum(new):] == 9).all())
    tab, raw = table.cpu().numpy(), cache.cpu().numpy()
    want = [quantised(x.double().cpu().numpy()) for x in (k, v)]
    touched = np.zeros(raw.shape, bool)
    a, b, w = page * d // 2, page * d // 32, d // 32
    t = 0
    for s, m in enumerate(new):
        for i in range(m):
            pos = lens[s] - m + i
            for x, wx in ((kr, want[0]), (vr, want[1])):
                np.testing.assert_array_equal(x[t].double().cpu().numpy(), wx[t] if pos >= 0 else 0 * wx[t])
            if pos >= 0:
                pg, at = tab[s, pos // page], pos % page
                touched[pg, :, at * d // 2: (at + 1) * d // 2] = True
                q = a + b + (at // 4) * 2 * d + (at % 4) * w
                for ch in range(16):
                    touched[pg, :, q + ch * 4 * w: q + ch * 4 * w + w] = True
                for blk in range(d // 32):
                    touched[pg, :, a + blk * page + at] = touched[pg, :, 2 * a + b + blk * page + at] = True
                # the documented layout, byte by byte, of one head
                row = raw[pg, Hkv - 1]
                by = row[at * d // 2: (at + 1) * d // 2].astype(int)
                code = np.stack([by & 15, by >> 4], -1).ravel()
                sc = 2.0 ** (row[a + np.arange(d // 32) * page + at].astype(float) - 127)
                val = np.where(code > 7, -1.0, 1.0) * GRID[code & 7] * np.repeat(sc, 32)
                np.testing.assert_array_equal(val, want[0][t, Hkv - 1])
                by = np.concatenate([row[q + ch * 4 * w: q + ch * 4 * w + w] for ch in range(16)]).astype(int)
                code = np.stack([by & 15, by >> 4], -1).ravel()
                sc = 2.0 ** (row[2 * a + b + np.arange(d // 32) * page + at].astype(float) - 127)
                val = np.where(code > 7, -1.0, 1.0) * GRID[code & 7] * np.repeat(sc, 32)
                np.testing.assert_array_equal(val, want[1][t, Hkv - 1])
            t += 1
    assert (raw[~touched] == 0xAB).all()                              # nothing else was written


def test_pages_that_do_not_exist():
    d, page, Hkv = 128, 16, 2
    lens = [50, 40]
    table = torch.tensor([[3, -1, 1, 2, 7], [0, 4, 1000000, -5, 2]], dtype=torch.int32, device="cuda")
    cache = la.kv4_cache(5, Hkv, d, page)
    k, v = (torch.randn((90, Hkv, d), device="cuda").to(torch.bfloat16) for _ in range(2))
    la.kv4_append(cache, k, v, R.starts(lens), ints(lens), table)
    kr, vr = la.kv4_read(cache, R.starts(lens), ints(lens), table, 90, d)
    gone = torch.zeros(90, dtype=torch.bool)
    gone[16:32] = gone[50 + 32: 90] = True
    for x, y in ((k, kr), (v, vr)):
        want = quantised(x.double().cpu().numpy())
        want[gone.numpy()] = 0
        np.testing.assert_array_equal(y.double().cpu().numpy(), want)
    # the attention sees rows of zeros there
    for lq in ([1, 1], [9, 3], [50, 40]):
        q = torch.randn((sum(lq), 4, d), device="cuda").to(torch.bfloat16)
        o, lse = la.kv4_attn(q, cache, R.starts(lq), ints(lens), table, max(lq), want_lse=True)
        want = R.attention(q, lambda s, h: (kr[50 * s: 50 * s + lens[s], h // 2], vr[50 * s: 50 * s + lens[s], h // 2]),
                           lq, lens, True)
        R.check(o, lse, want, f"missing pages, queries {lq}")
    # a table that ends before the sequence does: it ends there
    short = table[:, :1].contiguous()
    q = torch.randn((2, 4, d), device="cuda").to(torch.bfloat16)
    o = la.kv4_attn(q, cache, R.starts([1, 1]), ints(lens), short, 1)
    want = R.attention(q, lambda s, h: (kr[50 * s: 50 * s + 16, h // 2], vr[50 * s: 50 * s + 16, h // 2]), [1, 1],
                       [16, 16], True)
    R.check(o, None, want, "short table")


ATTN = [
    # (queries, lengths, Hq, Hkv, d, page, causal)
    ([1], [1], 1, 1, 128, 16, True),
    ([1], [1], 2, 1, 64, 64, True),
    ([1, 1, 1, 1], [0, 63, 64, 65], 4, 2, 128, 64, True),
    ([1, 1], [1000, 3], 16, 2, 128, 16, True),
    ([1, 1], [1000, 3], 16, 2, 64, 32, True),
    ([1], [20000], 8, 1, 128, 128, True),                      # one long sequence, split
    ([1], [9000], 3, 3, 64, 1024, True),
    ([1] * 40, list(range(0, 400, 10)), 5, 1, 128, 16, True),
    ([1] * 40, list(range(0, 400, 10)), 24, 1, 64, 16, True),  # a group of more heads than 16 rows
    ([1, 1], [300, 500], 100, 1, 128, 64, True),               # and than 64
    ([4, 2, 0, 3], [200, 1, 50, 130], 6, 2, 128, 32, True),    # a few queries, one sequence shorter than they are
    ([16, 1, 5], [16, 77, 1000], 4, 1, 64, 16, True),
    ([7, 9], [700, 100], 8, 8, 128, 64, False),
    ([60, 3], [400, 90], 2, 2, 128, 16, True),                 # both kinds of sequences
    ([70, 1, 0, 200], [100, 900, 10, 150], 4, 2, 128, 64, True),
    ([70, 1, 0, 200], [100, 900, 10, 250], 4, 2, 64, 16, True),
    ([300], [1500], 6, 3, 128, 128, False),
    ([300, 5], [10, 600], 14, 2, 64, 32, True),
    ([1000], [1000], 2, 1, 128, 16, True),
]


@pytest.mark.parametrize("case", ATTN, ids=[str(i) for i in range(len(ATTN))])
def test_attention(case):
    lq, lens, Hq, Hkv, d, page, causal = case
    print(f"[kv4 attn] {str(lq)[:50]} over {str(lens)[:50]} Hq {Hq} Hkv {Hkv} d {d} page {page}", flush=True)
    cache, table, L, k, v = filled(lens, Hkv, d, page, 4)
    g = torch.Generator(device="cuda").manual_seed(5)
    q = (torch.randn((sum(lq) + 2, Hq, d), generator=g, device="cuda") * 1.5).to(torch.bfloat16)
    cu = R.starts(lq)
    out, lse = torch.full_like(q, 7.0), torch.full((sum(lq) + 2, Hq), 7.0, device="cuda")
    la.kv4_attn(q, cache, cu, L, table, max(lq), causal=causal, out=out, lse_out=lse)
    n, at, G = sum(lq), [sum(lens[:s]) for s in range(len(lens))], Hq // Hkv
    want = R.attention(q[:n], lambda s, h: (k[at[s]: at[s] + lens[s], h // G], v[at[s]: at[s] + lens[s], h // G]), lq,
                       lens, causal)
    R.check(out[:n], lse[:n], want, str(case)[:80])
    assert bool((out[n:] == 7).all()) and bool((lse[n:] == 7).all())
    again, lse2 = la.kv4_attn(q, cache, cu, L, table, max(lq), causal=causal, want_lse=True)
    assert torch.equal(out[:n], again[:n]) and torch.equal(lse[:n], lse2[:n])


def test_both_kernels_agree_with_the_prompt():
    # attention over the values that the cache stands for, as bf16 rows
    for lq, lens in (([1, 1, 1], [100, 513, 64]), ([90, 33, 200], [100, 513, 200])):
        cache, table, L, k, v = filled(lens, 2, 128, 32, 6)
        q = torch.randn((sum(lq), 8, 128), device="cuda").to(torch.bfloat16)
        a, la_ = la.kv4_attn(q, cache, R.starts(lq), L, table, max(lq), want_lse=True)
        b, lb = la.prompt_attn(q, k, v, R.starts(lq), R.starts(lens), want_lse=True)
        assert float((a.double() - b.double()).abs().max()) <= 2 * R.U * 4 and torch.allclose(la_, lb, atol=1e-4)


def test_max_q_leaves_longer_sequences_out():
    cache, table, L, k, v = filled([100, 200], 2, 64, 16, 7)
    q = torch.randn((9, 4, 64), device="cuda").to(torch.bfloat16)
    out = torch.full_like(q, 7.0)
    la.kv4_attn(q, cache, R.starts([2, 7]), L, table, 3, out=out)
    full = la.kv4_attn(q, cache, R.starts([2, 7]), L, table, 7)
    assert bool((out[2:] == 7).all())
    assert float((out[:2].double() - full[:2].double()).abs().max()) <= 2 * R.U * 4


def test_graph():
    lens = [700, 64, 1]
    cache, table, L, k, v = filled(lens, 2, 128, 64, 8)
    q = torch.randn((3, 8, 128), device="cuda").to(torch.bfloat16)
    nk, nv = (torch.randn((3, 2, 128), device="cuda").to(torch.bfloat16) for _ in range(2))
    cu, out = R.starts([1, 1, 1]), torch.empty_like(q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        la.kv4_append(cache, nk, nv, cu, L, table)
        la.kv4_attn(q, cache, cu, L, table, 1, out=out)
    for r in range(4):
        nk.normal_(), nv.normal_(), out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        la.kv4_append(cache, nk, nv, cu, L, table)
        assert torch.equal(la.kv4_attn(q, cache, cu, L, table, 1), got), r


def test_far_pages():
    # a cache of more than 4 GiB: the last pages are past 32 bits of bytes
    d, page, Hkv = 128, 1024, 8
    nbytes = page * (d + d // 16)
    n = (5 << 30) // (Hkv * nbytes)
    cache = torch.empty((n, Hkv, nbytes), dtype=torch.uint8, device="cuda")
    cache[-3:] = 0xFF
    lens = [2500, 100]
    table = torch.tensor([[n - 1, n - 2, 0], [n - 3, -1, -1]], dtype=torch.int32, device="cuda")
    k, v = (torch.randn((2600, Hkv, d), device="cuda").to(torch.bfloat16) for _ in range(2))
    la.kv4_append(cache, k, v, R.starts(lens), ints(lens), table)
    kr, vr = la.kv4_read(cache, R.starts(lens), ints(lens), table, 2600, d)
    np.testing.assert_array_equal(kr.double().cpu().numpy(), quantised(k.double().cpu().numpy()))
    for lq in ([1, 1], [80, 100]):
        q = torch.randn((sum(lq), Hkv, d), device="cuda").to(torch.bfloat16)
        o = la.kv4_attn(q, cache, R.starts(lq), ints(lens), table, max(lq))
        want = R.attention(q, lambda s, h: (kr[2500 * s: 2500 * s + lens[s], h], vr[2500 * s: 2500 * s + lens[s], h]), lq,
                           lens, True)
        R.check(o, None, want, f"far pages, queries {lq}")


@pytest.mark.parametrize("d", [64, 128])
def test_missing_and_far_pages_with_many_queries(d):
    # as above, with enough query rows for the kernel that converts tiles on their way to LDS
    page, Hkv = 16, 2
    lens = [50, 40]
    table = torch.tensor([[3, -1, 1, 2, 7], [0, 4, 1000000, -5, 2]], dtype=torch.int32, device="cuda")
    cache = la.kv4_cache(5, Hkv, d, page)
    cache.fill_(0xFF)
    k, v = (torch.randn((90, Hkv, d), device="cuda").to(torch.bfloat16) for _ in range(2))
    la.kv4_append(cache, k, v, R.starts(lens), ints(lens), table)
    kr, vr = la.kv4_read(cache, R.starts(lens), ints(lens), table, 90, d)
    lq = [230, 300]
    q = torch.randn((sum(lq), 4, d), device="cuda").to(torch.bfloat16)
    for causal in (False, True):
        o, lse = la.kv4_attn(q, cache, R.starts(lq), ints(lens), table, max(lq), causal=causal, want_lse=True)
        want = R.attention(q, lambda s, h: (kr[50 * s: 50 * s + lens[s], h // 2], vr[50 * s: 50 * s + lens[s], h // 2]),
                           lq, lens, causal)
        R.check(o, lse, want, f"missing pages, many queries, causal {causal}")
    # past 32 bits of bytes
    nbytes = 1024 * (d + d // 16)
    n = (5 << 30) // (Hkv * nbytes)
    cache = torch.empty((n, Hkv, nbytes), dtype=torch.uint8, device="cuda")
    cache[-3:] = 0xFF
    lens = [2500, 100]
    table = torch.tensor([[n - 1, n - 2, n - 3], [5, -1, -1]], dtype=torch.int32, device="cuda")
    k, v = (torch.randn((2600, Hkv, d), device="cuda").to(torch.bfloat16) for _ in range(2))
    la.kv4_append(cache, k, v, R.starts(lens), ints(lens), table)
    kr, vr = la.kv4_read(cache, R.starts(lens), ints(lens), table, 2600, d)
    lq = [400, 40]
    q = torch.randn((sum(lq), Hkv, d), device="cuda").to(torch.bfloat16)
    o = la.kv4_attn(q, cache, R.starts(lq), ints(lens), table, max(lq))
    want = R.attention(q, lambda s, h: (kr[2500 * s: 2500 * s + lens[s], h], vr[2500 * s: 2500 * s + lens[s], h]), lq, lens,
                       True)
    R.check(o, None, want, "far pages, many queries")


def test_values_that_are_not_finite():
    # a block with such a value reads as NaN, and reaches the queries that see it and no others
    lens, d, page = [100, 100], 128, 16
    cache, table, L, _, _ = filled(lens, 1, d, page, 9, fill=0x00)
    k, v = (torch.randn((2, 1, d), device="cuda").to(torch.bfloat16) for _ in range(2))
    v[1, 0, 40] = float("inf")
    la.kv4_append(cache, k, v, R.starts([0, 2]), L, table)              # the last tokens of sequence 1
    kr, vr = la.kv4_read(cache, R.starts([0, 2]), L, table, 2, d)
    assert bool(torch.isnan(vr[1, 0, 32:64]).all()) and bool(torch.isfinite(vr[1, 0, :32]).all())
    assert bool(torch.isfinite(kr).all()) and bool(torch.isfinite(vr[0]).all())
    q = torch.randn((2, 4, d), device="cuda").to(torch.bfloat16)
    o = la.kv4_attn(q, cache, R.starts([1, 1]), L, table, 1)
    assert bool(torch.isfinite(o[0]).all()) and bool(torch.isnan(o[1, :, 32:64]).all())
    assert bool(torch.isfinite(o[1, :, :32]).all()) and bool(torch.isfinite(o[1, :, 64:]).all())
    short = L - torch.tensor([0, 1], dtype=torch.int32, device="cuda")  # the token is behind the end now
    assert bool(torch.isfinite(la.kv4_attn(q, cache, R.starts([1, 1]), short, table, 1)).all())


def test_random_caches():
    gen = torch.Generator().manual_seed(7)
    for n in range(24):
        S = int(torch.randint(1, 7, (1,), generator=gen))
        page = [16, 32, 64, 256][n % 4]
        most = [1, 3, 20, 300][n % 4 if n < 16 else (n + 1) % 4]
        lq = torch.randint(0, most + 1, (S,), generator=gen).tolist()
        lens = torch.randint(0, 1500, (S,), generator=gen).tolist()
        Hkv, G, d, causal = [1, 2, 3][n % 3], [1, 2, 4, 5, 20][n % 5], [64, 128][n % 2], n % 4 != 2
        print(f"[kv4] random {n}: {lq} over {lens} G {G} Hkv {Hkv} d {d} page {page}", flush=True)
        cache, table, L, k, v = filled(lens, Hkv, d, page, 50 + n)
        q = (torch.randn((sum(lq), G * Hkv, d), device="cuda") * 1.5).to(torch.bfloat16)
        o, lse = la.kv4_attn(q, cache, R.starts(lq), L, table, max(lq), causal=causal, want_lse=True)
        at = [sum(lens[:s]) for s in range(S)]
        want = R.attention(q, lambda s, h: (k[at[s]: at[s] + lens[s], h // G], v[at[s]: at[s] + lens[s], h // G]), lq, lens,
                           causal)
        R.check(o, lse, want, f"random {n}")


@pytest.mark.parametrize("lq", [1, 2, 70])
@pytest.mark.parametrize("d", [64, 128])
def test_narrow_and_wide_tables(lq, d):
    # tables of up to 1024 tokens (512 for many queries) leave no work to be joined, wider ones may; a wider
    # table alone changes no result beyond the roundings of both ways
    lens = [1024, 1, 64, 500, 0, 1000] * (12 if lq < 3 else 2)
    cache, table, L, k, v = filled(lens, 2, d, 64, 9)
    S, n = len(lens), lq * len(lens)
    table = table[:, :16].contiguous()
    q = (torch.randn((n, 8, d), device="cuda") * 1.5).to(torch.bfloat16)
    cu, at = R.starts([lq] * S), [sum(lens[:s]) for s in range(S)]
    want = R.attention(q, lambda s, h: (k[at[s]: at[s] + lens[s], h // 4], v[at[s]: at[s] + lens[s], h // 4]), [lq] * S,
                       lens, True)
    for more in (0, 1, 300):
        t = torch.cat([table, torch.full((S, more), -1, dtype=torch.int32, device="cuda")], 1).contiguous()
        o, lse = la.kv4_attn(q, cache, cu, L, t, lq, want_lse=True)
        R.check(o, lse, want, f"{more} more columns")
    # a table of 512 tokens: what lies behind them is not seen
    short = table[:, :8].contiguous()
    lens = [min(x, 512) for x in lens]
    want = R.attention(q, lambda s, h: (k[at[s]: at[s] + lens[s], h // 4], v[at[s]: at[s] + lens[s], h // 4]), [lq] * S,
                       lens, True)
    o, lse = la.kv4_attn(q, cache, cu, L, short, lq, want_lse=True)
    R.check(o, lse, want, "512 tokens")


@pytest.mark.parametrize("lq", [1, 200])
def test_longest_table(lq):
    # a table of 2^31 tokens, all of its pages missing, and a length of 2^31 - 1: the sequence ends at
    # 2^31 - 4096, every value reads as zero and every weight is one
    cache = la.kv4_cache(1, 1, 64, 1024)
    cache.fill_(0x22)
    table = torch.full((2, 1 << 21), -1, dtype=torch.int32, device="cuda")
    q = torch.randn((1 + lq, 1, 64), device="cuda").to(torch.bfloat16)
    print(f"[kv4] 2^31 tokens, {lq} queries", flush=True)
    o, lse = la.kv4_attn(q, cache, R.starts([1, lq]), ints([5, (1 << 31) - 1]), table, lq, want_lse=True)
    torch.cuda.synchronize()
    assert bool((o == 0).all())
    seen = torch.tensor([5.0] + [2.0 ** 31 - 4096 - (lq - 1 - i) for i in range(lq)], dtype=torch.float64)
    # a lane counts fewer than 2^24 weights, so exactly; up to 512 counts are joined, 2^-24 each, and the
    # logarithm near 31 (21.5 in the end) is rounded by 2^-20 twice
    assert float((lse[:, 0].double().cpu() - seen.log()).abs().max()) < 512 * 2.0 ** -24 + 4 * 2.0 ** -20


def test_any_large_max_q():
    cache, table, L, k, v = filled([100, 200], 2, 64, 16, 10)
    q = torch.randn((9, 4, 64), device="cuda").to(torch.bfloat16)
    want = la.kv4_attn(q, cache, R.starts([2, 7]), L, table, 9)
    for most in (10, 1 << 31, 1 << 32, (1 << 63) - 1):
        assert torch.equal(la.kv4_attn(q, cache, R.starts([2, 7]), L, table, most), want), most
