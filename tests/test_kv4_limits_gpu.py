"""Entering and reading rows of the 4-bit cache with as many sequences as the calls take."""
import pytest
import torch

from paper_2605_31158_amd import la

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("S", [(1 << 30) + 5, (1 << 31) - 4096], ids=["2^30+5", "2^31-4096"])
def test_most_sequences(S):
    # all of them empty but five: the first, two in the middle, the last two
    print(f"[kv4] {S} sequences", flush=True)
    d, page = 64, 16
    new = {0: 2, S // 2: 1, S // 2 + 1: 3, S - 2: 1, S - 1: 2}
    T = sum(new.values())
    cu, lens = torch.zeros(S + 1, dtype=torch.int32, device="cuda"), torch.zeros(S, dtype=torch.int32, device="cuda")
    table = torch.full((S, 1), -1, dtype=torch.int32, device="cuda")
    t = 0
    for page_of, (s, n) in enumerate(new.items()):
        t += n
        cu[s + 1:] = t
        lens[s], table[s, 0] = n + 4, page_of            # behind four tokens that are there already
    cache = la.kv4_cache(len(new), 1, d, page)
    cache.fill_(0xAB)
    # small whole numbers are e2m1 values: they come back as they are
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randint(-4, 5, (T + 2, 1, d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    la.kv4_append(cache, k, v, cu, lens, table)
    out = [torch.full_like(k, 9.0) for _ in range(2)]
    la.kv4_read(cache, cu, lens, table, T + 2, d, out=out)
    torch.cuda.synchronize()
    for x, y in ((k, out[0]), (v, out[1])):
        assert torch.equal(y[:T], x[:T]) and bool((y[T:] == 9).all())
    # each on its own page, at tokens 4 and on, and nowhere else
    t = 0
    for p, n in enumerate(new.values()):
        rows = cache[p, 0, : page * d // 2].view(page, d // 2)
        assert bool((rows[:4] == 0xAB).all()) and bool((rows[4 + n:] == 0xAB).all())
        low = rows[4: 4 + n] & 15
        assert torch.equal(low >= 8, (k[t: t + n, 0, ::2] < 0))      # the sign bit of every second value
        t += n
