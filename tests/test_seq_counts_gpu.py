"""Numbers past 31 bits that a tensor's shape can hold, which the C structs cannot: refused, not wrapped; and
heads of no values."""
import pytest
import torch

from paper_2605_31158_amd import la

pytestmark = pytest.mark.gpu
FAR = 1 << 32


def ints(*shape):
    return torch.empty(shape, dtype=torch.int32, device="cuda")


def test_heads():
    q, k = (torch.zeros((3, 1, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cu = torch.tensor([0, 3], dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        la.prompt_attn(q, k.expand(3, FAR + 1, 64), k.expand(3, FAR + 1, 64), cu)


def test_sequences():
    q = torch.zeros((3, 1, 64), dtype=torch.bfloat16, device="cuda")
    cu = ints(FAR + 2)                                   # 17 GB, not read
    with pytest.raises(ValueError):
        la.prompt_attn(q, q, q, cu)
    cache = la.kv4_cache(1, 1, 64, 16)
    lens, table = cu[: FAR + 1], cu[: FAR + 1].view(FAR + 1, 1)
    with pytest.raises(ValueError):
        la.kv4_append(cache, q, q, cu, lens, table)
    with pytest.raises(ValueError):
        la.kv4_read(cache, cu, lens, table, 3, 64)
    with pytest.raises(ValueError):
        la.kv4_attn(q, cache, cu, lens, table, 1)


def test_pages():
    q = torch.zeros((3, 1, 64), dtype=torch.bfloat16, device="cuda")
    cache = la.kv4_cache(1, 1, 64, 16)
    cu, lens, table = ints(2), ints(1), ints(1, FAR + 5)
    with pytest.raises(ValueError):
        la.kv4_append(cache, q, q, cu, lens, table)
    with pytest.raises(ValueError):
        la.kv4_attn(q, cache, cu, lens, table, 3)


def test_negative_max_q():
    q = torch.zeros((3, 1, 64), dtype=torch.bfloat16, device="cuda")
    cache = la.kv4_cache(1, 1, 64, 16)
    cu, lens, table = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((2,), (1,), (1, 1)))
    for most in (-1, -FAR + 5, -FAR):
        with pytest.raises(la.LaError):
            la.kv4_attn(q, cache, cu, lens, table, most)


def test_heads_of_no_values():
    q = torch.zeros((3, 1, 0), dtype=torch.bfloat16, device="cuda")
    cache = la.kv4_cache(1, 1, 64, 16)
    cu, lens, table = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((2,), (1,), (1, 1)))
    with pytest.raises(ValueError):
        la.kv4_attn(q, cache, cu, lens, table, 1)
    with pytest.raises(ValueError):
        la.kv4_append(cache, q, q, cu, lens, table)
    for d in (0, -64, -1):
        with pytest.raises(ValueError):
            la.kv4_read(cache, cu, lens, table, 3, d)
    with pytest.raises(la.LaError):
        la.prompt_attn(q, q, q, cu)
    with pytest.raises(la.LaError):
        la.rope(q, cu.new_zeros(3), la.rope_frequencies(64))
