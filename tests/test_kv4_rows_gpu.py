"""The tests of the attention over a 4-bit cache once more, with tables so wide that sequences of many
queries are left to the kernel that converts tiles on their way to LDS (with few products in all, the
kernel for few queries takes them too)."""
import pytest
import torch

from paper_2605_31158_amd import la
from test_kv4_gpu import (test_attention, test_both_kernels_agree_with_the_prompt, test_far_pages,  # noqa: F401
                          test_max_q_leaves_longer_sequences_out, test_missing_and_far_pages_with_many_queries,
                          test_random_caches)

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def wide_tables(monkeypatch):
    attn = la.kv4_attn

    def call(q, cache, cu_q, lens, table, max_q, **kw):
        d = q.shape[2]
        page, Tq, Hq = cache.shape[2] // (d + d // 16), q.shape[0], q.shape[1]
        if min(max_q, Tq) * (Hq // cache.shape[1]) > 192:
            more = torch.full((len(table), -(-10 ** 8 // (Tq * Hq * page))), -1, dtype=torch.int32, device="cuda")
            table = torch.cat([table, more], 1).contiguous()
        return attn(q, cache, cu_q, lens, table, max_q, **kw)

    monkeypatch.setattr(la, "kv4_attn", call)
