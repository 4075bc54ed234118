"""Paged cache calls of more rows or sequences than one launch has threads for."""
import pytest
import torch

from paper_2608_14498_amd.runtime import PagedKV

pytestmark = pytest.mark.gpu


def numbered(n, start=0):
    """[1, n, 1, 8] rows of 16 bytes that hold their number (as four int32)."""
    return torch.arange(start, start + n, dtype=torch.int32, device="cuda").repeat_interleave(4).view(torch.bfloat16).view(1, n, 1, 8)


def test_append_of_more_rows_than_waves_of_one_launch():
    """2^26 rows and some at a wave a row: 2^32 threads."""
    first, second = (1 << 26) - 700, 711
    n = first + second
    c = PagedKV.empty(1, (n + 1023) // 1024 + 2, 1024, 1, 8, 2, (first + 1023) // 1024, dtype=torch.bfloat16)
    k, v = numbered(n), numbered(n, 1 << 27)
    print(f"[pages] append of {n} rows", flush=True)
    assert c.append([1, 0], [0, first, n], k, v).tolist() == [0, 0]
    assert c.length.tolist() == [second, first]
    assert int(c.refs.sum()) == (first + 1023) // 1024 + 1
    slots = lambda pool, b, m: pool.view(-1, 1024, 8)[c.table[b, :(m + 1023) // 1024].long()].view(-1, 8)[:m].view(torch.int32)
    for pool, rows in ((c.k, k), (c.v, v)):
        rows = rows.view(n, 8).view(torch.int32)
        assert torch.equal(slots(pool, 1, first), rows[:first])
        assert torch.equal(slots(pool, 0, second), rows[first:])


def test_compaction_of_a_pool_of_more_sequences_than_waves_of_one_launch():
    """2^26 sequences and some, all but a few empty, the last ones in pages that move."""
    n = (1 << 26) + 9
    c = PagedKV.empty(1, 12, 8, 1, 8, n, 1, dtype=torch.bfloat16)
    c.k.copy_(numbered(96).view(1, 12, 8, 1, 8))
    c.v.copy_(numbered(96, 1000).view(1, 12, 8, 1, 8))
    held = {0: 11, 1 << 18: 2, (1 << 26) - 1: 10, n - 1: 8}
    for b, page in held.items():
        c.table[b, 0], c.length[b] = page, 5
        c.refs[page] = 1
    print(f"[pages] compaction of {n} sequences", flush=True)
    assert c.compact().item() == 4
    assert c.refs.tolist() == [1] * 4 + [0] * 8
    now = {2: 2, 8: 0, 10: 1, 11: 3}
    for b, page in held.items():
        assert c.table[b, 0].item() == now[page]
        for pool, first in ((c.k, 0), (c.v, 1000)):
            assert torch.equal(pool[0, now[page], :5], numbered(96, first).view(12, 8, 1, 8)[page, :5])
    assert int((c.table >= 0).sum()) == 4
