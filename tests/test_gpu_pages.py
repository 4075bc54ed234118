"""Paged cache on the GPU against its rules in Python (pages_model.py): tables, lengths, reference
counts, missing and every slot's bits, over random sequences of calls and at the edges."""
import random

import pytest
import torch

from paper_2608_14498_amd.runtime import PagedKV
from tests.pages_model import PoolModel, walk

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


class Both:
    """A pool on the GPU beside its model.  Token x's key in layer l is the number x + l / 4 in every
    element (v: its negative), rounded to the type."""

    def __init__(self, dtype, n_pages, page, n_seqs, table_ld, L=2, H=2, D=64):
        self.gpu = PagedKV.empty(L, n_pages, page, H, D, n_seqs, table_ld, dtype=TYPES[dtype])
        self.gpu.k.fill_(-1)
        self.gpu.v.fill_(1)
        self.model = PoolModel(n_pages, page, n_seqs, table_ld)
        self.L, self.H, self.D = L, H, D

    def rows(self, values):
        t = torch.tensor(values, dtype=torch.float64).view(1, -1, 1, 1).expand(self.L, -1, self.H, self.D)
        t = (t + torch.arange(self.L).view(-1, 1, 1, 1) / 4).to(self.gpu.k.dtype).contiguous().cuda()
        return t, -t

    def append(self, items):
        cu = [0]
        for _, v in items:
            cu.append(cu[-1] + len(v))
        k, v = self.rows([x for _, vs in items for x in vs])
        return self.gpu.append([b for b, _ in items], cu, k, v).tolist(), self.model.append(items)

    def check(self):
        g, m = self.gpu, self.model
        assert g.length.tolist() == m.len
        assert g.refs.tolist() == m.refs
        table = g.table.tolist()
        for b, row in enumerate(m.table):
            assert table[b][:len(row)] == row, b
        want = torch.tensor(m.slots).view(1, *m.slots.shape, 1, 1)
        used = want >= 0
        want = torch.where(used, want + torch.arange(self.L).view(-1, 1, 1, 1, 1) / 4, want).expand_as(g.k.cpu())
        # slots behind a sequence's end may hold what a moved page held: compare those that hold a token
        hold = torch.zeros(m.slots.shape, dtype=torch.bool)
        for b, row in enumerate(m.table):
            for t in range(m.len[b]):
                hold[row[t // m.page], t % m.page] = True
        want = want.to(g.k.dtype)  # (as rows() rounded them: 64.25 needs nine bits, bf16 has eight)
        assert torch.equal(g.k.cpu().double()[:, hold], want.double()[:, hold])
        assert torch.equal(g.v.cpu().double()[:, hold], -want.double()[:, hold])


@pytest.mark.parametrize("dtype,page,n_pages,H,D", [("bf16", 8, 48, 2, 64), ("f16", 16, 24, 4, 128), ("f32", 64, 30, 1, 64), ("bf16", 8, 700, 5, 8)])
def test_random_calls(dtype, page, n_pages, H, D):
    rng = random.Random(page * n_pages)
    both = Both(dtype, n_pages, page, 9, 7, H=H, D=D)
    for step in range(60):
        op = rng.choice(["append", "append", "append", "fork", "free", "compact"])
        if op == "append":
            items = [(b, [rng.randrange(64) for _ in range(rng.choice([0, 1, 2, page - 1, page, page + 1, 3 * page]))])
                     for b in rng.sample(range(9), rng.randint(1, 5))]
            got, want = both.append(items)
        elif op == "fork":
            seqs = rng.sample(range(9), 6)
            src, dst = [rng.choice(seqs[:2]) for _ in range(4)], seqs[2:]
            got, want = both.gpu.fork(src, dst).tolist(), both.model.fork(src, dst)
        elif op == "free":
            seqs = rng.sample(range(9), rng.randint(1, 3))
            got = want = None
            both.gpu.free(seqs)
            both.model.free(seqs)
        else:
            got, want = both.gpu.compact().tolist(), [both.model.compact()]
        print(f"[pages] {dtype} page {page} step {step} {op}", flush=True)
        assert got == want
        both.check()


def test_pages_run_out_in_list_order_and_tables_overflow():
    both = Both("f32", 5, 8, 4, 3)
    got, want = both.append([(0, [1] * 16), (1, [2] * 25), (2, [3] * 17), (3, [4] * 8)])
    # 1: more than three pages; 2: its three pages are two and a bit too many for the pool with 0's two; 3 behind it
    assert got == want == [0, -1, 0, 1]
    both.check()
    got, want = both.append([(3, []), (0, [5]), (2, [6] * 7)])  # no page left, 2 fits its last page
    assert got == want == [0, 1, 0]
    both.check()
    assert both.gpu.fork([2, 0], [1, 3]).tolist() == both.model.fork([2, 0], [1, 3]) == [0, 0]  # whole pages: no page needed
    both.check()
    both.gpu.free([0])
    both.model.free([0])
    got, want = both.append([(1, [7])])  # sequence 1 is full up to its table
    assert got == want == [-1]
    both.check()


def test_fork_without_a_page_leaves_the_child_empty():
    both = Both("f32", 4, 8, 5, 3)
    both.append([(0, list(range(20)))])
    assert both.gpu.fork([0, 0], [1, 2]).tolist() == both.model.fork([0, 0], [1, 2]) == [0, 1]
    both.check()
    assert both.gpu.length.tolist() == [20, 20, 0, 0, 0]
    assert both.gpu.fork([0], [1]).tolist() == both.model.fork([0], [1]) == [0]  # its old page is free again first
    both.check()


@pytest.mark.parametrize("n_pages,rows", [(6000, 5003), (9000, 2048), (9000, 2049)])
def test_thousands_of_pages_in_one_call(n_pages, rows):
    """More pages than the plan lists in one search, taken and refused."""
    both = Both("bf16", n_pages, 8, 3, n_pages, L=1, H=1, D=8)
    both.append([(2, [9] * 8 * 37)])
    both.gpu.free([2])
    both.model.free([2])
    both.append([(0, [1] * 9)])
    got, want = both.append([(1, [x % 64 for x in range(rows * 8)]), (2, [3] * (n_pages - rows) * 8)])
    assert got == want
    both.check()
    n = both.gpu.compact().tolist()
    assert n == [both.model.compact()]
    both.check()


def test_device_values_out_of_range_stay_inside_the_pool():
    c = PagedKV.empty(1, 6, 8, 1, 64, 4, 3, dtype=torch.float32)
    c.k.zero_()
    c.v.zero_()
    c.table.copy_(torch.tensor([[-7, 1 << 30, 2], [0, 1, -1], [99, 98, 97], [-1, -1, -1]], dtype=torch.int32))
    c.length.copy_(torch.tensor([1 << 30, -5, 24, 0], dtype=torch.int32))
    k = torch.ones(1, 4, 1, 64, device="cuda")
    assert c.append([0, 1], [0, 2, 4], k, k).tolist() == [-1, 0]  # a clamped length is a full table; a negative one is 0
    c.fork([0, 2], [1, 3])
    c.free([0, 2])
    c.compact()
    torch.cuda.synchronize()
    assert c.length.tolist()[0] == 0


@pytest.mark.parametrize("dtype,N,B", [("f32", 7, 5), ("bf16", 16, 12), ("f16", 64, 3), ("bf16", 130, 2), ("f32", 1, 4), ("bf16", 256, 1)])
def test_commit(dtype, N, B):
    rng = random.Random(N)
    both = Both(dtype, 200, 8, B + 1, 40)
    both.append([(b, [b] * rng.randint(0, 20)) for b in range(B)])
    for step in range(4):
        parents = [[-1] + [rng.randint(max(0, i - 4), i - 1) for i in range(1, N)] for _ in range(B)]
        tokens = [[rng.randrange(3) for _ in range(N)] for _ in range(B)]
        chosen = [[rng.randrange(3) for _ in range(N)] for _ in range(B)]
        n = [rng.choice([0, 1, N, rng.randint(0, N)]) for _ in range(B)]
        k, v = both.rows([x % 64 for x in range(B * N)])
        dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        acc, cnt, out, missing = both.gpu.commit(dev(tokens), dev(parents), dev(chosen), k, v, n_nodes=dev(n))
        paths = [walk(tokens[b], parents[b], chosen[b], n[b]) for b in range(B)]
        want = both.model.append([(b, [(b * N + j) % 64 for j in p]) for b, p in enumerate(paths)])
        assert missing.tolist() == want
        for b, p in enumerate(paths):
            if want[b]:
                p = []
            assert acc[b].tolist() == p + [-1] * (N - len(p))
            assert cnt[b].item() == len(p)
            assert out[b].item() == (chosen[b][p[-1]] if p else -1)
        both.check()
        print(f"[commit] {dtype} N {N} step {step} accepted {cnt.tolist()[:8]}", flush=True)


def test_commit_without_room_commits_nothing():
    both = Both("f32", 2, 8, 2, 2)
    both.append([(0, [1] * 8), (1, [2] * 7)])
    k, v = both.rows([1, 2])
    i = torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    acc, cnt, out, missing = both.gpu.commit(i, None, i + 5, k, v)
    assert both.model.append([(0, [1]), (1, [2])]) == missing.tolist() == [1, 0]
    assert acc.tolist() == [[-1], [0]] and cnt.tolist() == [0, 1] and out.tolist() == [-1, 5]
    both.check()


def test_commit_of_many_sequences():
    B = 1500
    both = Both("f32", 4000, 8, B, 3, L=1, H=1, D=8)
    k, v = both.rows([b % 64 for b in range(B)])
    i = torch.zeros(B, 1, dtype=torch.int32, device="cuda")
    for step in range(9):
        assert both.gpu.commit(i, None, i, k, v)[3].tolist() == both.model.append([(b, [b % 64]) for b in range(B)])
    both.check()


def test_calls_in_a_graph():
    """append, fork, commit, free and compact captured once and replayed on restored tables."""
    both = Both("bf16", 40, 8, 6, 6)
    c = both.gpu
    both.append([(0, [1] * 19), (1, [2] * 3)])
    first = [t.clone() for t in (c.table, c.length, c.refs, c.k, c.v)]
    k, v = both.rows([3] * 9)
    dk, dv = both.rows([4] * 6 * 2)
    tok = torch.zeros(6, 2, dtype=torch.int32, device="cuda")
    ints = lambda *s: torch.empty(s, dtype=torch.int32, device="cuda")
    m1, m2, m3, acc, cnt, out, live, ws = ints(1), ints(2), ints(6), ints(6, 2), ints(6), ints(6), ints(1), c.compact_workspace()

    def work():
        c.append([1], [0, 9], k, v, missing=m1)
        c.fork([0, 1], [2, 3], missing=m2)
        c.commit(tok, None, tok, dk, dv, accepted=acc, n_accepted=cnt, token_out=out, missing=m3)
        c.free([0, 4])
        c.compact(n_live=live, workspace=ws)

    work()
    torch.cuda.synchronize()
    state = lambda: [t.clone() for t in (c.table, c.length, c.refs, c.k, c.v, m1, m2, m3, acc, cnt, out, live)]
    want = state()

    def restore():
        for t, x in zip((c.table, c.length, c.refs, c.k, c.v), first):
            t.copy_(x)

    restore()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            work()
    torch.cuda.current_stream().wait_stream(side)
    for rep in range(3):
        restore()
        _ = torch.randn(4096, device="cuda").sum().item()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(state(), want):
            assert torch.equal(x, y), rep


@pytest.mark.parametrize("N,B", [(256, 16), (256, 17), (64, 64), (64, 65)])
def test_commit_at_the_most_nodes_of_one_workgroup(N, B):
    test_commit("bf16", N, B)
