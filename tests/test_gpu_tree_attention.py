"""Attention of drafted trees over pages against float64, element by element.

Bound of an element, from the arithmetic: u = half a step of the type (finfo.eps / 2).  The output
is rounded once (u |o|), a 16-bit type rounds each weight of the value product once (u sum p |v|);
fp32 sums of n terms are off by n 2^-24 of the sum of magnitudes, so a score is off by
e = (D + 8) 2^-24 max sum |q k| scale and a weight by 2 e (numerator and denominator), and the sums
over K keys by 2 K 2^-24 (bounded at 2^-12 for the split and tiled sums of long rows), the
exponential and the merges by 2^-18."""
import math

import pytest
import torch

from paper_2608_14498_amd.runtime import PagedKV

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def make(dtype, lens, N, Hkv, D, page, nodes=None, seed=0, spread=1.0, layers=2, fill=float("nan"), table_ld=None):
    """A pool whose unused slots hold `fill`, with the sequences' pages in random order."""
    g = torch.Generator().manual_seed(seed)
    B = len(lens)
    need = [(n + page - 1) // page for n in lens]
    P = sum(need) + 3
    c = PagedKV.empty(layers, P, page, Hkv, D, B, table_ld or max(max(need), 1), dtype=TYPES[dtype])
    order = torch.randperm(P, generator=g)
    c.k.fill_(fill)
    c.v.fill_(fill)
    table, o = c.table.cpu(), 0
    for b, n in enumerate(need):
        table[b, :n] = order[o:o + n]
        o += n
    c.table.copy_(table)
    c.length.copy_(torch.tensor(lens, dtype=torch.int32))
    draw = lambda *s: (torch.randn(s, generator=g) * spread).to(TYPES[dtype]).cuda()
    K, V = [], []
    for b, n in enumerate(lens):
        K.append(draw(layers, n, Hkv, D))
        V.append(draw(layers, n, Hkv, D))
        for t in range(0, n, page):
            m = min(page, n - t)
            c.k[:, table[b, t // page], :m] = K[b][:, t:t + m]
            c.v[:, table[b, t // page], :m] = V[b][:, t:t + m]
    kn, vn = draw(B, N, Hkv, D), draw(B, N, Hkv, D)
    if nodes is not None:
        for b, n in enumerate(nodes):
            kn[b, n:] = float("nan")
            vn[b, n:] = float("inf")
    return c, K, V, kn, vn, draw, g


def words(sees):
    B, N, _ = sees.shape
    W = (N + 31) // 32
    out = torch.zeros(B, N, W, dtype=torch.int64)
    for j in range(N):
        out[:, :, j // 32] |= sees[:, :, j].long() << (j % 32)
    return torch.where(out >= 1 << 31, out - (1 << 32), out).to(torch.int32).cuda()


def tree(B, N, g, back=5):
    sees = torch.zeros(B, N, N, dtype=torch.bool)
    for b in range(B):
        for i in range(N):
            if i:
                sees[b, i] = sees[b, max(0, i - 1 - int(torch.randint(0, back, (1,), generator=g)))]
            sees[b, i, i] = True
    return sees


def check(dtype, out, q, K, V, kn, vn, lens, sees, nodes, scale, before=None):
    B, N, Hq, D = q.shape
    Hkv = kn.shape[2]
    u = torch.finfo(TYPES[dtype]).eps / 2
    worst = 0.0
    for b in range(B):
        m = N if nodes is None else nodes[b]
        if before is not None:
            assert torch.equal(out[b, m:].view(torch.int32 if dtype == "f32" else torch.int16),
                               before[b, m:].view(torch.int32 if dtype == "f32" else torch.int16)), "padding rows"
        if m == 0:
            continue
        k = torch.cat([K[b], kn[b, :m]]).double().repeat_interleave(Hq // Hkv, 1)  # [keys, Hq, D]
        v = torch.cat([V[b], vn[b, :m]]).double().repeat_interleave(Hq // Hkv, 1)
        qb = q[b, :m].double()
        see = torch.cat([torch.ones(m, lens[b], dtype=torch.bool), sees[b, :m, :m]], 1).cuda()
        v = torch.where(see.any(0)[:, None, None], v, torch.zeros_like(v))
        k = torch.where(see.any(0)[:, None, None], k, torch.zeros_like(k))
        for h in range(Hq):
            s = qb[:, h] @ k[:, h].T.contiguous() * scale
            mag = ((qb[:, h].abs() @ k[:, h].abs().T.contiguous()) * abs(scale)).max().item()
            s = s.masked_fill(~see, -math.inf)
            top = s.amax(1, keepdim=True)
            p = torch.exp(s - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
            total = p.sum(1, keepdim=True)
            p = p / torch.where(total > 0, total, torch.ones_like(total))
            o = p @ v[:, h]
            pv = p @ v[:, h].abs()
            e = (D + 8) * 2.0 ** -24 * mag
            n = min(2 * see.shape[1] * 2.0 ** -24, 2.0 ** -12)
            bound = u * o.abs() + (2 * e + n + 2.0 ** -18 + (u if dtype != "f32" else 0)) * pv + 1e-30
            if dtype == "f16":
                bound = bound + 2.0 ** -25  # half a subnormal step
            got = out[b, :m, h].double()
            assert torch.isfinite(got).all(), (b, h)
            off = ((got - o).abs() / bound).max().item()
            assert off <= 1.0, (b, h, off)
            worst = max(worst, off)
    print(f"[tree] worst error / bound {worst:.3f}", flush=True)


CASES = [
    # dtype, Hq, Hkv, D, page, N, lens
    ("bf16", 28, 4, 128, 64, 1, [4000, 0, 1, 63, 64, 65, 8191]),
    ("bf16", 28, 4, 128, 8, 16, [500, 7, 8, 9, 0, 3001]),
    ("bf16", 40, 8, 128, 128, 64, [1000, 0, 129, 2049]),
    ("f16", 40, 8, 128, 32, 5, [777, 31, 32, 33]),
    ("f16", 8, 8, 64, 16, 33, [100, 0, 15, 2000]),
    ("f16", 5, 1, 64, 8, 31, [1, 5000]),
    ("bf16", 16, 2, 64, 256, 130, [300, 0, 255, 256, 257]),
    ("bf16", 8, 1, 128, 1024, 256, [1023, 1500, 0]),
    ("bf16", 2, 2, 64, 64, 256, [90, 640]),
    ("f32", 4, 2, 64, 16, 7, [577, 0, 1, 100, 31, 32, 33]),
    ("f32", 6, 2, 128, 8, 40, [9, 0, 1030]),
    ("f32", 8, 1, 64, 64, 1, [4097, 3]),
    ("f32", 3, 3, 128, 32, 256, [50, 700]),
]


@pytest.mark.parametrize("dtype,Hq,Hkv,D,page,N,lens", CASES)
@pytest.mark.parametrize("form", ["chain", "tree", "padded"])
def test_against_float64(dtype, Hq, Hkv, D, page, N, lens, form):
    B = len(lens)
    nodes = None if form != "padded" else [[N, max(1, N // 2), 0, 1, N - 1 if N > 1 else 1][b % 5] for b in range(B)]
    c, K, V, kn, vn, draw, g = make(dtype, lens, N, Hkv, D, page, nodes, seed=N + page)
    q = draw(B, N, Hq, D)
    sees = torch.tril(torch.ones(N, N, dtype=torch.bool)).expand(B, N, N) if form == "chain" else tree(B, N, g)
    out = torch.full_like(q, 7.0)
    before = out.clone()
    n_dev = None if nodes is None else torch.tensor(nodes, dtype=torch.int32, device="cuda")
    print(f"[tree] {dtype} {Hq}/{Hkv} heads of {D}, page {page}, N {N}, {form}", flush=True)
    c.tree_attention(1, q, kn, vn, mask=None if form == "chain" else words(sees), n_nodes=n_dev, out=out)
    torch.cuda.synchronize()
    check(dtype, out, q, [k[1] for k in K], [v[1] for v in V], kn, vn, lens, sees, nodes, D ** -0.5, before)


@pytest.mark.parametrize("dtype,Hq,Hkv,D,N", [("bf16", 7, 1, 128, 4), ("bf16", 7, 1, 128, 40), ("f32", 2, 1, 64, 9), ("f16", 8, 2, 64, 20)])
def test_rows_that_see_nothing_and_poisoned_tokens(dtype, Hq, Hkv, D, N):
    """Some rows see no token at all (0), and tokens that only some rows see hold NaN and infinities."""
    lens = [0, 70]
    c, K, V, kn, vn, draw, g = make(dtype, lens, N, Hkv, D, 16, seed=5)
    q = draw(2, N, Hq, D)
    sees = tree(2, N, g)
    sees[0, 1] = False
    sees[0, N - 1] = False
    sees[:, :, 2] = False  # nobody sees token 2
    kn[:, 2], vn[:, 2] = float("nan"), float("nan")
    sees[:, 1:, 0] = False  # token 0 is seen by row 0 alone, whose key and value break it
    kn[:, 0, :, 0], vn[:, 0, :, 1] = float("inf"), float("-inf")
    out = c.tree_attention(0, q, kn, vn, mask=words(sees))
    torch.cuda.synchronize()
    assert not torch.isfinite(out[:, 0].float()).all()
    assert (out[0, 1] == 0).all() and (out[0, N - 1] == 0).all()
    sees[:, 0] = False
    got = out.clone()
    got[:, 0] = 0
    sees[1, 0] = True  # (row 0 of sequence 1: not compared, any finite row will do)
    kn[:, 0], vn[:, 0], kn[:, 2], vn[:, 2] = 0, 0, 0, 0
    want_rows = [i for i in range(N) if i != 0]
    sub = lambda t: t[:, want_rows].contiguous()
    check_sub(dtype, sub(got), sub(q), [k[0] for k in K], [v[0] for v in V], kn, vn, lens, sees[:, want_rows], D ** -0.5)


def check_sub(dtype, out, q, K, V, kn, vn, lens, sees, scale):
    """check() where the rows are fewer than the tokens: the missing rows are filled up with empty ones."""
    B, n, Hq, D = q.shape
    N = kn.shape[1]
    qq = torch.zeros(B, N, Hq, D, dtype=q.dtype, device="cuda")
    oo = torch.zeros_like(qq)
    ss = torch.zeros(B, N, N, dtype=torch.bool)
    qq[:, 1:], oo[:, 1:], ss[:, 1:] = q, out, sees
    for b in range(B):  # row 0 sees the cache alone, with equal scores
        if lens[b]:
            oo[b, 0] = V[b].double().mean(0).repeat_interleave(Hq // kn.shape[2], 0).to(q.dtype)
    check(dtype, oo, qq, K, V, kn, vn, lens, ss, None, scale)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("spread,scale", [(6.0, 1.0), (1e-3, 0.125), (1.0, 0.0), (1.0, -0.3)])
def test_score_ranges(dtype, spread, scale):
    """Peaked rows, flat rows, equal scores, a negative scale."""
    lens = [300, 45]
    c, K, V, kn, vn, draw, g = make(dtype, lens, 6, 2, 128, 32, seed=9, spread=spread)
    q = draw(2, 6, 8, 128)
    sees = tree(2, 6, g)
    out = c.tree_attention(0, q, kn, vn, mask=words(sees), scale=scale)
    torch.cuda.synchronize()
    check(dtype, out, q, [k[0] for k in K], [v[0] for v in V], kn, vn, lens, sees, None, scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_far_below_zero_and_infinite_ones(dtype):
    """A cached key of -inf scores weighs nothing beside others; scores of -2^28 are softmaxed as others."""
    c, K, V, kn, vn, draw, g = make(dtype, [40], 1, 1, 64, 8, seed=2)
    q = torch.zeros(1, 1, 1, 64, dtype=TYPES[dtype], device="cuda")
    q[..., 0] = 2.0 ** 14
    flat = c.k.view(2, -1, 64)
    slots = (c.table[0, :5].long()[:, None] * 8 + torch.arange(8, device="cuda")).view(-1)
    flat[0, slots] = 0
    flat[0, slots, 0] = -2.0 ** 14
    kn.zero_()
    kn[..., 0] = -2.0 ** 14
    kv = torch.zeros(2, 40, 1, 64, dtype=TYPES[dtype], device="cuda")
    kv[0, :, 0, 0] = -2.0 ** 14
    out = c.tree_attention(0, q, kn, vn, scale=1.0)
    want = torch.cat([V[0][0], vn[0]]).double().mean(0)
    assert torch.allclose(out[0, 0].double(), want, atol=2.0 ** -7 if dtype == "bf16" else 1e-5, rtol=0)
    flat[0, slots[::2], 0] = -math.inf
    out = c.tree_attention(0, q, kn, vn, scale=1.0)
    want = torch.cat([V[0][0][1::2], vn[0]]).double().mean(0)
    assert torch.allclose(out[0, 0].double(), want, atol=2.0 ** -7 if dtype == "bf16" else 1e-5, rtol=0)


@pytest.mark.parametrize("dtype,N", [("bf16", 3), ("bf16", 30), ("f32", 3)])
def test_strided_queries_streams_and_batches_of_two_calls(dtype, N):
    lens = [333, 20, 1200]
    c, K, V, kn, vn, draw, g = make(dtype, lens, N, 2, 128, 16, seed=4)
    wide = draw(3 * N, 3 * 14 * 128)  # q beside other columns of one projection
    q = wide[:, 14 * 128:2 * 14 * 128].unflatten(0, (3, N)).unflatten(2, (14, 128))
    sees = tree(3, N, g)
    mask = words(sees)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = [torch.empty(3, N, 14, 128, dtype=q.dtype, device="cuda") for _ in range(2)]
    wss = [c.attention_workspace(3, N, 14) for _ in range(2)]
    for _ in range(5):
        for s, layer in ((s1, 0), (s2, 1)):
            c.tree_attention(layer, q, kn, vn, mask=mask, out=outs[layer], workspace=wss[layer], stream=s)
    torch.cuda.synchronize()
    for layer in range(2):
        check(dtype, outs[layer], q, [k[layer] for k in K], [v[layer] for v in V], kn, vn, lens, sees, None, 128 ** -0.5)


def test_tables_longer_than_the_lengths_and_bad_page_ids():
    lens = [100, 40]
    c, K, V, kn, vn, draw, g = make("bf16", lens, 2, 1, 64, 16, seed=6, table_ld=50, fill=0.0)
    q = draw(2, 2, 4, 64)
    sees = torch.tril(torch.ones(2, 2, dtype=torch.bool)).expand(2, 2, 2)
    check("bf16", c.tree_attention(0, q, kn, vn), q, [k[0] for k in K], [v[0] for v in V], kn, vn, lens, sees, None, 0.125)
    c.table.fill_(1 << 30)  # any page id is brought into the pool
    c.length.copy_(torch.tensor([1 << 30, -4], dtype=torch.int32))
    out = c.tree_attention(0, q, kn, vn)
    torch.cuda.synchronize()
    assert torch.isfinite(out.float()).all()


def test_shared_pages_are_read_by_all_that_hold_them():
    c, K, V, kn, vn, draw, g = make("bf16", [90, 90, 90], 4, 2, 128, 32, seed=8)
    c.table[1:] = c.table[0]
    K, V = [K[0]] * 3, [V[0]] * 3
    q = draw(3, 4, 14, 128)
    sees = tree(3, 4, g)
    out = c.tree_attention(1, q, kn, vn, mask=words(sees))
    check("bf16", out, q, [k[1] for k in K], [v[1] for v in V], kn, vn, [90] * 3, sees, None, 128 ** -0.5)


@pytest.mark.parametrize("B,N", [(700, 1), (300, 3)])
def test_more_sequences_than_threads(B, N):
    lens = [(37 * b) % 90 for b in range(B)]
    nodes = [(b % (N + 1)) if b % 7 else N for b in range(B)]
    c, K, V, kn, vn, draw, g = make("bf16", lens, N, 1, 64, 8, nodes, seed=1, layers=1)
    q = draw(B, N, 8, 64)
    out = torch.zeros_like(q)
    sees = torch.tril(torch.ones(N, N, dtype=torch.bool)).expand(B, N, N)
    c.tree_attention(0, q, kn, vn, n_nodes=torch.tensor(nodes, dtype=torch.int32, device="cuda"), out=out)
    check("bf16", out, q, [k[0] for k in K], [v[0] for v in V], kn, vn, lens, sees, nodes, 0.125, torch.zeros_like(q))


@pytest.mark.parametrize("dtype,N", [("bf16", 2), ("f16", 24), ("f32", 4)])
def test_in_a_graph_with_growing_lengths(dtype, N):
    """Captured once; the lengths on the device grow between replays."""
    lens = [900, 100, 0]
    c, K, V, kn, vn, draw, g = make(dtype, lens, N, 2, 128, 16, seed=12)
    q = draw(3, N, 10, 128)
    out, ws = torch.zeros_like(q), c.attention_workspace(3, N, 10)
    full = c.length.clone()
    c.tree_attention(0, q, kn, vn, out=out, workspace=ws)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            c.tree_attention(0, q, kn, vn, out=out, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    sees = torch.tril(torch.ones(N, N, dtype=torch.bool)).expand(3, N, N)
    for rep, cut in enumerate([0, 333, 0, 870]):
        now = [max(0, n - cut) for n in lens]
        c.length.copy_((full - cut).clamp(min=0))
        _ = torch.randn(4096, device="cuda").sum().item()
        graph.replay()
        torch.cuda.synchronize()
        check(dtype, out, q, [k[0][:n] for k, n in zip(K, now)], [v[0][:n] for v, n in zip(V, now)], kn, vn, now, sees, None, 128 ** -0.5)


@pytest.mark.parametrize("dtype,Hq,N", [("bf16", 2, 1), ("f16", 8, 5), ("bf16", 8, 20), ("f32", 2, 3)])
@pytest.mark.parametrize("scale", [0.125, 0.088, 0.1, 0.3, 2.0])
def test_last_tile_of_infinitely_low_scores(dtype, Hq, N, scale):
    """The only key of the last tile scores -inf for every row: the rest of the softmax stays as it is."""
    c, K, V, kn, vn, draw, g = make(dtype, [65], N, 1, 64, 16, seed=14, layers=1)
    q = draw(1, N, Hq, 64)
    q[..., 0] = 1.0
    c.k.view(-1, 64)[int(c.table[0, 4]) * 16, 0] = -math.inf
    sees = torch.tril(torch.ones(N, N, dtype=torch.bool)).expand(1, N, N)
    out = c.tree_attention(0, q, kn, vn, scale=scale)
    check(dtype, out, q, [K[0][0, :64]], [V[0][0, :64]], kn, vn, [64], sees, None, scale)


@pytest.mark.parametrize("dtype,B,N,Hq,Hkv,D", [("bf16", 70, 20, 8, 1, 64), ("f32", 80, 9, 4, 1, 128), ("f16", 66, 130, 2, 1, 128),
                                                ("bf16", 40, 1, 8, 8, 128), ("f16", 20, 64, 16, 2, 64), ("f32", 64, 2, 8, 8, 64)])
def test_shares_that_end_one_sequence_and_begin_the_next(dtype, B, N, Hq, Hkv, D):
    """More sequences than lanes, or than shares."""
    lens = [(53 * b) % 211 for b in range(B)]
    nodes = [(b % (N + 1)) if b % 5 else N for b in range(B)]
    c, K, V, kn, vn, draw, g = make(dtype, lens, N, Hkv, D, 16, nodes, seed=15, layers=1)
    q = draw(B, N, Hq, D)
    out = torch.full_like(q, 3.0)
    sees = tree(B, N, g)
    c.tree_attention(0, q, kn, vn, mask=words(sees), n_nodes=torch.tensor(nodes, dtype=torch.int32, device="cuda"), out=out)
    check(dtype, out, q, [k[0] for k in K], [v[0] for v in V], kn, vn, lens, sees, nodes, D ** -0.5, torch.full_like(q, 3.0))


def test_drafted_tiles_of_large_trees_side_by_side():
    """Eight drafted tiles a sequence and hardly any cached ones: the stages are filled again and again."""
    lens = [0, 3, 40, 0, 33]
    c, K, V, kn, vn, draw, g = make("bf16", lens, 250, 2, 128, 8, seed=16, layers=1)
    q = draw(5, 250, 14, 128)
    sees = tree(5, 250, g, back=40)
    want = c.tree_attention(0, q, kn, vn, mask=words(sees))
    check("bf16", want, q, [k[0] for k in K], [v[0] for v in V], kn, vn, lens, sees, None, 128 ** -0.5)
    for _ in range(3):
        assert torch.equal(c.tree_attention(0, q, kn, vn, mask=words(sees)), want)


def test_own_workspace_on_another_stream():
    """A call on another stream leaves its workspace to that stream: what is allocated next on this one is elsewhere."""
    c, K, V, kn, vn, draw, g = make("bf16", [4000], 2, 2, 128, 16, seed=17, layers=1)
    q = draw(1, 2, 14, 128)
    sees = torch.tril(torch.ones(2, 2, dtype=torch.bool)).expand(1, 2, 2)
    n = c.attention_workspace(1, 2, 14).numel()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    out = c.tree_attention(0, q, kn, vn, stream=side)
    over = [torch.full((n,), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    check("bf16", out, q, [K[0][0]], [V[0][0]], kn, vn, [4000], sees, None, 128 ** -0.5)
    assert all((t == 0x7F).all() for t in over)


@pytest.mark.parametrize("dtype,Hq,Hkv,D,N,lens", [("f16", 300, 300, 64, 1, [70, 0, 333]), ("bf16", 80, 40, 64, 250, [90, 17]),
                                                   ("f32", 600, 600, 64, 1, [40, 3]), ("bf16", 96, 96, 128, 70, [45, 0, 100])])
def test_more_heads_than_shares(dtype, Hq, Hkv, D, N, lens):
    """One share or a few hold everything."""
    c, K, V, kn, vn, draw, g = make(dtype, lens, N, Hkv, D, 16, seed=18, layers=1)
    q = draw(len(lens), N, Hq, D)
    sees = tree(len(lens), N, g)
    out = c.tree_attention(0, q, kn, vn, mask=words(sees))
    check(dtype, out, q, [k[0] for k in K], [v[0] for v in V], kn, vn, lens, sees, None, D ** -0.5)


@pytest.mark.parametrize("dtype,N,Hq,Hkv", [("bf16", 1, 28, 4), ("bf16", 16, 28, 4), ("f32", 7, 4, 2)])
def test_one_workspace_in_two_graphs(dtype, N, Hq, Hkv):
    """Two captured calls share a workspace and are replayed in turn, with eager calls between them."""
    lens = [[1500, 3, 400], [10, 2900, 0]]
    made = [make(dtype, n, N, Hkv, 128, 32, seed=19 + i, layers=1) for i, n in enumerate(lens)]
    qs = [m[5](3, N, Hq, 128) for m in made]
    ws = made[0][0].attention_workspace(3, N, Hq)
    outs = [torch.zeros_like(q) for q in qs]
    sees = torch.tril(torch.ones(N, N, dtype=torch.bool)).expand(3, N, N)
    call = lambda i: made[i][0].tree_attention(0, qs[i], made[i][3], made[i][4], out=outs[i], workspace=ws)
    want = [call(i).clone() for i in range(2)]
    graphs, side = [torch.cuda.CUDAGraph() for _ in range(2)], torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for i in range(2):
        with torch.cuda.stream(side):
            with torch.cuda.graph(graphs[i], stream=side):
                call(i)
    torch.cuda.current_stream().wait_stream(side)
    for rep in range(3):
        for i in (0, 1, 1, 0):
            outs[i].zero_()
            graphs[i].replay()
            call(1 - i)
            torch.cuda.synchronize()
            assert torch.equal(outs[i], want[i]) and torch.equal(outs[1 - i], want[1 - i]), (rep, i)
    for i in range(2):
        c, K, V, kn, vn = made[i][:5]
        check(dtype, want[i], qs[i], [k[0] for k in K], [v[0] for v in V], kn, vn, lens[i], sees, None, 128 ** -0.5)


@pytest.mark.parametrize("dtype,Hq,Hkv,D,N,lens", [("f32", 2, 1, 64, 2, [8800]), ("bf16", 4, 1, 128, 1, [20000]), ("f32", 2, 1, 64, 1, [30, 9000]),
                                                   ("bf16", 4, 1, 64, 40, [9000])])
def test_one_long_sequence_in_many_shares(dtype, Hq, Hkv, D, N, lens):
    """Up to 64 records a sequence, and more where lengths differ."""
    c, K, V, kn, vn, draw, g = make(dtype, lens, N, Hkv, D, 16, seed=20, layers=1)
    q = draw(len(lens), N, Hq, D)
    sees = tree(len(lens), N, g)
    out = c.tree_attention(0, q, kn, vn, mask=words(sees))
    check(dtype, out, q, [k[0] for k in K], [v[0] for v in V], kn, vn, lens, sees, None, D ** -0.5)
