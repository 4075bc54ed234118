"""Rollout steps over the paged cache as a program makes them: prefix passes, their K/V into pages, a
group's responses forked from their prompt, drafted trees through the model, the confirmed tokens
committed, sequences freed and the pool compacted in between."""
import os
import random
import subprocess
import sys

import numpy as np
import pytest
import torch

import oracle
from paper_2608_14498_amd import binding as rb
from paper_2608_14498_amd import configs, inputs
from paper_2608_14498_amd.runtime import DeviceModel, PagedKV, to_device

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SMALL = dict(n_layers=2, d_model=384, n_q_heads=6, n_kv_heads=2, head_dim=128, ffn_dim=768, vocab=1000)
MODELS = {"tiny": configs.TINY, "bf16": configs.ModelShape(dtype="bf16", **SMALL), "f16": configs.ModelShape(dtype="f16", **SMALL),
          "f16_d64": configs.ModelShape(2, 256, 4, 2, 64, 704, 2048, "f16")}


def setup(name, prefix, visual, index, max_position=600, page=16, n_pages=64, n_seqs=8, table_ld=24):
    m = MODELS[name]
    w = configs.custom(m, prefix, visual, [1] * len(prefix), index=index)
    hw = inputs.make_weights(w, norm="random", bias=True)
    bt = inputs.make_batch(w)
    dm = DeviceModel(hw, max_position)
    cu = [int(x) for x in bt.cu_prefix]
    vis = to_device(bt.visual, dm.device) if bt.visual.shape[0] else None
    K, V, h = dm.prefix(cu, to_device(bt.token_ids, dm.device), vis)
    c = PagedKV.empty(m.n_layers, n_pages, page, m.n_kv_heads, m.head_dim, n_seqs, table_ld, dtype=dm.dtype)
    c.k.fill_(float("nan"))
    c.v.fill_(float("nan"))
    assert c.append(list(range(len(prefix))), cu, K, V).tolist() == [0] * len(prefix)
    return m, hw, bt, dm, cu, c, K, V, h


def dev(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def path_to(parents, i):
    out = []
    while i >= 0:
        out.append(i)
        i = parents[i] if 0 <= parents[i] < i else -1
    return out[::-1]


@pytest.mark.parametrize("name,bar", [("tiny", 1e-4), ("f16", 2e-2), ("f16_d64", 2e-2), ("bf16", 8 * 2e-2)])
def test_every_node_against_the_oracle(name, bar):
    """Log-probabilities of every node of every tree.  The bars are the framework's: 1e-4 in fp32, 2e-2
    with fp16's 11 bits; bf16 has 3 bits fewer, 8 times fp16's bar."""
    m, hw, bt, dm, cu, c, *_ = setup(name, [70, 33, 5], [40, 0, 0], 301)
    try:
        rng = random.Random(1)
        B, N = 3, 9
        nodes = [9, 4, 7]
        parents = [[-1] + [rng.randint(max(-1, i - 4), i - 1) for i in range(1, N)] for _ in range(B)]
        parents[1][2] = 2  # no parent: a root beside node 0
        tokens = [[rng.randrange(m.vocab) for _ in range(N)] for _ in range(B)]
        logits = torch.empty(B, N, m.vocab, device="cuda")
        nxt, dk, dv = dm.tree_step(c, dev(tokens), parents=dev(parents), n_nodes=dev(nodes), logits=logits)
        torch.cuda.synchronize()
        W = hw.as_f32()
        Ko, Vo, _ = oracle.prefix_forward(W, m, bt.cu_prefix, bt.token_ids, inputs.to_f32(bt.visual))
        worst = 0.0
        for b in range(B):
            n0 = cu[b + 1] - cu[b]
            for i in range(nodes[b]):
                path = path_to(parents[b], i)
                ck = np.zeros((m.n_layers, 1, n0 + len(path), m.n_kv_heads, m.head_dim))
                cv = np.zeros_like(ck)
                ck[:, 0, :n0], cv[:, 0, :n0] = Ko[:, cu[b]:cu[b + 1]], Vo[:, cu[b]:cu[b + 1]]
                for k, j in enumerate(path):
                    lg, _, nk, nv = oracle.decode_step(W, m, ck, cv, [n0 + k], [tokens[b][j]])
                    ck[:, 0, n0 + k], cv[:, 0, n0 + k] = nk[:, 0], nv[:, 0]
                got = torch.log_softmax(logits[b, i].double().cpu(), -1).numpy()
                want = lg[0] - lg[0].max()
                want = want - np.log(np.exp(want).sum())
                worst = max(worst, np.abs(got - want).max())
                assert nxt[b, i].item() == logits[b, i].argmax().item()
        print(f"[tree step] {name}: max |d log-prob| {worst:.3g} (bar {bar:g})", flush=True)
        assert worst <= bar
    finally:
        dm.close()


@pytest.mark.parametrize("name", ["tiny", "f16", "bf16"])
def test_chain_equals_the_suffix_pass_after_mrope_prompts(name):
    """A chain of drafted tokens scores as the suffix pass does, rotary positions from pos0 on."""
    m = MODELS[name]
    w = configs.custom(m, [60, 20], [48, 0], [12, 12], index=302)
    hw = inputs.make_weights(w, norm="random", bias=True)
    bt = inputs.make_batch(w)
    dm = DeviceModel(hw, 200)
    try:
        half = m.head_dim // 2
        pos = np.stack([np.concatenate([np.arange(48) // 16 * 2, np.arange(12) + 20, np.arange(20)]),
                        np.concatenate([np.arange(48) // 4 % 4, np.arange(12) + 20, np.arange(20)]),
                        np.concatenate([np.arange(48) % 4, np.arange(12) + 20, np.arange(20)])]).astype(np.int32)
        cp, cs = [0, 60, 80], [0, 12, 24]
        K, V, h = dm.prefix(cp, to_device(bt.token_ids, dm.device), to_device(bt.visual, dm.device), positions=to_device(pos, dm.device),
                            mrope_section=[half // 4, half * 3 // 8, half * 3 // 8])
        resp = to_device(bt.response_ids, dm.device)
        want = dm.suffix_grouped(cp, [0, 1], cs, K, V, h, resp, rope_pos0=[32, 20])
        c = PagedKV.empty(m.n_layers, 24, 8, m.n_kv_heads, m.head_dim, 2, 12, dtype=dm.dtype)
        c.append([0, 1], cp, K, V)
        logits = torch.empty(2, 12, m.vocab, device="cuda")
        dm.tree_step(c, resp.view(2, 12), pos0=dev([32, 20]), logits=logits)
        lp = torch.log_softmax(logits, -1)[:, :-1].gather(2, resp.view(2, 12)[:, 1:, None].long())[..., 0]
        d = (lp - want.view(2, 12)[:, 1:]).abs().max().item()
        print(f"[tree step] {name}: against the suffix pass {d:.3g}", flush=True)
        assert d <= {"tiny": 2e-4, "f16": 4e-2, "bf16": 16 * 2e-2}[name]  # two results within their bars
    finally:
        dm.close()


def greedy(dm, m, K, V, cu, first, steps):
    """The plain greedy rollout by rp_decode_step over a dense cache."""
    B, cap = len(cu) - 1, 200
    ck = torch.zeros(m.n_layers, B, cap, m.n_kv_heads, m.head_dim, dtype=dm.dtype, device="cuda")
    cv = torch.zeros_like(ck)
    for b in range(B):
        n = cu[b + 1] - cu[b]
        ck[:, b, :n], cv[:, b, :n] = K[:, cu[b]:cu[b + 1]], V[:, cu[b]:cu[b + 1]]
    lens, tok, out = dev([cu[b + 1] - cu[b] for b in range(B)]), dev(first), []
    for _ in range(steps):
        tok = dm.decode(ck, cv, lens, tok)
        lens += 1
        out.append(tok.tolist())
    return np.array(out).T


def test_speculative_rollout_equals_the_greedy_one():
    """Groups of three responses forked from two prompts, drafts that are sometimes right, one
    sequence ending early, compactions: the same tokens as one decode step after the other."""
    m, hw, bt, dm, cu, c, K, V, h = setup("tiny", [45, 32], [30, 0], 303, n_pages=60, n_seqs=8, table_ld=10)
    try:
        rng = random.Random(7)
        first = [[rng.randrange(m.vocab) for _ in range(3)] for _ in range(2)]
        want = [None] * 6
        for p in range(2):
            n = cu[p + 1] - cu[p]
            Kp, Vp = K[:, cu[p]:cu[p + 1]].repeat(1, 3, 1, 1), V[:, cu[p]:cu[p + 1]].repeat(1, 3, 1, 1)
            want[3 * p:3 * p + 3] = list(greedy(dm, m, Kp, Vp, [0, n, 2 * n, 3 * n], first[p], 40))
        # the prompts move to rows 6 and 7, their responses to rows 0 .. 5
        assert c.fork([0, 1], [6, 7]).tolist() == [0, 0]
        c.free([0, 1])
        assert c.fork([6, 6, 6, 7, 7, 7], list(range(6))).tolist() == [0] * 6
        c.free([6, 7])
        B, N = 6, 8
        cur = [first[b // 3][b % 3] for b in range(B)]
        got = [[] for _ in range(B)]
        for step in range(60):
            live = [b for b in range(B) if len(got[b]) < (9 if b == 4 else 24)]
            if not live:
                break
            tokens, parents = [[0] * N for _ in range(B)], [[-1] * N for _ in range(B)]
            for b in live:
                tokens[b][0] = cur[b]
                k = len(got[b])
                for i in range(1, N):  # two chains below the root; the right one is right up to a point
                    parents[b][i] = i - 2 if i > 2 else 0
                    d = k + (i - 1) // 2
                    right = i % 2 == b % 2 and rng.random() < 0.8
                    tokens[b][i] = int(want[b][d]) if right else rng.randrange(m.vocab)
            nodes = [N if b in live else 0 for b in range(B)]
            if step % 2:
                nodes = [min(n, 5) for n in nodes]
            t, p, n = dev(tokens), dev(parents), dev(nodes)
            nxt, dk, dv = dm.tree_step(c, t, parents=p, n_nodes=n)
            acc, cnt, out, missing = c.commit(t, p, nxt, dk, dv, n_nodes=n)
            assert missing.tolist() == [0] * B
            for b in range(B):
                k = cnt[b].item()
                assert (k > 0) == (b in live)
                if k:
                    got[b] += [tokens[b][j] for j in acc[b].tolist()[1:k]] + [out[b].item()]
                    cur[b] = out[b].item()
            if step == 3:
                c.compact()
            if len(got[4]) >= 9 and 4 in live:
                c.free([4])
                c.compact()
        for b in range(B):
            assert len(got[b]) >= (9 if b == 4 else 24)
            assert got[b] == [int(x) for x in want[b][:len(got[b])]], b
        assert step < 23, "some drafts were confirmed"
    finally:
        dm.close()


@pytest.mark.parametrize("name,B,N", [("bf16", 3, 5), ("f16", 4, 20), ("tiny", 2, 3)])
def test_step_and_commit_in_a_graph(name, B, N):
    """Two rollout steps replayed from one graph equal the eager ones, bit for bit."""
    m, hw, bt, dm, cu, c, *_ = setup(name, [50, 17, 64, 3], [0, 0, 0, 0], 304)
    try:
        first = [t.clone() for t in (c.table, c.length, c.refs, c.k, c.v)]
        g = torch.Generator().manual_seed(3)
        tok0 = torch.randint(0, m.vocab, (B, N), generator=g, dtype=torch.int32).cuda()
        tok, parents = tok0.clone(), dev([[-1] + [max(0, i - 2) for i in range(1, N)]] * B)
        nodes = dev([N, N - 1, 1, N][:B])
        draft, nxt = dm.alloc_kv(B * N), torch.empty(B, N, dtype=torch.int32, device="cuda")
        logits = torch.zeros(B, N, m.vocab, device="cuda") if N < 10 else None
        ws = dm.workspace(rb.rp_tree_step_workspace_bytes(dm.handle, B, N))
        ints = lambda *s: torch.empty(s, dtype=torch.int32, device="cuda")
        acc, cnt, out, miss = ints(B, N), ints(B), ints(B), ints(B)

        def step():
            dm.tree_step(c, tok, parents=parents, n_nodes=nodes, draft=draft, logits=logits, next_ids=nxt, workspace=ws)
            c.commit(tok, parents, nxt, *draft, n_nodes=nodes, accepted=acc, n_accepted=cnt, token_out=out, missing=miss)
            tok[:, 0].copy_(out)

        def state():
            torch.cuda.synchronize()
            real = torch.arange(N, device="cuda") < nodes[:, None]
            keep = [t.clone() for t in (tok, acc, cnt, out, miss, c.table, c.length, c.refs)]
            return keep + [c.k.view(torch.int32 if name == "tiny" else torch.int16).clone(), nxt[real].clone()] + \
                ([logits[real].clone()] if logits is not None else [])

        def restore():
            tok.copy_(tok0)
            for t, x in zip((c.table, c.length, c.refs, c.k, c.v), first):
                t.copy_(x)

        want = []
        for _ in range(2):
            step()
            want.append(state())
        restore()
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            with torch.cuda.graph(graph, stream=side):
                step()
        torch.cuda.current_stream().wait_stream(side)
        for rep in range(2):
            restore()
            for k in range(2):
                _ = torch.randn(4096, device="cuda").sum().item()
                graph.replay()
                for i, (x, y) in enumerate(zip(state(), want[k])):
                    assert torch.equal(x, y), (rep, k, i)
    finally:
        dm.close()


def test_large_step_equals_small_ones():
    """More rows than the 64 of the decode-shaped projections: each tree's tokens as in a step of its own."""
    m, hw, bt, dm, cu, c, *_ = setup("tiny", [40, 20, 77], [0, 0, 0], 305)
    try:
        g = torch.Generator().manual_seed(5)
        tok = torch.randint(0, m.vocab, (3, 40), generator=g, dtype=torch.int32).cuda()
        big = torch.empty(3, 40, m.vocab, device="cuda")
        dm.tree_step(c, tok, logits=big)
        for b in range(3):
            one = PagedKV(c.k, c.v, c.table[b:b + 1].contiguous(), c.length[b:b + 1].contiguous(), c.refs)
            lg = torch.empty(1, 40, m.vocab, device="cuda")
            dm.tree_step(one, tok[b:b + 1].contiguous(), logits=lg)
            assert (big[b] - lg[0]).abs().max().item() <= 1e-4
    finally:
        dm.close()


CHILD = r'''
import os, sys, torch
sys.path.insert(0, %(root)r)
import tests.test_gpu_tree_step as t
m, hw, bt, dm, cu, c, *_ = t.setup("bf16", [50, 17], [0, 0], 306)
tok = t.dev([[3, 4, 5], [6, 7, 8]])
if sys.argv[1] == "bad":
    tok[1, 1] = m.vocab
if sys.argv[1] == "guard":  # (read when the call ends: the set-up's calls are over)
    os.environ["RP_DEBUG_CORRUPT_GUARD"] = "1"
try:
    nxt, K, V = dm.tree_step(c, tok)
    q = torch.randn(2, 3, 6, 128, device="cuda").bfloat16()
    c.tree_attention(0, q, K[0].view(2, 3, 2, 128), V[0].view(2, 3, 2, 128))
    print("STATUS OK", nxt.tolist(), flush=True)
except t.rb.RollplexError as e:
    print("STATUS", e, flush=True)
'''


@pytest.mark.parametrize("case,needle", [("good", "OK"), ("bad", "token_ids[4] = 1000"), ("guard", "guard")])
def test_debug_mode(case, needle):
    env = {k: v for k, v in os.environ.items() if not k.startswith("RP_DEBUG")}
    said = []
    for on in ([False, True] if case == "good" else [True]):
        e = dict(env, RP_DEBUG="1") if on else env
        r = subprocess.run([sys.executable, "-c", CHILD % {"root": ROOT}, case], env=e, capture_output=True, text=True, timeout=300, cwd=ROOT)
        line = [x for x in r.stdout.splitlines() if x.startswith("STATUS")]
        assert r.returncode == 0 and line, r.stdout[-2000:] + r.stderr[-2000:]
        said.append(line[-1])
    assert needle in said[-1] and len(set(said)) == 1, said
