"""Model steps of more than 64 new tokens, whose projections, logits and argmax take other kernels than those of
smaller steps: every node against the oracle, and against steps of one tree each."""
import random

import numpy as np
import pytest
import torch

import oracle
from paper_2608_14498_amd import inputs
from paper_2608_14498_amd.runtime import PagedKV
from tests.gpu_helpers import rel_err
from tests.test_gpu_tree_step import dev, setup

pytestmark = pytest.mark.gpu

# log-probabilities: the framework's bars (fp32 1e-4, fp16 2e-2, bf16 with 3 bits fewer 8 times that); keys and values: the
# decode step's
BARS = {"tiny": (1e-4, 1e-5), "f16": (2e-2, 3e-2), "f16_d64": (2e-2, 3e-2), "bf16": (8 * 2e-2, 3e-2)}


@pytest.mark.parametrize("name", list(BARS))
@pytest.mark.parametrize("nodes", [[30, 17, 29], [30, 30, 30]])
def test_every_node_of_padded_trees_against_the_oracle(name, nodes):
    """90 rows, 76 of them new tokens or all; and the same choices where no logits are asked for."""
    m, hw, bt, dm, cu, c, *_ = setup(name, [70, 33, 5], [40, 0, 0], 311)
    try:
        rng = random.Random(sum(nodes))
        B, N = 3, 30
        parents = [[-1] + [rng.randint(-1 if i == 20 else 0, i - 1) for i in range(1, N)] for _ in range(B)]
        tokens = [[rng.randrange(m.vocab) for _ in range(N)] for _ in range(B)]
        logits = torch.empty(B, N, m.vocab, device="cuda")
        n_dev = None if min(nodes) == N else dev(nodes)
        nxt, dk, dv = dm.tree_step(c, dev(tokens), parents=dev(parents), n_nodes=n_dev, logits=logits)
        alone, ak, av = dm.tree_step(c, dev(tokens), parents=dev(parents), n_nodes=n_dev)
        torch.cuda.synchronize()
        W = hw.as_f32()
        Ko, Vo, _ = oracle.prefix_forward(W, m, bt.cu_prefix, bt.token_ids, inputs.to_f32(bt.visual))
        shape = (m.n_layers, B, N, m.n_kv_heads, m.head_dim)
        dk, dv, ak, av = (t.view(shape) for t in (dk, dv, ak, av))
        lp_bar, kv_bar = BARS[name]
        worst = worst_kv = 0.0
        for b in range(B):
            prompt = (Ko[:, None, cu[b]:cu[b + 1]], Vo[:, None, cu[b]:cu[b + 1]])
            held = {-1: prompt}  # keys and values up to and with a node
            for i in range(nodes[b]):
                k, v = held[parents[b][i]]
                lg, _, nk, nv = oracle.decode_step(W, m, k, v, [k.shape[2]], [tokens[b][i]])
                held[i] = (np.concatenate([k, nk[:, :, None]], 2), np.concatenate([v, nv[:, :, None]], 2))
                got = torch.log_softmax(logits[b, i].double().cpu(), -1).numpy()
                want = lg[0] - lg[0].max()
                worst = max(worst, np.abs(got - want + np.log(np.exp(want).sum())).max())
                worst_kv = max(worst_kv, rel_err(dk[:, b, i].float().cpu().numpy(), nk[:, 0]), rel_err(dv[:, b, i].float().cpu().numpy(), nv[:, 0]))
                assert nxt[b, i].item() == alone[b, i].item() == logits[b, i].argmax().item(), (b, i)
            assert torch.equal(dk[:, b, :nodes[b]], ak[:, b, :nodes[b]]) and torch.equal(dv[:, b, :nodes[b]], av[:, b, :nodes[b]])
        print(f"[tree step] {name}, 90 rows: max |d log-prob| {worst:.3g} (bar {lp_bar:g}), K and V {worst_kv:.3g} (bar {kv_bar:g})", flush=True)
        assert worst <= lp_bar and worst_kv <= kv_bar
    finally:
        dm.close()


@pytest.mark.parametrize("name", list(BARS))
@pytest.mark.parametrize("N", [40, 100])
def test_large_steps_equal_small_ones(name, N):
    """120 and 300 rows of chains against 40 of one chain at a time: two results, each within its bar."""
    m, hw, bt, dm, cu, c, *_ = setup(name, [40, 20, 77], [0, 0, 0], 312)
    try:
        g = torch.Generator().manual_seed(5)
        tok = torch.randint(0, m.vocab, (3, N), generator=g, dtype=torch.int32).cuda()
        big = torch.empty(3, N, m.vocab, device="cuda")
        dm.tree_step(c, tok, logits=big)
        for b in range(3):
            one = PagedKV(c.k, c.v, c.table[b:b + 1].contiguous(), c.length[b:b + 1].contiguous(), c.refs)
            lg = torch.empty(1, 40, m.vocab, device="cuda")
            dm.tree_step(one, tok[b:b + 1, :40].contiguous(), logits=lg)
            d = (torch.log_softmax(big[b, :40], -1) - torch.log_softmax(lg[0], -1)).abs().max().item()
            print(f"[tree step] {name}, {3 * N} rows against 40, sequence {b}: {d:.3g}", flush=True)
            assert d <= 2 * BARS[name][0]
    finally:
        dm.close()
