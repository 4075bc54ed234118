"""Paged cache and drafted trees without a GPU: refusals before any HIP call, workspace sizes, the
Python layer's checks, and the rules' model in pages_model.py against itself."""
import ctypes
import os
import random

import pytest
import torch

from paper_2608_14498_amd import binding as rb
from paper_2608_14498_amd import configs
from paper_2608_14498_amd.runtime import PagedKV
from tests.pages_model import PoolModel, walk
from tests.test_abi_cpu import FAKE, fake_weights


def pages(**over):
    f = dict(k=FAKE, v=FAKE, layer_stride=64 * 16 * 2 * 64, dtype="f32", n_layers=2, n_kv_heads=2, head_dim=64, n_pages=64,
             page_size=16, table=FAKE, length=FAKE, refs=FAKE, n_seqs=8, table_ld=12)
    f.update(over)
    return rb.make_pages(**f)


def refused(status, text, call, *args):
    with pytest.raises(rb.RollplexError, match=text) as e:
        call(*args)
    assert e.value.status == status


ROWS = rb.make_kv(FAKE, FAKE, 1 << 20)
BAD_PAGES = [
    (dict(k=None), rb.RP_ERR_INVALID_ARG, "required"),
    (dict(table=None), rb.RP_ERR_INVALID_ARG, "required"),
    (dict(length=None), rb.RP_ERR_INVALID_ARG, "required"),
    (dict(refs=None), rb.RP_ERR_INVALID_ARG, "required"),
    (dict(v=FAKE + 8), rb.RP_ERR_INVALID_ARG, "aligned"),
    (dict(layer_stride=64 * 16 * 2 * 64 + 4), rb.RP_ERR_INVALID_ARG, "multiple of 8"),
    (dict(layer_stride=64 * 16 * 2 * 64 - 8), rb.RP_ERR_SHAPE, "layer_stride"),
    (dict(page_size=4), rb.RP_ERR_SHAPE, "page_size"),
    (dict(page_size=24), rb.RP_ERR_SHAPE, "page_size"),
    (dict(page_size=2048), rb.RP_ERR_SHAPE, "page_size"),
    (dict(n_pages=0), rb.RP_ERR_SHAPE, "positive"),
    (dict(n_seqs=0), rb.RP_ERR_SHAPE, "positive"),
    (dict(table_ld=-1), rb.RP_ERR_SHAPE, "positive"),
    (dict(n_layers=0), rb.RP_ERR_SHAPE, "positive"),
    (dict(table_ld=1 << 27), rb.RP_ERR_UNSUPPORTED, "table_ld"),
    (dict(n_kv_heads=1, head_dim=1), rb.RP_ERR_UNSUPPORTED, "16-byte"),
    (dict(n_kv_heads=1 << 20), rb.RP_ERR_UNSUPPORTED, "16-byte"),
]


@pytest.mark.parametrize("over,status,text", BAD_PAGES)
def test_bad_pool_is_refused_by_every_call(over, status, text):
    p = pages(**over)
    refused(status, text, rb.rp_pages_append, p, 0, 1, [0], [0, 1], ROWS, FAKE)
    refused(status, text, rb.rp_pages_fork, p, 0, 1, [0], [1], FAKE)
    refused(status, text, rb.rp_pages_free, p, 0, 1, [0])
    refused(status, text, rb.rp_pages_compact_workspace_bytes, p)
    refused(status, text, rb.rp_pages_compact, p, 0, None, FAKE, 1 << 20)
    refused(status, text, rb.rp_tree_attention_workspace_bytes, p, 1, 1, 4)
    refused(status, text, rb.rp_tree_attention, p, 0, 0, 1, 1, 4, None, None, FAKE, 256, FAKE, FAKE, 0.1, FAKE, FAKE, 1 << 30)
    refused(status, text, rb.rp_tree_commit, p, 0, 1, 1, None, FAKE, None, FAKE, ROWS, FAKE, FAKE, FAKE, FAKE)


def test_bad_dtype_and_null_pool():
    p = pages()
    p.dtype = 7
    refused(rb.RP_ERR_INVALID_ARG, "dtype", rb.rp_pages_free, p, 0, 1, [0])
    lib = rb.lib()
    one = (ctypes.c_int32 * 1)(0)
    assert lib.rp_pages_free(None, None, 1, one) == rb.RP_ERR_INVALID_ARG
    assert lib.rp_pages_free(ctypes.byref(pages()), None, 1, None) == rb.RP_ERR_INVALID_ARG


@pytest.mark.parametrize("seqs,text", [([8], "outside"), ([-1], "outside"), ([3, 1, 3], "twice"), ([], "count"), (list(range(8)) * 40, "count")])
def test_sequence_lists(seqs, text):
    p = pages()
    refused(rb.RP_ERR_SHAPE, text, rb.rp_pages_free, p, 0, len(seqs), seqs)
    refused(rb.RP_ERR_SHAPE, text, rb.rp_pages_append, p, 0, len(seqs), seqs, list(range(len(seqs) + 1)), ROWS, FAKE)
    if text != "count":
        refused(rb.RP_ERR_SHAPE, text, rb.rp_pages_fork, p, 0, len(seqs), [7] * len(seqs), seqs, FAKE)


def test_append_and_fork_refusals():
    p = pages()
    refused(rb.RP_ERR_SHAPE, "must be 0", rb.rp_pages_append, p, 0, 1, [0], [1, 2], ROWS, FAKE)
    refused(rb.RP_ERR_SHAPE, "< cu", rb.rp_pages_append, p, 0, 2, [0, 1], [0, 5, 4], ROWS, FAKE)
    refused(rb.RP_ERR_INVALID_ARG, "missing", rb.rp_pages_append, p, 0, 1, [0], [0, 2], ROWS, None)
    refused(rb.RP_ERR_SHAPE, "layer_stride", rb.rp_pages_append, p, 0, 1, [0], [0, 9000], ROWS, FAKE)
    refused(rb.RP_ERR_INVALID_ARG, "k or v", rb.rp_pages_append, p, 0, 1, [0], [0, 1], rb.make_kv(None, FAKE, 1024), FAKE)
    refused(rb.RP_ERR_INVALID_ARG, "aligned", rb.rp_pages_append, p, 0, 1, [0], [0, 1], rb.make_kv(FAKE + 4, FAKE, 1024), FAKE)
    refused(rb.RP_ERR_SHAPE, "both a src and a dst", rb.rp_pages_fork, p, 0, 2, [0, 1], [2, 0], FAKE)
    refused(rb.RP_ERR_SHAPE, "both a src and a dst", rb.rp_pages_fork, p, 0, 1, [3], [3], FAKE)
    refused(rb.RP_ERR_INVALID_ARG, "missing", rb.rp_pages_fork, p, 0, 1, [0], [1], None)
    huge = [0, (1 << 30) + 1]
    refused(rb.RP_ERR_UNSUPPORTED, "2\\^30", rb.rp_pages_append, p, 0, 1, [0], huge, rb.make_kv(FAKE, FAKE, 1 << 40), FAKE)


@pytest.mark.parametrize("seq", [[3, 1], (3, 1), b"\x03\x01", iter([3, 1]), [3.0, 1.0], iter([3, 1.5]), torch.tensor([3, 1])])
def test_host_lists_of_any_kind(seq):
    assert list(rb._i32(seq)) == [3, 1]


def test_listed_numbers_that_do_not_fit():
    """(They would wrap round to another sequence.)"""
    p = pages()
    for call, args in ((rb.rp_pages_append, (1, [1 << 32], [0, 1], ROWS, FAKE)), (rb.rp_pages_append, (1, [0], [0, 1 << 32], ROWS, FAKE)),
                       (rb.rp_pages_fork, (1, [1 << 32], [1], FAKE)), (rb.rp_pages_fork, (1, [1], [1 << 32], FAKE)),
                       (rb.rp_pages_free, (1, [-(1 << 32)]))):
        with pytest.raises(ValueError, match="32 bits"):
            call(p, 0, *args)


def test_compact_workspace():
    need = rb.rp_pages_compact_workspace_bytes(pages())
    assert 2 * 64 * 4 <= need <= 4 * 64 * 4
    refused(rb.RP_ERR_WORKSPACE, "workspace", rb.rp_pages_compact, pages(), 0, None, FAKE, need - 1)
    refused(rb.RP_ERR_INVALID_ARG, "256-byte", rb.rp_pages_compact, pages(), 0, None, FAKE + 16, need)
    refused(rb.RP_ERR_INVALID_ARG, "NULL", rb.rp_pages_compact, pages(), 0, None, None, need)


def attention(p=None, layer=0, B=1, N=3, Hq=4, n_nodes=None, mask=None, q=FAKE, q_ld=256, k=FAKE, v=FAKE, scale=0.1, out=FAKE, ws=FAKE,
              nbytes=1 << 40):
    rb.rp_tree_attention(p or pages(), 0, layer, B, N, Hq, n_nodes, mask, q, q_ld, k, v, scale, out, ws, nbytes)


@pytest.mark.parametrize("over,status,text", [
    (dict(layer=2), rb.RP_ERR_SHAPE, "layer"), (dict(layer=-1), rb.RP_ERR_SHAPE, "layer"),
    (dict(B=0), rb.RP_ERR_SHAPE, "batch"), (dict(B=9), rb.RP_ERR_SHAPE, "batch"),
    (dict(N=0), rb.RP_ERR_SHAPE, "new tokens"), (dict(N=257), rb.RP_ERR_SHAPE, "new tokens"),
    (dict(Hq=3), rb.RP_ERR_SHAPE, "multiple"), (dict(Hq=0), rb.RP_ERR_SHAPE, "multiple"), (dict(Hq=18), rb.RP_ERR_UNSUPPORTED, "group"),
    (dict(q=None), rb.RP_ERR_INVALID_ARG, "required"), (dict(out=None), rb.RP_ERR_INVALID_ARG, "required"),
    (dict(k=None), rb.RP_ERR_INVALID_ARG, "required"), (dict(v=FAKE + 2), rb.RP_ERR_INVALID_ARG, "aligned"),
    (dict(q_ld=248), rb.RP_ERR_SHAPE, "q_ld"), (dict(q_ld=260), rb.RP_ERR_SHAPE, "q_ld"),
    (dict(scale=float("nan")), rb.RP_ERR_SHAPE, "scale"), (dict(scale=float("inf")), rb.RP_ERR_SHAPE, "scale"),
    (dict(nbytes=0), rb.RP_ERR_WORKSPACE, "workspace"), (dict(ws=FAKE + 16), rb.RP_ERR_INVALID_ARG, "256-byte"),
    (dict(p=pages(n_kv_heads=4, head_dim=32)), rb.RP_ERR_UNSUPPORTED, "head_dim"),
])
def test_attention_refusals(over, status, text):
    refused(status, text, lambda: attention(**over))


def test_commit_refusals():
    args = dict(B=2, N=3, n_nodes=None, token_ids=FAKE, parents=None, next_ids=FAKE, draft=ROWS, accepted=FAKE, n_accepted=FAKE,
                token_out=FAKE, missing=FAKE)
    call = lambda p=None, **o: rb.rp_tree_commit(p or pages(), 0, **dict(args, **o))
    for name in ("token_ids", "next_ids", "accepted", "n_accepted", "token_out", "missing"):
        refused(rb.RP_ERR_INVALID_ARG, "required", lambda: call(**{name: None}))
    refused(rb.RP_ERR_SHAPE, "batch", lambda: call(B=9))
    refused(rb.RP_ERR_SHAPE, "new tokens", lambda: call(N=300))
    refused(rb.RP_ERR_UNSUPPORTED, "4096", lambda: call(p=pages(n_seqs=5000), B=4097))
    refused(rb.RP_ERR_SHAPE, "layer_stride", lambda: call(draft=rb.make_kv(FAKE, FAKE, 6 * 128 - 8)))


def test_step_refusals():
    w, keep = fake_weights(configs.TINY)
    h = rb.rp_create(rb.make_config(configs.TINY, 1024), w)
    try:
        need = rb.rp_tree_step_workspace_bytes(h, 2, 5)
        assert need > 2 * 5 * configs.TINY.vocab * 4
        refused(rb.RP_ERR_SHAPE, "new tokens", rb.rp_tree_step_workspace_bytes, h, 2, 257)
        refused(rb.RP_ERR_UNSUPPORTED, "2\\^24", rb.rp_tree_step_workspace_bytes, h, 1 << 20, 256)
        call = lambda p=None, B=2, N=5, ids=FAKE, draft=ROWS, logits=None, nxt=FAKE, ws=FAKE, n=need: rb.rp_tree_step(
            h, 0, p or pages(), B, N, None, ids, None, None, draft, logits, nxt, ws, n)
        refused(rb.RP_ERR_SHAPE, "model's", lambda: call(p=pages(dtype="bf16")))
        refused(rb.RP_ERR_SHAPE, "model's", lambda: call(p=pages(n_layers=1)))
        refused(rb.RP_ERR_SHAPE, "batch", lambda: call(B=9))
        refused(rb.RP_ERR_INVALID_ARG, "required", lambda: call(ids=None))
        refused(rb.RP_ERR_INVALID_ARG, "required", lambda: call(nxt=None))
        refused(rb.RP_ERR_INVALID_ARG, "aligned", lambda: call(logits=FAKE + 4))
        refused(rb.RP_ERR_SHAPE, "draft", lambda: call(draft=rb.make_kv(FAKE, FAKE, 8)))
        refused(rb.RP_ERR_WORKSPACE, "workspace", lambda: call(n=need - 1))
    finally:
        rb.rp_destroy(h)


def test_bf16_step_at_head_dim_64_is_refused_as_the_decode_step_is():
    import dataclasses

    m = dataclasses.replace(configs.TINY, dtype="bf16", ffn_dim=704)
    w, keep = fake_weights(m)
    h = rb.rp_create(rb.make_config(m, 1024), w)
    try:
        refused(rb.RP_ERR_UNSUPPORTED, "head_dim 64", rb.rp_tree_step, h, 0, pages(dtype="bf16"), 1, 1, None, FAKE, None, None, ROWS, None, FAKE,
                FAKE, 1 << 40)
    finally:
        rb.rp_destroy(h)


def test_workspace_of_the_attention_does_not_grow_with_the_cache():
    a = rb.rp_tree_attention_workspace_bytes(pages(), 8, 16, 4)
    b = rb.rp_tree_attention_workspace_bytes(pages(table_ld=5000), 8, 16, 4)
    assert a == b


def test_first_launch_failure_is_reported(monkeypatch):
    monkeypatch.setenv("RP_FAULT_INJECT", "1")
    refused(rb.RP_ERR_HIP, "injected", rb.rp_pages_free, pages(), 0, 1, [0])
    refused(rb.RP_ERR_HIP, "injected", rb.rp_pages_append, pages(), 0, 1, [0], [0, 1], ROWS, FAKE)
    refused(rb.RP_ERR_HIP, "injected", lambda: attention())


def test_python_layer_checks_shapes_and_types():
    c = PagedKV.empty(2, 4, 8, 2, 64, 3, 2, dtype=torch.float32, device="cpu")
    K = torch.zeros(2, 5, 2, 64)
    with pytest.raises(ValueError, match="one entry more"):
        c.append([0], [0], K, K)
    with pytest.raises(ValueError, match="elements"):
        c.append([0], [0, 4], K, K)
    with pytest.raises(ValueError, match="type and device"):
        c.append([0], [0, 5], K.half(), K)
    with pytest.raises(ValueError, match="same length"):
        c.fork([0, 1], [2])
    q = torch.zeros(2, 3, 4, 64)
    n = torch.zeros(2, 3, 2, 64)
    with pytest.raises(ValueError, match="q is"):
        c.tree_attention(0, q.half(), n, n)
    with pytest.raises(ValueError, match="evenly"):
        c.tree_attention(0, q.transpose(1, 2).contiguous().transpose(1, 2), n, n)
    with pytest.raises(ValueError, match="k_new"):
        c.tree_attention(0, q, n[:1], n)
    with pytest.raises(ValueError, match="mask"):
        c.tree_attention(0, q, n, n, mask=torch.zeros(2, 3, 1, dtype=torch.int64))
    with pytest.raises(ValueError, match="out"):
        c.tree_attention(0, q, n, n, out=q[:1])
    with pytest.raises(ValueError, match="workspace"):
        c.tree_attention(0, q, n, n, workspace=torch.zeros(1 << 20))
    with pytest.raises(ValueError, match="workspace"):
        c.compact(workspace=torch.zeros(1 << 20, dtype=torch.int32))
    ids = torch.zeros(2, 3, dtype=torch.int32)
    with pytest.raises(ValueError, match="parents"):
        c.commit(ids, ids[:1], ids, K, K)
    with pytest.raises(ValueError):
        PagedKV(c.k, c.v.half(), c.table, c.length, c.refs)
    with pytest.raises(ValueError, match="refs"):
        PagedKV(c.k, c.v, c.table, c.length, c.refs[:2])
    assert os.path.exists(rb.LIB_PATH)


def test_pool_model_keeps_its_invariants():
    rng = random.Random(3)
    m = PoolModel(40, 8, 9, 6)
    told = {b: [] for b in range(9)}
    x = 0
    for _ in range(400):
        op = rng.choice(["append", "append", "fork", "free", "compact"])
        if op == "append":
            items = []
            for b in rng.sample(range(9), rng.randint(1, 4)):
                k = rng.randint(0, 20)
                items.append((b, [x + i for i in range(k)]))
                x += k
            for (b, v), lack in zip(items, m.append(items)):
                told[b] += v if lack == 0 else []
        elif op == "fork":
            seqs = rng.sample(range(9), 5)
            src, dst = [rng.choice(seqs[:2]) for _ in range(3)], seqs[2:]
            for s, d, lack in zip(src, dst, m.fork(src, dst)):
                told[d] = list(told[s]) if lack == 0 else []
        elif op == "free":
            b = rng.randrange(9)
            m.free([b])
            told[b] = []
        else:
            n = m.compact()
            assert all(r == 0 for r in m.refs[n:]) and all(m.refs[:n])
        for b in range(9):
            assert m.tokens(b) == told[b]
        held = [p for row in m.table for p in row]
        assert [held.count(p) for p in range(40)] == m.refs


def test_walk_takes_the_first_matching_child():
    tokens, parents = [5, 7, 7, 9, 7], [-1, 0, 0, 1, 1]
    assert walk(tokens, parents, [7, 9, 0, 0, 0], 5) == [0, 1, 3]
    assert walk(tokens, parents, [7, 9, 0, 0, 0], 3) == [0, 1]
    assert walk(tokens, parents, [8, 9, 0, 0, 0], 5) == [0]
    assert walk(tokens, parents, [7, 7, 0, 0, 0], 5) == [0, 1, 4]
    assert walk(tokens, parents, [7, 7, 0, 0, 0], 0) == []
