"""Queries that lie apart: one token a sequence, taken out of a wider projection, against float64."""
import pytest
import torch

from tests.test_gpu_tree_attention import check, make, tree, words

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,Hq,Hkv,D", [("bf16", 28, 4, 128), ("f16", 8, 2, 64), ("f32", 4, 2, 64), ("bf16", 1, 1, 64)])
@pytest.mark.parametrize("B", [1, 5])
def test_one_token_out_of_a_projection(dtype, Hq, Hkv, D, B):
    lens = [333, 20, 1200, 0, 64][:B]
    c, K, V, kn, vn, draw, g = make(dtype, lens, 1, Hkv, D, 16, seed=21)
    wide = draw(B, (Hq + 2 * Hkv) * D)
    rows = wide[:, :Hq * D]
    plain = rows.contiguous().view(B, 1, Hq, D)
    sees = torch.ones(B, 1, 1, dtype=torch.bool)
    for q in (rows.view(B, 1, Hq, D), rows.unflatten(1, (Hq, D)).unsqueeze(1), wide.view(B, 1, Hq + 2 * Hkv, D)[:, :, :Hq], plain):
        print(f"[tree] {dtype} {Hq}/{Hkv} heads of {D}, {B} sequences, strides {q.stride()}", flush=True)
        out = c.tree_attention(1, q, kn, vn)
        check(dtype, out, plain, [k[1] for k in K], [v[1] for v in V], kn, vn, lens, sees, None, D ** -0.5)


@pytest.mark.parametrize("dtype,N", [("bf16", 3), ("f32", 9), ("f16", 70)])
def test_one_head_of_several(dtype, N):
    lens = [100, 33]
    c, K, V, kn, vn, draw, g = make(dtype, lens, N, 1, 64, 8, seed=22)
    q = draw(2, N, 4, 64)[:, :, 2:3]
    sees = tree(2, N, g)
    out = c.tree_attention(0, q, kn, vn, mask=words(sees))
    check(dtype, out, q, [k[0] for k in K], [v[0] for v in V], kn, vn, lens, sees, None, 0.125)
