"""fp32 tree attention where the last tile of keys, cached or drafted, ends anywhere."""
import pytest
import torch

from tests.test_gpu_tree_attention import check, make, tree, words

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,D,page", [(4, 2, 64, 8), (3, 1, 128, 16)])
@pytest.mark.parametrize("N", [1, 9, 33])
def test_every_length_of_the_last_tile(Hq, Hkv, D, page, N):
    """Cached lengths 1 .. 64 and drafted ones 1 .. N, in pools whose other slots hold NaN."""
    lens = list(range(1, 65))
    nodes = [1 + b % N for b in range(64)]
    c, K, V, kn, vn, draw, g = make("f32", lens, N, Hkv, D, page, nodes, seed=23, layers=1)
    q = draw(64, N, Hq, D)
    sees = tree(64, N, g)
    out = torch.full_like(q, 3.0)
    print(f"[tree] f32 {Hq}/{Hkv} heads of {D}, page {page}, N {N}", flush=True)
    c.tree_attention(0, q, kn, vn, mask=words(sees), n_nodes=torch.tensor(nodes, dtype=torch.int32, device="cuda"), out=out)
    check("f32", out, q, [k[0] for k in K], [v[0] for v in V], kn, vn, lens, sees, nodes, D ** -0.5, torch.full_like(q, 3.0))
