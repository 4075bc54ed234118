"""One key that outweighs each of the others by far, and so many others that together they count.

The bound of an element is test_gpu_tree_attention's: half a step of the type for the output and for each weight of
the value product, the scores' and sums' fp32 roundings."""
import pytest
import torch

from paper_2608_14498_amd.runtime import PagedKV

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
KEYS = 1 << 18


@pytest.mark.parametrize("gap", [17.5, 12.0, 20.0])
@pytest.mark.parametrize("dtype,N,Hq,B", [("f16", 1, 1, 256), ("f16", 6, 8, 256), ("f16", 256, 8, 32), ("bf16", 1, 8, 256), ("f32", 4, 1, 16)])
def test_many_small_weights_beside_a_large_one(dtype, N, Hq, B, gap):
    """2^18 cached keys, the first one `gap` above the others; the sequences share its pages, so that a share of the work
    (a workgroup, in fp16 and bf16) holds one sequence as a whole."""
    D, page, t = 64, 256, TYPES[dtype]
    g = torch.Generator().manual_seed(24)
    c = PagedKV.empty(1, KEYS // page, page, 1, D, B, KEYS // page, dtype=t)
    c.k.zero_()
    c.k.view(KEYS, D)[0, 0] = gap
    v = (torch.rand(KEYS, D, generator=g) + 0.5).to(t).cuda()
    v[0] = -1
    c.v.view(KEYS, D).copy_(v)
    c.table.copy_(torch.randperm(KEYS // page, generator=g).to(torch.int32).cuda().sort()[0].expand(B, -1))
    c.length.fill_(KEYS)
    q = torch.zeros(B, N, Hq, D, dtype=t, device="cuda")
    q[..., 0] = 1
    q[..., 1:] = (torch.randn(B, N, Hq, D - 1, generator=g) * 2).to(t).cuda()  # (of no effect but on the drafted key)
    kn, vn = torch.zeros(B, N, 1, D, dtype=t, device="cuda"), torch.ones(B, N, 1, D, dtype=t, device="cuda")
    print(f"[tree] {dtype}, {B} x {N} tokens, {Hq} heads, gap {gap}", flush=True)
    out = c.tree_attention(0, q, kn, vn, scale=1.0).double()
    u = torch.finfo(t).eps / 2
    w = torch.exp(torch.tensor(-gap, dtype=torch.float64)).item()
    e, n = (D + 8) * 2.0 ** -24 * gap, 2.0 ** -12
    for i in {0, N // 2, N - 1}:
        seen = torch.cat([v.double(), vn[0, :i + 1, 0].double()])
        p = torch.full((len(seen),), w, dtype=torch.float64, device="cuda")
        p[0] = 1
        p /= p.sum()
        want, pv = (p[:, None] * seen).sum(0), (p[:, None] * seen.abs()).sum(0)
        bound = u * want.abs() + (2 * e + n + 2.0 ** -18 + (u if dtype != "f32" else 0)) * pv + 1e-30 + (2.0 ** -25 if dtype == "f16" else 0)
        off = ((out[:, i] - want).abs() / bound).max().item()
        print(f"[tree] row {i}: worst error / bound {off:.3f}", flush=True)
        assert off <= 1.0
