"""Which queries PagedKV.tree_attention takes as they lie in memory, and the row distance that it passes on (CPU)."""
import pytest
import torch

from paper_2608_14498_amd import binding as rb
from paper_2608_14498_amd.runtime import PagedKV


def row_distance(monkeypatch, q, heads_kv):
    """q_ld of the C call that tree_attention(q) makes."""
    B, N, Hq, D = q.shape
    c = PagedKV.empty(1, 8, 16, heads_kv, D, B, 2, dtype=q.dtype, device="cpu")
    said = {}

    def call(self, fn, stream, *args):
        assert fn is rb.rp_tree_attention
        said["q_ld"], said["q"] = args[7], args[6]

    monkeypatch.setattr(PagedKV, "_call", call)
    new = torch.zeros(B, N, heads_kv, D, dtype=q.dtype)
    c.tree_attention(0, q, new, new, out=torch.empty(q.shape, dtype=q.dtype), workspace=torch.empty(1 << 10, dtype=torch.uint8))
    assert said["q"].data_ptr() == q.data_ptr()
    return said["q_ld"]


WIDE = (4 + 2 * 2) * 64  # one row of a q/k/v projection: 4 query heads and 2 kv heads of 64


def views(B):
    x = torch.zeros(B, WIDE)
    q = x[:, :256]
    return {"view": q.view(B, 1, 4, 64), "unsqueeze": q.unflatten(1, (4, 64)).unsqueeze(1), "unflatten": q.unflatten(0, (B, 1)).unflatten(2, (4, 64)),
            "heads of a wider view": x.view(B, 1, 8, 64)[:, :, :4]}


@pytest.mark.parametrize("B", [1, 2, 7])
@pytest.mark.parametrize("how", list(views(1)))
def test_one_token_out_of_a_wider_projection(monkeypatch, B, how):
    assert row_distance(monkeypatch, views(B)[how], 2) == (WIDE if B > 1 else 256)


def test_one_head_of_several(monkeypatch):
    x = torch.zeros(3, 5, 4, 64)
    assert row_distance(monkeypatch, x[:, :, 1:2], 1) == 256
    one = torch.zeros(3, 5, 64).unsqueeze(2)  # the head's own stride is 64; and one that says nothing:
    assert row_distance(monkeypatch, one, 1) == 64
    assert row_distance(monkeypatch, x.as_strided((3, 5, 1, 64), (5 * 256, 256, 1, 1)), 1) == 256
    assert row_distance(monkeypatch, x[:1, 0:1].as_strided((1, 1, 4, 64), (7, 7, 64, 1)), 2) == 256
    assert row_distance(monkeypatch, x[:, ::2][:1], 2) == 512


def test_uneven_rows_and_heads_apart_are_refused(monkeypatch):
    x = torch.zeros(3, 6, 4, 64)
    for q in (x[:, :5], x.transpose(0, 1), x[:, :, ::2], x.transpose(1, 2).contiguous().transpose(1, 2)):
        with pytest.raises(ValueError, match="evenly"):
            row_distance(monkeypatch, q, 1)
