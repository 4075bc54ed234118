"""Rotary positions of drafted tokens at and past the ends of the model's table."""
import pytest
import torch

from tests.test_gpu_tree_step import dev, setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["tiny", "f16"])
def test_positions_are_clamped_to_the_models_table(name):
    """max_position 64 and a prompt of 60 tokens: node i of a chain runs at min(pos0 + i, 63), whatever pos0 is."""
    m, hw, bt, dm, cu, c, *_ = setup(name, [60], [0], 313, max_position=64)
    try:
        tok = torch.arange(5, dtype=torch.int32, device="cuda").view(1, 5) * 7
        roots = dev([[-1] * 5])  # five roots: one position for all

        def step(pos0, parents):
            lg = torch.empty(1, 5, m.vocab, device="cuda")
            dm.tree_step(c, tok, parents=parents, pos0=None if pos0 is None else dev([pos0]), logits=lg)
            return lg

        last, first = step(63, roots), step(0, roots)
        assert torch.equal(step(64, roots), last) and torch.equal(step(2 ** 31 - 1, roots), last)
        assert torch.equal(step(-1, roots), first) and torch.equal(step(-2 ** 31, roots), first)
        assert not torch.equal(last, first)
        chain = step(None, None)  # from 60 on: 60 .. 63, 63
        assert torch.equal(step(60, None), chain) and torch.isfinite(chain).all()
        assert not torch.equal(step(59, None), chain)
    finally:
        dm.close()
