"""The largest paged caches and batches that the calls on pages and drafted trees take, on the host."""
import pytest

from paper_2608_14498_amd import binding as rb
from paper_2608_14498_amd import configs
from tests.test_abi_cpu import FAKE, fake_weights
from tests.test_pages_cpu import pages, refused


@pytest.mark.parametrize("page", [8, 16, 64, 1024])
def test_tables_whose_lengths_rounded_up_would_pass_32_bits(page):
    """A clamped length, rounded up to a tile or looked ahead of, stays in 32 bits."""
    most = ((1 << 31) - (1 << 14)) // page
    assert rb.rp_pages_compact_workspace_bytes(pages(page_size=page, n_pages=1, table_ld=most)) > 0
    for ld in (most + 1, (1 << 31) // page - 1, (1 << 31) // page):
        p = pages(page_size=page, n_pages=1, table_ld=ld)
        refused(rb.RP_ERR_UNSUPPORTED, "table_ld", rb.rp_pages_compact_workspace_bytes, p)
        refused(rb.RP_ERR_UNSUPPORTED, "table_ld", rb.rp_tree_attention_workspace_bytes, p, 1, 1, 4)


def test_batches_whose_launches_would_pass_32_bits_of_threads():
    """The merge of the attention's pieces: a workgroup of 256 threads each 32 rows of a kv head."""
    big = dict(n_seqs=1 << 24, page_size=8, n_pages=1, table_ld=1)
    one = pages(n_kv_heads=1, layer_stride=1 << 20, **big)
    two = pages(n_kv_heads=2, layer_stride=1 << 20, **big)
    assert rb.rp_tree_attention_workspace_bytes(one, (1 << 24) - 1, 1, 1) > 0
    assert rb.rp_tree_attention_workspace_bytes(two, (1 << 23) - 1, 2, 16) > 0  # 16 rows a kv head
    refused(rb.RP_ERR_UNSUPPORTED, "2\\^24", rb.rp_tree_attention_workspace_bytes, one, 1 << 24, 1, 1)
    refused(rb.RP_ERR_UNSUPPORTED, "2\\^24", rb.rp_tree_attention_workspace_bytes, two, 1 << 23, 1, 2)
    refused(rb.RP_ERR_UNSUPPORTED, "2\\^24", rb.rp_tree_attention_workspace_bytes, two, 1 << 23, 2, 16)
    wide = pages(n_kv_heads=64, head_dim=64, layer_stride=1 << 20, **big)
    refused(rb.RP_ERR_UNSUPPORTED, "2\\^24", rb.rp_tree_attention, wide, 0, 0, 1 << 16, 256, 512, None, None, FAKE, 512 * 64, FAKE, FAKE, 0.1,
            FAKE, FAKE, 1 << 60)


def test_steps_of_more_tokens_than_a_launch_has_rows_for():
    """Row kernels of a step: a workgroup of up to 1024 threads a token."""
    w, keep = fake_weights(configs.TINY)
    h = rb.rp_create(rb.make_config(configs.TINY, 1024), w)
    try:
        assert rb.rp_tree_step_workspace_bytes(h, (1 << 22) - 1, 1) > 0
        refused(rb.RP_ERR_UNSUPPORTED, "2\\^22", rb.rp_tree_step_workspace_bytes, h, 1 << 22, 1)
        p = pages(n_seqs=1 << 22, page_size=8, n_pages=1, table_ld=1)
        draft = rb.make_kv(FAKE, FAKE, 1 << 40)
        refused(rb.RP_ERR_UNSUPPORTED, "2\\^22", rb.rp_tree_step, h, 0, p, 1 << 16, 64, None, FAKE, None, None, draft, None, FAKE, FAKE, 1 << 60)
    finally:
        rb.rp_destroy(h)


def test_a_steps_merge_is_bounded_where_its_workspace_is_asked_for():
    import dataclasses

    m = dataclasses.replace(configs.TINY, n_q_heads=64, n_kv_heads=64, head_dim=64)
    w, keep = fake_weights(m)
    h = rb.rp_create(rb.make_config(m, 1024), w)
    try:
        assert rb.rp_tree_step_workspace_bytes(h, (1 << 18) - 1, 1) > 0
        refused(rb.RP_ERR_UNSUPPORTED, "kv heads", rb.rp_tree_step_workspace_bytes, h, 1 << 18, 1)
        refused(rb.RP_ERR_UNSUPPORTED, "kv heads", rb.rp_tree_step_workspace_bytes, h, 1 << 18, 8)
    finally:
        rb.rp_destroy(h)
