"""The largest paged caches and batches that the calls on pages and drafted trees take, on the host."""
import pytest

from paper_2608_14498_amd import binding as rb
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
