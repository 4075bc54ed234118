"""Paged cache whose tables, lengths and reference counts lie next to each other in one buffer, at any offset: what a
call changes of one must not be read as it was before by way of another in the same cache line."""
import random

import pytest
import torch

from paper_2608_14498_amd.runtime import PagedKV
from tests.test_gpu_pages import Both

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_pages,n_seqs,table_ld,offset", [(14, 9, 3, 1), (31, 12, 4, 0), (48, 20, 5, 7)])
def test_forks_over_living_children_in_a_tight_pool(n_pages, n_seqs, table_ld, offset):
    """Children that hold pages are forked anew, which need the pages that they give back."""
    rng = random.Random(n_pages)
    both = Both("f32", n_pages, 8, n_seqs, table_ld, L=1, H=1, D=64)
    g, n = both.gpu, n_seqs * table_ld
    flat = torch.zeros(offset + n + n_seqs + n_pages, dtype=torch.int32, device="cuda")[offset:]
    flat[:n] = -1
    both.gpu = PagedKV(g.k, g.v, flat[:n].view(n_seqs, table_ld), flat[n:n + n_seqs], flat[n + n_seqs:])
    for step in range(150):
        op = rng.choice(["append", "fork", "fork", "fork", "free", "compact"])
        if op == "append":
            got, want = both.append([(b, [rng.randrange(64) for _ in range(rng.randint(1, 11))]) for b in rng.sample(range(n_seqs), 2)])
        elif op == "fork":
            seqs = rng.sample(range(n_seqs), rng.randint(3, n_seqs))
            src, dst = [rng.choice(seqs[:2]) for _ in seqs[2:]], seqs[2:]
            got, want = both.gpu.fork(src, dst).tolist(), both.model.fork(src, dst)
        elif op == "free":
            seqs = rng.sample(range(n_seqs), 1)
            got = want = None
            both.gpu.free(seqs)
            both.model.free(seqs)
        else:
            got, want = both.gpu.compact().tolist(), [both.model.compact()]
        assert got == want, (step, op)
        both.check()
