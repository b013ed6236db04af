"""GPU attention over the paged cache where a sequence's length reaches past its
page table: its keys end with the table, and a window that lies wholly behind it
holds none (o = 0, lse = -inf)."""
import numpy as np
import pytest
import torch

import paper_2609_23153_amd as sa
from test_gpu_fwd_cache import DEV, compare, ints, make_cache, queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    sa.library()
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("chunk,window", [(0, 0), (1, 0), (1, 40), (64, 2), (1000, 1)])
@pytest.mark.parametrize("n", [1, 150])                  # few rows, many rows
@pytest.mark.parametrize("pages", [5, 40])               # whole, in parts
@pytest.mark.parametrize("past", [1, 139, (1 << 31) - 5000])
def test_length_past_the_table(past, pages, n, chunk, window):
    held = 64 * pages
    k8, sk, v8, sv, table = make_cache([held, 30], 2, 41)
    assert table.shape[1] == pages
    lengths, start = [held + past, 30], [0, n, n + 2]
    q = queries(n + 2, 4, 42)
    o = torch.full((n + 2, 4, 128), 9.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((n + 2, 4), 9.0, device=DEV)
    sa.sparse_attn_fwd_cache(q, k8, sk, v8, sv, ints(table), ints(start), ints(lengths), o=o, lse=lse,
                             causal=(chunk, window) if chunk else None)
    compare(o, lse, q, (k8, sk, v8, sv), table, start, lengths, chunk, window,
            what=f"{n} rows, {held} + {past} tokens")
    if chunk == 1 and window and past >= 139 and n == 1:     # every window is past the table
        assert bool(lse[:n].isneginf().all()) and not bool(o[:n].any())
    if window == 0 and past >= n:                            # every row sees all that is held
        want, want_lse = sa.sparse_attn_fwd_cache(q, k8, sk, v8, sv, ints(table), ints(start), ints([held, 30]))
        assert torch.equal(o[:n], want[:n]) and torch.equal(lse[:n], want_lse[:n])
