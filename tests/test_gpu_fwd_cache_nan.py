"""GPU attention over the paged cache: a query that holds a NaN gets NaN for its
output and its lse, whatever kernel serves it and however its keys are cut; where
it sees no key, 0 and -inf as every other; and no other row changes."""
import numpy as np
import pytest
import torch

import paper_2609_23153_amd as sa
from test_gpu_fwd_cache import DEV, ints, make_cache, queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    sa.library()
    yield
    torch.cuda.synchronize()


# few rows whole, in parts of up to 16 and past 256 joined; many rows whole and in parts
@pytest.mark.parametrize("n,length", [(3, 650), (2, 9000), (1, 70000), (70, 650), (200, 9000)])
@pytest.mark.parametrize("causal", [None, (1, 0)])
def test_nan_queries(n, length, causal):
    k8, sk, v8, sv, pages = make_cache([length], 1, 31)
    q = queries(n, 2, 32)
    call = lambda q: sa.sparse_attn_fwd_cache(q, k8, sk, v8, sv, ints(pages), ints([0, n]), ints([length]),
                                              causal=causal)
    want, want_lse = call(q)
    bad = torch.zeros(n, 2, dtype=torch.bool, device=DEV)
    bad[0, 1] = bad[n // 2, 0] = bad[n - 1, 1] = True
    x = q.clone()
    x[0, 1, 5], x[n // 2, 0, 127], x[n - 1, 1] = float("nan"), float("nan"), float("nan")
    o, lse = call(x)
    assert torch.equal(o[~bad], want[~bad]) and torch.equal(lse[~bad], want_lse[~bad])
    assert bool(o[bad].isnan().all()) and bool(lse[bad].isnan().all())


@pytest.mark.parametrize("n,length", [(3, 650), (2, 9000), (70, 650), (200, 9000)])
def test_nan_queries_that_see_no_key(n, length):
    k8, sk, v8, sv, pages = make_cache([length], 1, 33)
    x = torch.full((n, 2, 128), float("nan"), dtype=torch.bfloat16, device=DEV)
    gone = np.full_like(pages, -1)
    for table, have in ((gone, length), (pages, 0)):
        o, lse = sa.sparse_attn_fwd_cache(x, k8, sk, v8, sv, ints(table), ints([0, n]), ints([have]))
        assert not bool(o.any()) and bool(lse.isneginf().all())
