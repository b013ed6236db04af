"""GPU paged-cache append with row numbers and no rotary table: the numbers are
of no effect, so every byte is the one of the call without them."""
import numpy as np
import pytest
import torch

import paper_2609_23153_amd as sa
from test_gpu_cache_append import DEV, Cache, bits, tokens

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    sa.library()
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("g,kv", [(1, 1), (5, 2)])
@pytest.mark.parametrize("new,total", [([1], [65]), ([3, 0, 70], [3, 40, 100])])
def test_rows_without_a_table(new, total, g, kv):
    start = np.concatenate([[0], np.cumsum(new)])
    T = int(start[-1])
    need = [-(-n // 64) for n in total]
    pages = np.full((len(new), max(need)), -1, dtype=np.int32)
    for b, m in enumerate(need):
        pages[b, :m] = sum(need[:b]) + np.arange(m)
    k, v, q = tokens(T, kv, 1), tokens(T, kv, 2), tokens(T, kv * g, 3)
    rows = np.random.default_rng(4).integers(-5, 1 << 20, T).astype(np.int32)
    plain, numbered = (Cache(sum(need) + 1, kv, pages, seed=5) for _ in range(2))
    # both against the reference, queries too (copied)
    plain.append(k, v, start, total, q=q, what="without rows")
    numbered.append(k, v, start, total, rope_row=rows, q=q, what="with rows")
    for a, b in zip(plain.dev, numbered.dev):
        assert torch.equal(a, b)
    out = sa.sparse_attn_cache_append(
        k, v, *numbered.dev, torch.from_numpy(pages).to(DEV), torch.tensor(start, dtype=torch.int32, device=DEV),
        torch.tensor(total, dtype=torch.int32, device=DEV), rope_row=torch.from_numpy(rows).to(DEV), q=q)
    assert np.array_equal(bits(out), bits(q))
