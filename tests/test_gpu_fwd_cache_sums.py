"""GPU attention over the paged cache: the softmax row sum over long ranges that
one workgroup walks alone.

All keys are zero but the first, which the query meets with one product: its
score d = tau 8 q and every other score, 0, carry no rounding of sums, and
lse = log(e^d + n - 1) in closed form.  Bound, in half steps u = 2^-24 of fp32
(an instruction good to one unit in the last place: 2 u):
  scores in log2 units: tau log2(e) is two roundings, 2 u d, the product with it
  one more; the maximum comes back through ln 2: 3 u d + 2 u |lse|;
  an exponential 2 u, its argument is exact for the zero scores;
  the logarithm 2 u log l, adding the maximum u |lse|, the result u |lse|;
  the sum: a page's 32 terms of a lane 5 u (a tree), up to 64 pages one after
  another 64 u, those sums one after another n / 4096 u, lanes and waves 6 u,
  parts (none or some) 8 u.
Together (3 d + 8 |lse| + 85 + n / 4096) u: 1.6e-5 at most here.  Summed term after
term the error grows with the number of keys: 1.3e-4 at 32,768, 8e-4 at 131,072.
"""
import numpy as np
import pytest
import torch

import paper_2609_23153_amd as sa
from gpu_helpers import say

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TAU = float(np.float32(1 / np.sqrt(128)))
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    sa.library()
    yield
    torch.cuda.synchronize()


def ints(v):
    return torch.as_tensor(np.asarray(v, dtype=np.int32)).to(DEV)


def one_key(n, kv):
    """A cache of n keys per head, the first (8, 0, ..), the others zero; values one."""
    k = torch.zeros(n, kv, 128, dtype=torch.bfloat16, device=DEV)
    k[0, :, 0] = 8.0
    v = torch.ones(n, kv, 128, dtype=torch.bfloat16, device=DEV)
    P = -(-n // 64)
    codes = lambda: torch.zeros(P, kv, 8192, dtype=torch.uint8, device=DEV)
    pool = [codes(), torch.ones(P, kv, device=DEV), codes(), torch.ones(P, kv, device=DEV)]
    sa.sparse_attn_cache_append(k, v, *pool, ints(np.arange(P)[None]), ints([0, n]), ints([n]))
    return pool


def query(T, heads, size):
    q = torch.zeros(T, heads, 128, dtype=torch.bfloat16, device=DEV)
    q[:, :, 0] = size
    return q


SIZES = (0.71875, 1.0, 1.9921875, 3.0, 5.0, 8.0, 14.0)


def check(o, lse, size, n, what):
    d = TAU * 8.0 * size
    want = np.log(np.exp(d) + n - 1)
    bound = (3 * d + 8 * abs(want) + 85 + n / 4096) * U
    err = float((lse.double() - want).abs().max())
    say(f"  {what}, score {d:.2f}: lse off by {err:.2e}, bound {bound:.2e}")
    assert err <= bound, (what, size)
    # o = sum p / l = 1: p rounded to bf16 (2^-8), the matrix cores' sums over n / 16
    # steps (2^-24 each of l), o to bf16 (2^-8)
    assert float((o.double() - 1).abs().max()) <= 2.0 ** -7 + n / 16 * U, (what, size)


@pytest.mark.parametrize("n", [32768, 131073])
def test_many_rows_walk_the_whole_range(n):
    # 512 x 64 rows over one key head: 257 tiles fill the chip, so none is cut
    pool, pages = one_key(n, 1), ints(np.arange(-(-n // 64))[None])
    for size in SIZES:
        o, lse = sa.sparse_attn_fwd_cache(query(512, 64, size), *pool, pages, ints([0, 512]), ints([n]))
        check(o, lse, size, n, f"{n} keys, many rows")


@pytest.mark.parametrize("n", [32768, 131073])
def test_one_row_of_many_short_sequences(n):
    # 1,056 tiles x 4 key heads: the long sequence is one of 1,024, and not cut
    B, kv, P = 1024, 4, -(-n // 64)
    pool = one_key(n, kv)
    pages = torch.zeros(B, P, dtype=torch.int32, device=DEV)
    pages[3] = torch.arange(P, dtype=torch.int32, device=DEV)
    length = np.ones(B, dtype=np.int32)
    length[3] = n
    for size in SIZES:
        o, lse = sa.sparse_attn_fwd_cache(query(B, kv, size), *pool, pages, ints(np.arange(B + 1)),
                                          ints(length))
        check(o[3:4], lse[3:4], size, n, f"{n} keys, one row")
        check(o[4:], lse[4:], size, 1, "one key")


@pytest.mark.parametrize("rows", [1, 300])
def test_ranges_in_parts(rows):
    # one token (some 500 parts) and 300 rows (many-row kernel in parts)
    n = 131073
    pool, pages = one_key(n, 1), ints(np.arange(-(-n // 64))[None])
    for size in SIZES:
        o, lse = sa.sparse_attn_fwd_cache(query(rows, 1, size), *pool, pages, ints([0, rows]), ints([n]))
        check(o, lse, size, n, f"{n} keys in parts, {rows} rows")


def test_pages_one_by_one():
    # a table that misses a page takes every page by itself
    n = 131072
    pool, pages = one_key(n, 1), ints(np.arange(n // 64)[None])
    pages[0, 1500] = -1
    for size in SIZES:
        o, lse = sa.sparse_attn_fwd_cache(query(512, 64, size), *pool, pages, ints([0, 512]), ints([n]))
        check(o, lse, size, n - 64, f"{n} keys, a page missing")
