"""GPU weight gradients of the layer norm, exactly.  Inputs are whole numbers of at
most 3, the row statistics 0 and 1: every product and every partial sum is a whole
number below 2^24, which fp32 holds, so the sums are exact in any order and have to
equal those in 64 bits.  A row left out, taken twice or given to another group shows,
however many there are."""
import pytest
import torch

import paper_2609_23153_amd as sa

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    sa.library()
    yield
    torch.cuda.synchronize()


# larger than the caches (over 512 MB) in whole pieces and not, at most 1,024
# workgroups; every team size; groups of one row, of fewer rows than workgroups, of many
CASES = [(1200000, 128, 1, BF16, 0), (1200000, 128, 3, BF16, 8), (1200001, 121, 1, BF16, 0),
         (14000, 10240, 1, BF16, 0), (9001, 8200, 1, F32, 8), (30000, 5120, 2, BF16, 0),
         (9000, 16384, 1, BF16, 0), (5000, 16383, 1, F32, 0), (20000, 5119, 4, BF16, 1),
         (1, 1, 1, F32, 0), (513, 7, 1, BF16, 0), (40000, 96, 5, F32, 0), (7, 128, 7, BF16, 0),
         (3001, 129, 1, F32, 0), (2049, 1024, 3, BF16, 0), (1554, 1531, 2, F32, 0), (70, 2048, 7, BF16, 0),
         (300, 6144, 1, F32, 0), (300, 6145, 2, BF16, 0), (50, 12288, 1, BF16, 0), (50, 12289, 1, F32, 0),
         (65535, 8, 65535, F32, 0)]


@pytest.mark.parametrize("rows,cols,groups,dtype,pad", CASES)
def test_sums_of_whole_numbers(rows, cols, groups, dtype, pad):
    assert 9 * (rows // groups) < 2 ** 24
    g = torch.Generator(device=DEV).manual_seed(rows + cols)
    make = lambda: torch.randint(-3, 4, (rows, cols + pad), generator=g, device=DEV).to(dtype)[:, :cols]
    x, dy = make(), make()
    mean, rstd = torch.zeros(rows, device=DEV), torch.ones(rows, device=DEV)
    _, dw, db = sa.sparse_attn_layer_norm_bwd(dy, x, mean, rstd, groups=groups)
    per, step = rows // groups, max(1, (1 << 25) // cols)
    want = torch.zeros(2, groups, cols, dtype=torch.float64, device=DEV)
    if per <= step:                       # whole groups at a time
        n = step // per
        for i in range(0, groups, n):
            part = slice(i * per, min(i + n, groups) * per)
            a, b = (t[part].double().view(-1, per, cols) for t in (dy, x))
            want[0, i:i + n], want[1, i:i + n] = (a * b).sum(1), a.sum(1)
    else:
        for i in range(groups):
            for r in range(i * per, i * per + per, step):
                part = slice(r, min(r + step, i * per + per))
                a, b = dy[part].double(), x[part].double()
                want[0, i] += (a * b).sum(0)
                want[1, i] += a.sum(0)
    assert torch.equal(dw.double(), want[0]) and torch.equal(db.double(), want[1])
