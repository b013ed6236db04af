"""GPU paged-cache append against the reference: codes, scales and rotated
queries bit for bit, and every byte that the call does not own unchanged."""
import numpy as np
import pytest
import torch

import paper_2609_23153_amd as sa
from gpu_helpers import say
from oracle import kv_cache as R

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    sa.library()
    yield
    torch.cuda.synchronize()


def bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


class Cache:
    """A pool of stale pages (any finite codes, scales 2^-3 .. 2^3)."""

    def __init__(self, P, kv, pages, seed=0):
        rng = np.random.default_rng(seed)
        codes = lambda: (rng.integers(0, 127, (P, kv, 8192)) +
                         128 * rng.integers(0, 2, (P, kv, 8192))).astype(np.uint8)
        scales = lambda: (2.0 ** rng.integers(-3, 4, (P, kv))).astype(np.float32)
        self.np = [codes(), scales(), codes(), scales()]
        self.dev = [torch.from_numpy(a).to(DEV) for a in self.np]
        self.pages = np.asarray(pages, dtype=np.int32)

    def append(self, k, v, q_start, kv_len, rope=None, rope_row=None, q=None, what="", pages=None):
        dev = lambda a: None if a is None else torch.as_tensor(a).to(DEV)
        wide = lambda t: None if t is None else t.float().cpu().numpy()
        q_start, kv_len = (np.asarray(a, dtype=np.int32) for a in (q_start, kv_len))
        *self.np, want_q = R.append(wide(k), wide(v), *self.np, self.pages, q_start, kv_len,
                                    rope, rope_row, wide(q))
        q_out = None if q is None else torch.zeros(q.shape, dtype=torch.bfloat16, device=DEV)
        got_q = sa.sparse_attn_cache_append(
            k, v, *self.dev, dev(self.pages) if pages is None else pages, dev(q_start), dev(kv_len),
            rope=dev(rope), rope_row=dev(rope_row), q=q, q_out=q_out)
        for name, got, want in zip(("k8", "sk", "v8", "sv"), self.dev, self.np):
            same = np.array_equal(got.cpu().numpy(), want)
            say(f"  {what}: {name} {'equal' if same else 'differs'}")
            assert same, (what, name)
        if q is None:
            assert got_q is None
        else:
            assert np.array_equal(bits(got_q), want_q), (what, "q")


def tokens(T, heads, seed, spread=0.5):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, heads, 128, generator=g) * torch.exp(spread * torch.randn(T, 1, 1, generator=g))
    return x.bfloat16().to(DEV)


def table(rows, dim, seed=0):
    ang = np.random.default_rng(seed).uniform(0, 7, (rows, dim // 2))
    return np.stack([np.cos(ang), np.sin(ang)], -1).astype(np.float32)


@pytest.mark.parametrize("kv,g,dim", [(1, 1, 0), (1, 1, 128), (3, 1, 64), (2, 5, 8), (1, 16, 120)])
@pytest.mark.parametrize("n,length", [(1, 1), (1, 64), (1, 65), (2, 65), (63, 63), (64, 64), (65, 130),
                                      (130, 131), (300, 333), (5, 1000)])
def test_one_sequence(kv, g, dim, n, length):
    need = -(-length // 64)
    c = Cache(need + 2, kv, [np.random.default_rng(n).permutation(need + 2)[:need]], seed=n)
    rope = table(length, dim) if dim else None
    c.append(tokens(n, kv, 1), tokens(n, kv, 2), [0, n], [length], rope=rope,
             q=tokens(n, kv * g, 3), what=f"{n} of {length}")


def test_ragged_batch_with_rows_and_strides():
    new, total = [3, 0, 70, 1, 129, 1], [3, 40, 100, 65, 1000, 64]
    start = np.concatenate([[2], 2 + np.cumsum(new)])     # two rows in front and three behind
    T = int(start[-1]) + 3
    need = [-(-t // 64) for t in total]
    pool = np.random.default_rng(5).permutation(sum(need) + 4)
    pages = np.full((6, max(need) + 1), -1, dtype=np.int32)
    at = 0
    for b, m in enumerate(need):
        pages[b, :m] = pool[at:at + m]
        at += m
    c = Cache(sum(need) + 4, 2, pages)
    # heads of a wider projection, as a fused qkv product leaves them
    qkv = tokens(T, 10, 7)
    rows = np.random.default_rng(6).integers(-3, 60, T).astype(np.int32)  # some outside the table
    wide = torch.full((6, max(need) + 5), -1, dtype=torch.int32, device=DEV)
    wide[:, :max(need) + 1] = torch.from_numpy(pages).to(DEV)
    c.append(qkv[:, 6:8], qkv[:, 8:10], start, total, rope=table(50, 128), rope_row=rows,
             q=qkv[:, :6], what="ragged", pages=wide[:, :max(need) + 1])


def test_many_sequences_of_one_token():
    B = 200                                               # more than a wave's worth of starts
    rng = np.random.default_rng(8)
    total = rng.integers(1, 200, B)
    pages = np.arange(B * 4, dtype=np.int32).reshape(B, 4)[rng.permutation(B)]
    c = Cache(B * 4, 1, pages)
    c.append(tokens(B, 1, 1), tokens(B, 1, 2), np.arange(B + 1), total, rope=table(200, 128),
             q=tokens(B, 4, 3), what="batch")


def test_thousands_of_sequences():
    # found in three steps; many get no token
    B = 5000
    rng = np.random.default_rng(10)
    new = rng.integers(0, 3, B)
    start = np.concatenate([[0], np.cumsum(new)])
    total = new + rng.integers(0, 62, B)
    T = int(start[-1])
    c = Cache(B, 1, rng.permutation(B).reshape(B, 1))
    c.append(tokens(T, 1, 4), tokens(T, 1, 5), start, total, rope=table(64, 64), q=tokens(T, 1, 6),
             what="5000 sequences")


def test_token_by_token_with_growing_and_shrinking_tokens():
    c = Cache(3, 2, [[2, 0]])
    rng = np.random.default_rng(9)
    for n in range(70):
        size = float(2.0 ** rng.integers(-12, 13))
        k, v = tokens(1, 2, 2 * n) * size, tokens(1, 2, 2 * n + 1) / size
        c.append(k.bfloat16(), v.bfloat16(), [0, 1], [n + 1], rope=table(70, 128), what=f"token {n}")


def test_zeros_signs_and_the_scale_borders():
    k, v = torch.zeros(3, 1, 128), torch.zeros(3, 1, 128)
    k[0, 0, :4] = torch.tensor([448.0, -448.0, -0.0, 2.0 ** -10])
    k[1, 0, 0] = 450.0                                    # the next bf16: scale 2
    v[2, 0, 5] = -2.0 ** -130                             # a subnormal value alone in its page
    k, v = k.bfloat16().to(DEV), v.bfloat16().to(DEV)
    c = Cache(2, 1, [[1, 0]])
    c.append(k[:1], v[:1], [0, 1], [1], what="border")
    c.append(k[1:2], v[1:2], [0, 1], [2], what="past the border")
    c.append(k[2:], v[2:], [0, 1], [3], what="zeros")
    huge = torch.full((1, 1, 128), 3.0e38).bfloat16().to(DEV)
    c.append(huge, huge, [0, 1], [4], what="the largest values")
    c.append(k[2:], v[2:], [0, 1], [1], what="slot 0 starts the page anew")


def test_pages_outside_the_pool_and_past_the_table():
    # entries outside [0, P) and positions past max_pages are not stored; their
    # queries are rotated all the same
    c = Cache(2, 1, [[1, -1, 2, 0]])
    c.append(tokens(250, 1, 1), tokens(250, 1, 2), [0, 250], [250], rope=table(250, 128),
             q=tokens(250, 2, 3), what="bad pages")
    c = Cache(2, 1, [[1]])
    c.append(tokens(80, 1, 1), tokens(80, 1, 2), [0, 80], [100], rope=table(60, 128),
             q=tokens(80, 2, 3), what="short table")
    # more new tokens than tokens, and starts outside the packed rows
    c = Cache(2, 1, [[1], [0]])
    c.append(tokens(9, 1, 1), tokens(9, 1, 2), [-4, 5, 99], [3, 7], rope=table(60, 128),
             q=tokens(9, 2, 3), what="out of contract")


def test_in_place_queries_no_queries_and_no_tokens():
    c = Cache(1, 1, [[0]])
    k, v, q = tokens(4, 1, 1), tokens(4, 1, 2), tokens(4, 3, 3)
    cs = torch.from_numpy(table(8, 128)).to(DEV)
    start, length = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([0, 4], [6]))
    pages = torch.zeros(1, 1, dtype=torch.int32, device=DEV)
    out = sa.sparse_attn_cache_append(k, v, *c.dev, pages, start, length, rope=cs, q=q)
    before = [t.clone() for t in c.dev]
    same = q.clone()
    assert sa.sparse_attn_cache_append(k, v, *c.dev, pages, start, length, rope=cs, q=same,
                                       q_out=same) is same
    assert torch.equal(same, out)
    for a, b in zip(before, c.dev):                       # appending again changes nothing
        assert torch.equal(a, b)
    none = torch.empty(0, 1, 128, dtype=torch.bfloat16, device=DEV)
    sa.sparse_attn_cache_append(none, none, *c.dev, pages, start * 0, length)
    for a, b in zip(before, c.dev):
        assert torch.equal(a, b)


def test_whole_pages_equal_the_tile_quantisation():
    B, H, N = 1, 3, 64 * 7 + 20
    x = tokens(N, H, 4)
    k8, sk = sa.sparse_attn_quant_fp8_tiles(x.permute(1, 0, 2)[None], sa.SA_FP8_K)
    v8, sv = sa.sparse_attn_quant_fp8_tiles(x.permute(1, 0, 2)[None], sa.SA_FP8_V)
    c = Cache(8, H, [np.arange(8)])
    for t in c.dev:
        t.zero_()
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    sa.sparse_attn_cache_append(x, x, *c.dev, ints([list(range(8))]), ints([0, N]), ints([N]))
    for got, want in zip(c.dev, (k8[0], sk[0], v8[0], sv[0])):
        assert torch.equal(got, want.transpose(0, 1))


def test_captured_and_replayed():
    c = Cache(6, 2, [[3, 1, 4], [0, 2, 5]])
    k, v, q = tokens(2, 2, 1), tokens(2, 2, 2), tokens(2, 4, 3)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    pages, start, length = ints(c.pages.tolist()), ints([0, 1, 2]), ints([1, 100])
    cs = torch.from_numpy(table(200, 128)).to(DEV)
    eager = [t.clone() for t in c.dev]
    out = torch.zeros_like(q)
    call = lambda pool, to: sa.sparse_attn_cache_append(k, v, *pool, pages, start, length, rope=cs,
                                                        q=q, q_out=to)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call([t.clone() for t in c.dev], torch.zeros_like(q))
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(c.dev, out)
    want = torch.zeros_like(q)
    for step in range(70):
        for t, s in ((k, 1), (v, 2), (q, 3)):
            t.copy_(tokens(2, t.shape[1], 100 * step + s))
        graph.replay()
        call(eager, want)
        torch.cuda.synchronize()
        for a, b in zip(c.dev + [out], eager + [want]):
            assert torch.equal(a, b), step
        length += 1


@pytest.mark.parametrize("g,kv", [(9, 1), (40, 2), (130, 1)])
@pytest.mark.parametrize("n", [3, 150])
def test_many_query_heads_of_a_key_head(n, g, kv):
    # more heads than a workgroup takes at a time, and than all of them do at once
    c = Cache(4, kv, [[2, 0, 3, 1]])
    c.append(tokens(n, kv, 7), tokens(n, kv, 8), [0, n], [n + 60], rope=table(256, 128),
             q=tokens(n, kv * g, 9), what=f"{n} tokens, {kv}x{g}")
