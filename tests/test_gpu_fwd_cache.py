"""GPU attention over the paged cache against the float64 reference.

Tolerances, per element.  Scores: 128 exact products added in fp32 are off by at
most 256 half steps of 2^-24 of tau |q| |k|, and the exponent's argument by three more half steps of
its size, together below ds = 2^-15 tau |q| max|k|.  A probability is off by a
factor exp(2 ds) and rounded to bf16, half a step: 2^-8 of it.  The fp32 sums of n
terms, with the running maximum's rescaling, are off by at most n 2^-23 of their
magnitudes.  The output is rounded to bf16, half a step: 2^-8.  With a = sum p |v| / l:
  |o - o*| <= (2^-8 + 2 ds + n 2^-23) a + 2^-8 |o*|, |lse - lse*| <= 2 ds + 2^-20.
"""
import numpy as np
import pytest
import torch

import paper_2609_23153_amd as sa
from gpu_helpers import say
from oracle import kv_cache as R

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TAU = float(np.float32(1 / np.sqrt(128)))


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    sa.library()
    yield
    torch.cuda.synchronize()


def ints(v):
    return torch.as_tensor(np.asarray(v, dtype=np.int32)).to(DEV)


def make_cache(lengths, kv, seed=0, extra=2, most=None):
    """A pool whose sequences hold appended tokens; the rest of it (free pages,
    slots behind the last tokens) is filled with NaN codes."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // 64) for n in lengths]
    P = sum(need) + extra
    perm = np.random.default_rng(seed).permutation(P)
    pages = np.full((len(lengths), max(max(need), 1) if most is None else most), -1, dtype=np.int32)
    at = 0
    for b, m in enumerate(need):
        pages[b, :m] = perm[at:at + m]
        at += m
    k8, v8 = (torch.full((P, kv, 8192), 0x7F, dtype=torch.uint8, device=DEV) for _ in range(2))
    sk, sv = (torch.full((P, kv), 4.0, device=DEV) for _ in range(2))
    T = sum(lengths)
    gain = torch.exp(0.5 * torch.randn(1, kv, 128, generator=g))
    k = (torch.randn(T, kv, 128, generator=g) * gain).bfloat16().to(DEV)
    v = (torch.randn(T, kv, 128, generator=g) * torch.exp(torch.randn(T, 1, 1, generator=g)))
    start = np.concatenate([[0], np.cumsum(lengths)])
    sa.sparse_attn_cache_append(k, v.bfloat16().to(DEV), k8, sk, v8, sv, ints(pages), ints(start),
                                ints(lengths))
    return k8, sk, v8, sv, pages


def queries(T, H, seed, size=1.5):
    g = torch.Generator().manual_seed(seed)
    return (size * torch.randn(T, H, 128, generator=g)).bfloat16().to(DEV)


def compare(o, lse, q, cache, pages, start, lengths, chunk, window, tau=TAU, what=""):
    k8, sk, v8, sv = (t.cpu().numpy() for t in cache)
    args = (np.asarray(pages), start, lengths, tau, chunk, window)
    qd = q.double().cpu().numpy()
    want, want_lse = R.attend(qd, k8, sk, v8, sv, *args)
    mag, _ = R.attend(qd, k8, sk, v8 & 0x7F, sv, *args)
    o, lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
    mine = ~np.isnan(want_lse)
    used = [p for row in pages for p in row if 0 <= p < len(k8)]
    dec = lambda c, s: np.nan_to_num(R.e4m3_decode(c[used])) * s[used][..., None]
    kmax = np.sqrt((dec(k8, sk)[..., R.K_PLACE] ** 2).sum(-1)).max() if used else 0.0
    ds = 2.0 ** -15 * tau * np.linalg.norm(qd, axis=2) * kmax
    tol = ((2.0 ** -8 + 2 * ds + max(lengths) * 2.0 ** -23)[..., None] * mag
           + 2.0 ** -8 * np.abs(want) + 1e-30)
    assert np.array_equal(np.isneginf(lse[mine]), np.isneginf(want_lse[mine])), what
    none = mine & np.isneginf(want_lse)
    assert not o[none].any(), (what, "rows without keys")
    fin = mine & np.isfinite(want_lse)
    if fin.any():
        r = (np.abs(o - want) / tol)[fin].max()
        rl = (np.abs(lse - want_lse) / (2 * ds + 2.0 ** -20))[fin].max()
        say(f"  {what}: o at {r:.3f} of its bound, lse at {rl:.3f}")
        assert r <= 1 and rl <= 1, what
    return want


def run(lengths, new, kv, g, chunk=0, window=0, seed=0, front=0, back=0, size=1.5, **kw):
    k8, sk, v8, sv, pages = make_cache(lengths, kv, seed)
    start = np.concatenate([[front], front + np.cumsum(new)])
    T = int(start[-1]) + back
    q = queries(T, kv * g, seed + 1, size)
    o = torch.full((T, kv * g, 128), 9.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((T, kv * g), 9.0, device=DEV)
    sa.sparse_attn_fwd_cache(q, k8, sk, v8, sv, ints(pages), ints(start), ints(lengths), o=o, lse=lse,
                             causal=(chunk, window) if chunk else None, **kw)
    compare(o, lse, q, (k8, sk, v8, sv), pages, start, lengths, chunk, window,
            what=f"{new} of {lengths}, {kv}x{g}, causal ({chunk}, {window})")
    for rows in (slice(0, front), slice(int(start[-1]), T)):
        assert bool((o[rows] == 9.0).all()) and bool((lse[rows] == 9.0).all()), "rows of no sequence"


@pytest.mark.parametrize("g,kv", [(1, 3), (4, 2), (5, 1), (8, 1), (32, 1), (40, 1)])
@pytest.mark.parametrize("length", [1, 2, 63, 64, 65, 128, 500, 2111])
def test_one_token(length, g, kv):
    run([length], [1], kv, g, seed=length)


@pytest.mark.parametrize("chunk,window", [(0, 0), (1, 0), (1, 100), (7, 0), (64, 3), (50, 1)])
@pytest.mark.parametrize("n,length,kv,g", [(2, 2, 1, 1), (5, 70, 2, 4), (33, 33, 1, 1), (64, 64, 2, 1),
                                           (130, 131, 1, 2), (150, 700, 1, 3), (257, 300, 1, 1)])
def test_many_tokens(n, length, kv, g, chunk, window):
    run([length], [n], kv, g, chunk, window, seed=n)


@pytest.mark.parametrize("chunk,window", [(0, 0), (1, 0), (16, 2)])
def test_ragged_batch_few_rows(chunk, window):
    run([700, 1, 64, 65, 1300, 3, 0], [1, 1, 0, 4, 2, 3, 0], 2, 4, chunk, window, front=2, back=3)


@pytest.mark.parametrize("chunk,window", [(0, 0), (1, 0), (1, 90)])
def test_ragged_batch_many_rows(chunk, window):
    run([300, 1, 200, 650, 90], [300, 1, 0, 77, 3], 2, 2, chunk, window, front=1, back=130)


def test_more_than_a_wave_of_sequences():
    rng = np.random.default_rng(11)
    lengths = rng.integers(1, 130, 150).tolist()
    run(lengths, [min(n, 1 + i % 2) for i, n in enumerate(lengths)], 1, 2)


@pytest.mark.parametrize("B", [65, 4096, 5000])
def test_thousands_of_sequences(B):
    # found in one, two or three steps; a third of them get no token, some hold none
    rng = np.random.default_rng(B)
    lengths = rng.integers(0, 9, B).tolist()
    run(lengths, [min(n, int(rng.integers(0, 3))) for n in lengths], 1, 1, 1, 0, front=1, back=2)


@pytest.mark.parametrize("chunk,window", [(0, 0), (1, 0), (1, 130), (5, 3), (300, 1)])
@pytest.mark.parametrize("g,most", [(3, 4), (8, 9), (1, 60)])
def test_equal_shares_of_ragged_long_caches(g, most, chunk, window):
    # several tiles a sequence, sequences without tokens or keys, more than 64 of
    # them, lengths from none to 2,000: shares begin and end anywhere
    rng = np.random.default_rng(most)
    lengths = [0, 2000] + np.exp(rng.uniform(0, 7.6, 68)).astype(int).tolist() + [0, 0]
    new = [min(n, int(rng.integers(0, most))) for n in lengths]
    run(lengths, new, 2, g, chunk, window, seed=3, front=1, back=2)


@pytest.mark.parametrize("kv", [1, 2, 9])
def test_one_long_sequence_in_many_parts(kv):
    run([40000], [1], kv, 2, seed=5)
    run([64, 9000, 1], [1, 3, 1], kv, 2, 1, 0, seed=6)


def test_parts_beyond_a_wave_of_them():
    run([70000], [1], 1, 64, seed=7)                     # 64 rows: the many-row kernel, 136 parts
    run([262144 + 100], [1], 1, 2, seed=8)               # 512 parts
    run([30000, 0, 5], [2, 0, 1], 1, 8, 1, 20000, seed=9)  # 117 parts at most, a window of 20,000


def test_large_scores_and_a_late_maximum():
    # logits spread over hundreds: later pages move the maximum far, most
    # probabilities vanish
    run([900], [1], 2, 4, size=60.0)
    run([900], [140], 1, 1, 1, 0, size=60.0)


def test_long_cache_of_equal_keys_loses_no_mass():
    # one key far above 20,000 equal ones whose probabilities are small: each is
    # held to 2^-21 of the largest, so their sum keeps its share
    n, kv = 20001, 1
    k = torch.zeros(n, kv, 128, dtype=torch.bfloat16, device=DEV)
    v = torch.zeros(n, kv, 128, dtype=torch.bfloat16, device=DEV)
    k[0, 0, 0], v[:, 0, 0], v[0, 0, 1] = 8.0, 1.0, 1.0
    P = -(-n // 64)
    pool = [torch.zeros(P, kv, 8192, dtype=torch.uint8, device=DEV), torch.ones(P, kv, device=DEV),
            torch.zeros(P, kv, 8192, dtype=torch.uint8, device=DEV), torch.ones(P, kv, device=DEV)]
    pages = np.arange(P, dtype=np.int32)[None]
    sa.sparse_attn_cache_append(k, v, *pool, ints(pages), ints([0, n]), ints([n]))
    q = torch.zeros(1, 1, 128, dtype=torch.bfloat16, device=DEV)
    q[0, 0, 0] = 14.0                                    # logit 9.9: 2e-5 of the first key's
    o, lse = sa.sparse_attn_fwd_cache(q, *pool, ints(pages), ints([0, 1]), ints([n]))
    compare(o, lse, q, pool, pages, [0, 1], [n], 0, 0, what="equal keys")


def test_strided_queries_and_outputs_own_scale_and_wider_table():
    lengths, kv, g = [200, 90], 2, 3
    k8, sk, v8, sv, pages = make_cache(lengths, kv, 5)
    T, H = 130, kv * g
    wide = queries(T, H + 4, 6)
    q = wide[:, 2:2 + H]
    o = torch.zeros(H, T, 128, dtype=torch.bfloat16, device=DEV).transpose(0, 1)
    start = [0, 100, 130]
    table = torch.full((2, pages.shape[1] + 7), 1 << 20, dtype=torch.int32, device=DEV)
    table[:, :pages.shape[1]] = ints(pages)
    _, lse = sa.sparse_attn_fwd_cache(q, k8, sk, v8, sv, table[:, :pages.shape[1]], ints(start),
                                      ints(lengths), softmax_scale=0.2, o=o, causal=(1, 0))
    compare(o, lse, q, (k8, sk, v8, sv), pages, start, lengths, 1, 0, tau=0.2, what="strided")
    # the whole row of the table: entries behind the sequence's pages are not read
    more, _ = sa.sparse_attn_fwd_cache(q, k8, sk, v8, sv, table, ints(start), ints(lengths),
                                       softmax_scale=0.2, causal=(1, 0), with_lse=False)
    again, none = sa.sparse_attn_fwd_cache(q, k8, sk, v8, sv, table, ints(start), ints(lengths),
                                           softmax_scale=0.2, causal=(1, 0), with_lse=False)
    assert none is None and torch.equal(more, again)
    assert (more.double() - o.double()).abs().max() < 0.1


@pytest.mark.parametrize("n", [1, 40])
def test_pages_outside_the_pool_are_not_seen(n):
    k8, sk, v8, sv, pages = make_cache([700], 2, 7)
    for holes in ([0], [3, 4], list(range(11)), [10]):
        p = pages.copy()
        p[0, holes] = [-1 if i % 2 else len(k8) + i for i in range(len(holes))]
        q = queries(n, 4, 8)
        o, lse = sa.sparse_attn_fwd_cache(q, k8, sk, v8, sv, ints(p), ints([0, n]), ints([700]))
        compare(o, lse, q, (k8, sk, v8, sv), p, [0, n], [700], 0, 0, what=f"holes {holes}")


@pytest.mark.parametrize("n", [2, 90])
def test_pages_that_sequences_share(n):
    # three sequences over the same first pages, one of them naming a page twice
    k8, sk, v8, sv, pages = make_cache([700, 200], 2, 24)
    p = np.stack([pages[0], np.concatenate([pages[0, :5], pages[1, :4], [-1, -1]]),
                  np.concatenate([pages[0, :2], pages[0, :2], pages[0, 4:]])])
    lengths, start = [700, 500, 640], [0, n, 2 * n, 3 * n]
    q = queries(3 * n, 4, 25)
    for causal in (None, (1, 0)):
        o, lse = sa.sparse_attn_fwd_cache(q, k8, sk, v8, sv, ints(p), ints(start), ints(lengths),
                                          causal=causal)
        compare(o, lse, q, (k8, sk, v8, sv), p, start, lengths, *(causal or (0, 0)), what="shared pages")


@pytest.mark.parametrize("n", [3, 70])
def test_rows_that_are_not_finite_stay_alone(n):
    k8, sk, v8, sv, pages = make_cache([650], 1, 26)
    q = queries(n, 4, 27)
    call = lambda q: sa.sparse_attn_fwd_cache(q, k8, sk, v8, sv, ints(pages), ints([0, n]), ints([650]),
                                              causal=(1, 0))
    want, want_lse = call(q)
    bad = torch.zeros(n, 4, dtype=torch.bool, device=DEV)
    bad[0, 1] = bad[n // 2, 0] = bad[n - 1, 3] = True
    x = q.clone()
    x[0, 1, 5], x[n // 2, 0], x[n - 1, 3, 127] = float("nan"), float("inf"), float("-inf")
    o, lse = call(x)
    assert torch.equal(o[~bad], want[~bad]) and torch.equal(lse[~bad], want_lse[~bad])
    assert bool(o[bad].isnan().any(-1).all())


def test_two_calls_at_once_on_streams_of_their_own():
    a = make_cache([9000, 300], 2, 28), queries(2, 8, 29), ints([0, 1, 2]), ints([9000, 300])
    b = make_cache([800], 2, 30), queries(500, 8, 31), ints([0, 500]), ints([800])
    run = lambda c, q, start, lengths: sa.sparse_attn_fwd_cache(q, *c[:4], c[4], start, lengths,
                                                                causal=(1, 0))
    a, b = ((*x[0][:4], ints(x[0][4])) for x in (a, b)), (a[1:], b[1:])
    calls = [(c, *rest) for c, rest in zip(a, b)]
    want = [run(*c) for c in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    got = []
    for _ in range(3):
        for s, c in zip(streams, calls):
            with torch.cuda.stream(s):
                got.append(run(*c))
    torch.cuda.synchronize()
    for i, (o, lse) in enumerate(got):
        assert torch.equal(o, want[i % 2][0]) and torch.equal(lse, want[i % 2][1]), i


def test_window_whose_pages_are_gone():
    # generation with a sliding window frees the pages behind it
    k8, sk, v8, sv, pages = make_cache([1000], 1, 9)
    q = queries(2, 2, 10)
    call = lambda p: sa.sparse_attn_fwd_cache(q, k8, sk, v8, sv, ints(p), ints([0, 2]), ints([1000]),
                                              causal=(1, 200))
    want = call(pages)
    freed = pages.copy()
    freed[0, :(1000 - 1 - 200) // 64] = -1
    got = call(freed)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_out_of_contract_lengths_stay_in_bounds():
    # a length past the table, more new tokens than tokens, negative lengths and
    # starts outside the packed rows: rows that see no key are zero
    k8, sk, v8, sv, pages = make_cache([300, 64], 1, 12)
    q = queries(12, 2, 13)
    for start, lengths in (([0, 6, 12], [320, 64]), ([0, 6, 12], [3, 0]), ([0, 6, 12], [-5, 64]),
                           ([-3, 6, 99], [300, 64])):
        o, lse = sa.sparse_attn_fwd_cache(q, k8, sk, v8, sv, ints(pages), ints(start), ints(lengths),
                                          causal=(1, 0))
        if lengths[0] <= 300:
            compare(o, lse, q, (k8, sk, v8, sv), pages, start, lengths, 1, 0, what=f"{start} {lengths}")


def test_decreasing_starts_stay_in_bounds():
    # q_start has to be non-decreasing; where it is not, results are undefined,
    # but nothing outside the tensors is touched
    lengths = [700, 64, 300, 80]
    for most in (11, 40):                                # few rows, many rows
        k8, sk, v8, sv, pages = make_cache(lengths, 2, 18, most=most)
        for n, start in ((40, [0, 30, 10, 35, 40]), (4000, [3900, 100, 2000, 50, 4000])):
            q = queries(n, 4, 19)
            pool = [t.clone() for t in (k8, sk, v8, sv)]
            kv = queries(n, 2, 20)
            sa.sparse_attn_cache_append(kv, kv, *pool, ints(pages), ints(start), ints(lengths), q=q)
            sa.sparse_attn_fwd_cache(q, k8, sk, v8, sv, ints(pages), ints(start), ints(lengths))
    torch.cuda.synchronize()


def test_pool_beyond_32_bit_offsets():
    # the same pages at the end of a pool of 4.9 GB a tensor
    lengths, kv = [1000, 70], 8
    k8, sk, v8, sv, pages = make_cache(lengths, kv, 21)
    P, far = 75000, 75000 - len(k8)
    big = [torch.zeros(P, kv, 8192, dtype=torch.uint8, device=DEV), torch.ones(P, kv, device=DEV),
           torch.zeros(P, kv, 8192, dtype=torch.uint8, device=DEV), torch.ones(P, kv, device=DEV)]
    for t, x in zip(big, (k8, sk, v8, sv)):
        t[far:] = x
    moved = np.where(pages >= 0, pages + far, -1)
    for new in ([1, 1], [200, 33]):
        start = np.concatenate([[0], np.cumsum(new)])
        q, x = queries(sum(new), 16, 22), queries(sum(new), kv, 23)
        small = [k8.clone(), sk.clone(), v8.clone(), sv.clone()]
        sa.sparse_attn_cache_append(x, x, *small, ints(pages), ints(start), ints(lengths))
        sa.sparse_attn_cache_append(x, x, *big, ints(moved), ints(start), ints(lengths))
        for a, b in zip(big, small):
            assert torch.equal(a[far:], b)
        want = sa.sparse_attn_fwd_cache(q, *small, ints(pages), ints(start), ints(lengths), causal=(1, 0))
        got = sa.sparse_attn_fwd_cache(q, *big, ints(moved), ints(start), ints(lengths), causal=(1, 0))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        k8, sk, v8, sv = small
    assert not bool(big[0][:far].any()) and not bool(big[2][:far].any())


def test_no_tokens():
    k8, sk, v8, sv, pages = make_cache([64], 1, 14)
    q = queries(0, 2, 15)
    o, lse = sa.sparse_attn_fwd_cache(q, k8, sk, v8, sv, ints(pages), ints([0, 0]), ints([64]))
    assert o.shape == (0, 2, 128) and lse.shape == (0, 2)


@pytest.mark.parametrize("lengths,new", [([3000, 40], [1, 1]), ([500, 200], [300, 5])])
def test_captured_and_replayed_as_the_cache_grows(lengths, new):
    k8, sk, v8, sv, pages = make_cache(lengths, 2, 16, most=60)
    start, have = ints(np.concatenate([[0], np.cumsum(new)])), ints(lengths)
    # the pool's free pages take the tokens to come
    table = ints(pages)
    used = set(pages[pages >= 0].tolist())
    free = next(p for p in range(len(k8)) if p not in used)
    table[1, -(-lengths[1] // 64)] = free
    for t in (k8, v8):                                   # finite tokens where the sequence grows
        t.copy_(torch.where(t == 0x7F, torch.zeros_like(t), t))
    q = queries(sum(new), 8, 17)
    o = torch.zeros_like(q)
    lse = torch.zeros(sum(new), 8, device=DEV)
    call = lambda o, lse: sa.sparse_attn_fwd_cache(q, k8, sk, v8, sv, table, start, have, o=o, lse=lse,
                                                   causal=(1, 0))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(torch.zeros_like(o), torch.zeros_like(lse))
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(o, lse)
    for step in range(4):
        q.copy_(queries(sum(new), 8, 20 + step))
        graph.replay()
        want, want_lse = call(torch.zeros_like(o), torch.zeros_like(lse))
        torch.cuda.synchronize()
        assert torch.equal(o, want) and torch.equal(lse, want_lse), step
        have[1] += 1                                     # slot by slot into its last page
