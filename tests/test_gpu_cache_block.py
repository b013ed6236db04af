"""The operators of one auto-regressive attention block together, as a program
calls them: layer norm, per-token quantisation and W8A8 projection, rotation
and append to the paged cache, attention over it, output projection; a prompt,
then token by token, and the same as one sequence without a cache.

Tolerances.  The stages agree with the float64 chain on the stages' own inputs
(each kernel's bound is tested apart); here the whole chain of one call is
compared with the chain run in another split of the same tokens: q, k, v are
the same bytes (rows do not depend on the batch), so only the pages' scales
(grown token by token or set at once) and the order of the keys' sums differ.
A key's code may round on a larger scale by the way, half a step: 2^-4 of the
value at most once more, so o stays within 2^-3 of its magnitude sums.
"""
import math

import numpy as np
import pytest
import torch

import oracle as O
import paper_2609_23153_amd as sa
from gpu_helpers import say
from oracle import kv_cache as RC
from oracle import layer_norm as RN

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
D, H, KV = 512, 4, 2      # model width, query heads, key heads


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    sa.library()
    yield
    torch.cuda.synchronize()


def ints(v):
    return torch.as_tensor(np.asarray(v, dtype=np.int32)).to(DEV)


class Block:
    def __init__(self, sequences, pages):
        g = torch.Generator().manual_seed(0)
        rnd = lambda *s: torch.randn(*s, generator=g)
        quant = lambda n, k: sa.sparse_attn_quant_rows_fp8((rnd(n, k) / math.sqrt(k)).bfloat16().to(DEV))
        self.gamma, self.beta = (1 + 0.2 * rnd(D)).to(DEV), (0.1 * rnd(D)).to(DEV)
        self.qkv, self.out = quant((H + 2 * KV) * 128, D), quant(D, H * 128)
        ang = np.arange(400)[:, None] * 10000.0 ** (-np.arange(64) / 64)
        self.rope = torch.from_numpy(np.stack([np.cos(ang), np.sin(ang)], -1).astype(np.float32)).to(DEV)
        P = sequences * pages
        self.pages = ints(np.random.default_rng(1).permutation(P).reshape(sequences, pages))
        self.pool = [torch.zeros(P, KV, 8192, dtype=torch.uint8, device=DEV), torch.ones(P, KV, device=DEV),
                     torch.zeros(P, KV, 8192, dtype=torch.uint8, device=DEV), torch.ones(P, KV, device=DEV)]

    def __call__(self, x, start, length, keep=None):
        y, _, _ = sa.sparse_attn_layer_norm(x, self.gamma, self.beta)
        a = sa.sparse_attn_linear_w8a8(*sa.sparse_attn_quant_rows_fp8(y), *self.qkv)
        qkv = a.view(len(x), H + 2 * KV, 128)
        q = sa.sparse_attn_cache_append(qkv[:, H:H + KV], qkv[:, H + KV:], *self.pool, self.pages, start,
                                        length, rope=self.rope, q=qkv[:, :H])
        o, lse = sa.sparse_attn_fwd_cache(q, *self.pool, self.pages, start, length, causal=(1, 0))
        z = sa.sparse_attn_linear_w8a8(*sa.sparse_attn_quant_rows_fp8(o.view(len(x), -1)), *self.out)
        if keep is not None:
            keep.update(y=y, a=a, q=q, o=o, lse=lse)
        return x + z


def test_block_prompt_and_tokens():
    totals, prompt = [150, 70], [140, 61]
    g = torch.Generator().manual_seed(5)
    xs = [torch.randn(n, D, generator=g).bfloat16().to(DEV) for n in totals]
    whole = Block(2, 3)
    keep = {}
    want = whole(torch.cat(xs), ints([0, 150, 220]), ints(totals), keep)
    # the first stages of that call against the references, on its own inputs
    x = torch.cat(xs).double().cpu().numpy()
    ry, _, _ = RN.layer_norm(x, whole.gamma.double().cpu().numpy(), whole.beta.double().cpu().numpy())
    assert np.abs(keep["y"].double().cpu().numpy() - ry).max() <= 2.0 ** -8 * np.abs(ry).max() + 1e-4
    tau = float(np.float32(1 / math.sqrt(128)))
    pool = [t.cpu().numpy() for t in whole.pool]
    ro, rl = RC.attend(keep["q"].double().cpu().numpy(), *pool, whole.pages.cpu().numpy(), [0, 150, 220],
                       totals, tau, 1, 0)
    mag, _ = RC.attend(keep["q"].double().cpu().numpy(), pool[0], pool[1], pool[2] & 0x7F, pool[3],
                       whole.pages.cpu().numpy(), [0, 150, 220], totals, tau, 1, 0)
    assert np.all(np.abs(keep["o"].double().cpu().numpy() - ro) <= 2.0 ** -7 * mag + 2.0 ** -8 * np.abs(ro))
    assert np.abs(keep["lse"].double().cpu().numpy() - rl).max() < 1e-3
    # a prompt, then token by token
    split = Block(2, 3)
    kept, got = {}, []
    got.append(split(torch.cat([x[:n] for x, n in zip(xs, prompt)]), ints([0, 140, 201]), ints(prompt), kept))
    lengths = list(prompt)
    rows = []
    while lengths != totals:
        new = [int(n < t) for n, t in zip(lengths, totals)]
        at = [n for n in lengths]
        lengths = [n + m for n, m in zip(lengths, new)]
        step = torch.cat([x[n:n + m] for x, n, m in zip(xs, at, new)])
        split(step, ints([0, new[0], sum(new)]), ints(lengths), kept)
        for b, r in zip([b for b in (0, 1) if new[b]], range(sum(new))):
            rows.append((b, at[b], kept["q"][r].clone(), kept["o"][r].clone()))
    for b, pos, q, o in rows:
        row = (0, 150)[b] + pos
        assert torch.equal(q, keep["q"][row]), "the same bytes whatever the batch"
        err = (o.double() - keep["o"][row].double()).abs().cpu().numpy()
        assert np.all(err <= 2.0 ** -3 * mag[row] + 2.0 ** -7), (b, pos)
    say(f"  {len(rows)} tokens after prompts of {prompt}: equal queries, attention within its bound")


def test_block_step_captured_while_the_cache_grows():
    eager, graphed = Block(2, 3), Block(2, 3)
    g = torch.Generator().manual_seed(6)
    prompt = torch.randn(100, D, generator=g).bfloat16().to(DEV)
    start = ints([0, 60, 100])
    for blk in (eager, graphed):
        blk(prompt, start, ints([60, 40]))
    x, one, length = torch.zeros(2, D, dtype=torch.bfloat16, device=DEV), ints([0, 1, 2]), ints([61, 41])
    scratch = Block(2, 3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        scratch(x, one, length)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = graphed(x, one, length)
    for step in range(12):
        x.copy_(torch.randn(2, D, generator=g).bfloat16())
        graph.replay()
        want = eager(x, one, length)
        torch.cuda.synchronize()
        assert torch.equal(out, want), step
        for a, b in zip(eager.pool, graphed.pool):
            assert torch.equal(a, b), step
        length += 1


def test_norm_trains_with_the_sparse_branch():
    # the norm's gradients behind the sparse attention's: q = k = v heads of one
    # normed input; dx, dweight, dbias against float64 of the same chain
    N, heads = 256, 2
    g = torch.Generator().manual_seed(7)
    x = torch.randn(N, heads * 128, generator=g).bfloat16().to(DEV)
    w, b = (1 + 0.2 * torch.randn(heads * 128, generator=g)).to(DEV), torch.zeros(heads * 128, device=DEV)
    y, mean, rstd = sa.sparse_attn_layer_norm(x, w, b)
    q = y.view(1, N, heads, 128).transpose(1, 2)
    idx, cnt = sa.sparse_attn_select(q, q, 2)
    o, lse = sa.sparse_attn_fwd(q, q, q, idx, cnt, o=torch.empty_like(q))
    d_o = torch.randn(1, N, heads, 128, generator=g).bfloat16().to(DEV).transpose(1, 2)
    grads = sa.sparse_attn_bwd(q, q, q, o, d_o, lse, idx, cnt)
    dy = sum(t.float() for t in grads).bfloat16().transpose(1, 2).reshape(N, heads * 128).contiguous()
    dx, dw, db = sa.sparse_attn_layer_norm_bwd(dy, x, mean, rstd, w)
    rdx, rdw, rdb = RN.layer_norm_bwd(dy.double().cpu().numpy(), x.double().cpu().numpy(),
                                      mean.double().cpu().numpy(), rstd.double().cpu().numpy(),
                                      w.double().cpu().numpy())
    near = lambda a, r, rel: np.abs(a.double().cpu().numpy() - r).max() <= rel * np.abs(r).max()
    assert near(dx, rdx, 2.0 ** -8 + 1e-4) and near(dw, rdw[0], 1e-4) and near(db, rdb[0], 1e-4)
