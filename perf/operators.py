"""Performance cases of the cache and layer-norm operators.

An auto-regressive video program keeps the keys and values of the frames it
has made and attends to them from the next ones; a language model does the
same a token at a time.  The operators measured here are the ones such a
transformer block calls around its projections:

``append``    new keys and values, rotated on the way, into a paged cache of
              e4m3 codes with one power-of-two scale per page (64 tokens) and
              head; the queries are rotated in the same call
``attend``    attention of the newest tokens of every sequence over its cached
              keys (one token a sequence up to whole frames, shared key heads,
              causal windows)
``norm``      layer norm over the channels, one weight and bias per group of
              rows (a video DiT modulates them per sample)
``norm_bwd``  its gradients of the input, the weights and the biases

Where ``own`` is false every operator is computed in elementary torch
operations in 32 bits.  ``exact`` follows the definitions in 64 bits.

A page holds 8192 codes of K and 8192 of V per head: byte 16 c + e of a page
(c = 64 f + l + 32 g; l < 32, g < 2, e < 16) is, for K with f = 4 rt + 2 ks +
hf, key 32 rt + l and channel 64 ks + 32 g + 16 hf + e; for V with f = 2 dt +
hf, channel 32 dt + l and key 32 hf + 8 (e / 4) + 4 g + e % 4.
"""
import math
import random

import torch

own = False

D = 128      # head dim
PAGE = 64    # tokens per page
TINY = -126  # smallest scale exponent


# ------------------------------------------------------------------- cases
def _cache(kind, name, **kw):
    case = dict(kind=kind, batch=1, heads=12, kv_heads=12, len_min=1, len_max=4096, new_min=1,
                new_max=1, mix=1)
    case.update(dict(rope_dim=128, rows=False) if kind == "append" else dict(chunk=0, window=0))
    case.update(kw)
    return dict(case, name=name) if name else case


def _norm(kind, name, rows, cols, dtype="bf16", groups=1):
    case = dict(kind=kind, rows=rows, cols=cols, dtype=dtype, groups=groups)
    return dict(case, name=name) if name else case


def listed():
    return [
        # one new token of one sequence of the 1.3B layer (12 heads): latency counts
        _cache("append", "append_one", len_min=4095, len_max=4095),
        # a step of a serving batch: a token or a few (a verified draft) of 64
        # sequences, five query heads per key head, rotary rows given per token
        _cache("append", "append_batch", batch=64, heads=40, kv_heads=8, len_min=2, len_max=16384,
               new_max=5, mix=2, rows=True),
        # three latent frames of the 1.3B 480P layer behind the cached ones
        _cache("append", "append_frames", len_min=32760, len_max=32760, new_min=4680, new_max=4680),
        # one token of one sequence over a short cache: latency counts
        _cache("attend", "attend_one", len_min=4095, len_max=4095),
        # a step of a serving batch, ragged lengths, shared key heads
        _cache("attend", "attend_batch", batch=64, heads=40, kv_heads=8, len_min=16,
               len_max=16384, mix=3),
        # one token over half a million cached ones
        _cache("attend", "attend_long", heads=40, kv_heads=8, len_min=524288, len_max=524288),
        # prompts of odd lengths behind cached ones, token by token causal with
        # a sliding window of 1000 tokens
        _cache("attend", "attend_prompts", batch=6, heads=16, kv_heads=4, len_min=500, len_max=5003,
               new_min=17, new_max=1999, chunk=1, window=1000, mix=4),
        # the newest three latent frames of the 1.3B 480P layer over the whole
        # video, every earlier chunk visible
        _cache("attend", "attend_frames", len_min=32760, len_max=32760, new_min=4680,
               new_max=4680, chunk=4680),
        # the modulated norm before a 14B 720P block's projections
        _norm("norm", "norm_720p", 75600, 5120),
        # the same of a few tokens, fp32 residuals
        _norm("norm", "norm_few", 17, 1536, "fp32"),
        # its backward pass in training
        _norm("norm_bwd", "norm_bwd_720p", 75600, 5120),
        # a short batch of two samples with their own modulation, an odd number
        # of channels, fp32
        _norm("norm_bwd", "norm_bwd_odd", 2 * 777, 1531, "fp32", groups=2),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "attend", "norm", "norm_bwd"])
    if kind.startswith("norm"):
        cols = rng.choice([_log_int(rng, 64, 13824), 8 * _log_int(rng, 8, 1728)])
        groups = rng.choice([1, 1, 2, 3])
        rows = groups * _log_int(rng, 1, max(1, min(75600, 75600 * 5120 // cols) // groups))
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        if dtype == "fp32":
            rows = max(groups, rows // 2 // groups * groups)
        return _norm(kind, None, rows, cols, dtype, groups)
    group = rng.choice([1, 1, 2, 4, 5, 8, 16])
    kv = rng.randint(1, 12)
    batch = rng.choice([1, 1, 2, 3, _log_int(rng, 2, 96)])
    top = _log_int(rng, 1, 65536)
    new = rng.choice([1, 1, _log_int(rng, 1, min(top, 4680))])
    case = _cache(kind, None, batch=batch, heads=group * kv, kv_heads=kv, len_max=top,
                  len_min=max(1, top // rng.choice([1, 2, 50])), new_max=new,
                  new_min=max(1, new // rng.choice([1, 3, 100])), mix=rng.randint(10, 9999))
    if kind == "append":
        case["rope_dim"] = rng.choice([128, 128, 64, 0])
        case["rows"] = rng.random() < 0.4
    else:
        case["chunk"] = rng.choice([0, 1, 1, max(1, new)])
        if case["chunk"]:
            case["window"] = rng.choice([0, 0, max(1, _log_int(rng, 1, top) // case["chunk"])])
    # no more than the largest listed cases: tokens appended, cache bytes read,
    # query-key pairs
    while (kind == "append" and case["batch"] * case["new_max"] * case["heads"] > 4680 * 12
           or case["batch"] * case["len_max"] * case["kv_heads"] > 64 * 16384 * 4
           or case["batch"] * case["len_max"] * case["new_max"] * case["heads"] > 32760 * 4680 * 12):
        for f in ("batch", "len_max", "len_min", "new_max", "new_min"):
            case[f] = max(1, case[f] // 2 + case[f] % 2)
    return case


def _lengths(case):
    """(cached tokens after the call, new tokens) of every sequence."""
    rng = random.Random(case["mix"])
    total, new = [], []
    for b in range(case["batch"]):
        n = case["len_max"] if b == 0 else _log_int(rng, case["len_min"], case["len_max"])
        m = case["new_max"] if b == 0 else _log_int(rng, case["new_min"], case["new_max"])
        total.append(n)
        new.append(min(m, n))
    return total, new


def _span(case, pos, n):
    """Keys [lo, hi) that the query at position `pos` of a sequence of n sees."""
    c, w = case["chunk"], case["window"]
    if not c:
        return 0, n
    return (max(0, pos // c - w + 1) * c if w else 0), min(n, (pos // c + 1) * c)


def work(case):
    """Each input read once, each output written once; products of visible pairs."""
    if case["kind"].startswith("norm"):
        r, c, g = case["rows"], case["cols"], case["groups"]
        e = 2 if case["dtype"] == "bf16" else 4
        if case["kind"] == "norm":
            return {"bytes": 2 * e * r * c + 8 * r + 8 * g * c, "flops": 8 * r * c}
        return {"bytes": 3 * e * r * c + 8 * r + 12 * g * c, "flops": 14 * r * c}
    total, new = _lengths(case)
    h, kv, t = case["heads"], case["kv_heads"], sum(new)
    if case["kind"] == "append":
        row = 4 * case["rope_dim"] if case["rope_dim"] else 0
        return {"bytes": t * (kv * (4 * D + 2 * D) + h * 4 * D + row) + 16 * len(new) * kv,
                "flops": t * (3 * case["rope_dim"] * (h + kv) + 4 * kv * D)}
    keys = pairs = 0
    for n, m in zip(total, new):
        spans = [_span(case, n - m + i, n) for i in range(m)]
        keys += spans[-1][1] - spans[0][0]
        pairs += sum(hi - lo for lo, hi in spans)
    return {"bytes": keys * kv * (2 * D + 8 / PAGE) + t * h * (4 * D + 4),
            "flops": 4 * D * h * pairs}


# ------------------------------------------------------------------ inputs
def _gen(seed, *parts):
    s = seed & 0x7FFFFFFF
    for p in parts:
        s = (s * 1000003 + p + 12345) & 0x7FFFFFFFFFFF
    g = torch.Generator(device="cuda")
    g.manual_seed(s)
    return g


def _places():
    """Byte offset in a page of (key, channel), for K and for V: [64, 128] each."""
    key = torch.arange(PAGE, device="cuda")[:, None]
    ch = torch.arange(D, device="cuda")[None, :]
    f = 4 * (key // 32) + 2 * (ch // 64) + ch // 16 % 2
    k = 16 * (64 * f + key % 32 + 32 * (ch // 32 % 2)) + ch % 16
    f = 2 * (ch // 32) + key // 32
    e = 4 * (key // 8 % 4) + key % 4
    v = 16 * (64 * f + ch % 32 + 32 * (key // 4 % 2)) + e
    return k, v


def _exponent(amax):
    """Smallest e >= -126 with amax <= 448 * 2^e."""
    m, ex = torch.frexp(amax)
    e = ex - 9 + (m > 0.875).to(ex.dtype)
    return torch.where(amax > 0, e, torch.full_like(e, TINY)).clamp(min=TINY)


def _full_pages(x, place):
    """x [P, Hkv, 64, 128] fp32 -> (codes [P, Hkv, 8192], scales [P, Hkv])."""
    scale = torch.ldexp(torch.ones((), device="cuda"), _exponent(x.abs().amax((2, 3))))
    code = (x / scale[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    out = torch.empty(*x.shape[:2], PAGE * D, dtype=torch.uint8, device="cuda")
    out[..., place.reshape(-1)] = code.reshape(*x.shape[:2], -1)
    return out, scale


def _rope_table(rows, dim):
    """fp32 (cos, sin) [rows, dim / 2, 2] of a 3D schedule over a 30 x 52 latent grid."""
    n = torch.arange(rows, device="cuda")
    pos = torch.stack([n // 1560, n // 52 % 30, n % 52], 1).double()
    third = 2 * (D // 6)
    bands = [(0, D - 2 * third), (1, third), (2, third)]
    ang = torch.cat([pos[:, a:a + 1] * 10000.0 ** (-2 * torch.arange(w // 2, device="cuda") / w)
                     for a, w in bands], 1)[:, :dim // 2]
    return torch.stack([ang.cos(), ang.sin()], -1).float().contiguous()


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _prepare_cache(case, seed):
    total, new = _lengths(case)
    h, kv, t = case["heads"], case["kv_heads"], sum(new)
    need = [-(-n // PAGE) for n in total]
    p = sum(need) + 3
    free = torch.randperm(p, generator=_gen(seed, 1), device="cuda").to(torch.int32)
    pages = torch.full((case["batch"], max(need)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        pages[b, :n] = free[at:at + n]
        at += n
    g = _gen(seed, 2)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    gain = torch.exp(0.3 * rnd(kv, 1, D))   # channels of a trained key head differ
    pk, pv = _places()
    k8, sk = _full_pages(rnd(p, kv, PAGE, D) * gain, pk)
    v8, sv = _full_pages(rnd(p, kv, PAGE, D), pv)
    start = [0]
    for m in new:
        start.append(start[-1] + m)
    q = (1.5 * rnd(t, h, D)).bfloat16()
    s = dict(case=case, k8=k8, sk=sk, v8=v8, sv=sv, pages=pages, q_start=_ints(start),
             kv_len=_ints(total), q=q, new_max=max(new), places=(pk, pv))
    if case["kind"] == "append":
        # tokens differ in size, so that pages grow their scales now and then
        size = torch.exp(0.3 * rnd(t, 1, 1))
        s["k"] = (rnd(t, kv, D) * gain[None, :, 0] * size).bfloat16()
        s["v"] = (rnd(t, kv, D) * size).bfloat16()
        s["rope"] = _rope_table(max(total), case["rope_dim"]) if case["rope_dim"] else None
        s["rope_row"] = None
        if case["rows"]:
            s["rope_row"] = torch.randint(0, max(total), (t,), generator=g, device="cuda",
                                          dtype=torch.int32)
    return s


def _prepare_norm(case, seed):
    r, c, n = case["rows"], case["cols"], case["groups"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    g = _gen(seed, 3)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    # residual rows differ in size and mean, and a few channels stand out
    x = rnd(r, c) * torch.exp(0.5 * rnd(r, 1)) + 0.3 * rnd(r, 1)
    x[:, torch.randperm(c, generator=g, device="cuda")[:max(1, c // 1000)]] *= 20.0
    s = dict(case=case, x=x.to(dt), w=1.0 + 0.2 * rnd(n, c), b=0.2 * rnd(n, c))
    if case["kind"] == "norm_bwd":
        s["dy"] = rnd(r, c).to(dt)
        m = x.to(dt).float().mean(1)
        s["mean"] = m
        s["rstd"] = torch.rsqrt((x.to(dt).float() - m[:, None]).square().mean(1) + 1e-6)
    return s


def prepare(case, seed):
    return (_prepare_norm if case["kind"].startswith("norm") else _prepare_cache)(case, seed)


# --------------------------------------------------------- the plain forms
def _tokens(s, t):
    """(sequence, position) of every new token."""
    tok = torch.arange(t, device="cuda")
    b = torch.searchsorted(s["q_start"], tok, right=True) - 1
    return b, s["kv_len"][b] - s["q_start"][b + 1] + tok


def _rotate(x, cs):
    """Pairs (2m, 2m + 1) of x [T, H, 128] turned by (cos, sin) cs [T, r / 2, 2]."""
    r = 2 * cs.shape[1]
    a, b = x[..., 0:r:2].float(), x[..., 1:r:2].float()
    c, d = cs[:, None, :, 0], cs[:, None, :, 1]
    out = torch.stack([a * c - b * d, a * d + b * c], -1).flatten(2)
    return torch.cat([out, x[..., r:].float()], 2)


def _store(x, code, scale, place, b, page, slot, first, s0):
    """x [T, Hkv, 128] fp32 into its pages: scales first, then codes."""
    p, kv = scale.shape
    amax = torch.zeros(p, kv, device="cuda")
    amax.scatter_reduce_(0, page[:, None].expand(-1, kv), x.abs().amax(2), "amax")
    low = torch.full((p,), PAGE, device="cuda")
    low.scatter_reduce_(0, page, slot, "amin")
    need, held = _exponent(amax), torch.frexp(scale)[1] - 1
    e = torch.where(low[:, None] == 0, need, torch.maximum(need, held))
    e = torch.where(low[:, None] == PAGE, held, e)
    # the tokens that a page held before, on its new scale
    old = code[first][..., place]                               # [B, Hkv, 64, 128]
    val = torch.ldexp(old.view(torch.float8_e4m3fn).float(), (held - e)[first][..., None, None])
    again = val.to(torch.float8_e4m3fn).view(torch.uint8)
    before = torch.arange(PAGE, device="cuda")[:, None] < s0[:, None, None, None]
    code[first[:, None, None], torch.arange(kv, device="cuda")[None, :, None],
         place.reshape(-1)] = torch.where(before, again, old).flatten(2)
    c = torch.ldexp(x, -e[page][..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
    code[page[:, None, None], torch.arange(kv, device="cuda")[None, :, None],
         place[slot][:, None, :]] = c
    scale.copy_(torch.ldexp(torch.ones_like(scale), e))


def _plain_append(s):
    t = s["k"].shape[0]
    b, pos = _tokens(s, t)
    k, q = s["k"].float(), s["q"].float()
    if s["rope"] is not None:
        cs = s["rope"][pos if s["rope_row"] is None else s["rope_row"].long()]
        k, q = _rotate(s["k"], cs), _rotate(s["q"], cs)
    page, slot = s["pages"][b, pos // PAGE].long(), pos % PAGE
    p0 = s["kv_len"] - s["q_start"][1:] + s["q_start"][:-1]   # first new position
    first = s["pages"].gather(1, (p0 // PAGE)[:, None].long())[:, 0].long()
    for x, code, scale, place in ((k, s["k8"], s["sk"], s["places"][0]),
                                  (s["v"].float(), s["v8"], s["sv"], s["places"][1])):
        _store(x, code, scale, place, b, page, slot, first, p0 % PAGE)
    return q.bfloat16()


def _plain_attend(s):
    case = s["case"]
    t, h, _ = s["q"].shape
    bsz, kv, n = case["batch"], case["kv_heads"], s["new_max"]
    length = s["kv_len"].long()
    new = (s["q_start"][1:] - s["q_start"][:-1]).long()
    i = torch.arange(n, device="cuda")
    rows = (s["q_start"][:-1, None] + i).clamp(max=t - 1).long()          # [B, n]
    pg = s["pages"].clamp(min=0).long()
    keys = pg.shape[1] * PAGE

    def held(code, scale, place):
        x = code[pg][..., place].view(torch.float8_e4m3fn).float() * scale[pg][..., None, None]
        return x.permute(0, 2, 1, 3, 4).reshape(bsz, kv, keys, D)

    q = s["q"][rows].float().view(bsz, n, kv, h // kv, D).permute(0, 2, 3, 1, 4)
    q = q.reshape(bsz, kv, -1, D) / math.sqrt(D)
    x = torch.matmul(q, held(s["k8"], s["sk"], s["places"][0]).transpose(2, 3).contiguous())
    pos = (length - new)[:, None] + i                                     # [B, n]
    lo, hi = torch.zeros_like(pos), length[:, None].expand_as(pos)
    if case["chunk"]:
        c = pos // case["chunk"]
        hi = torch.minimum(hi, (c + 1) * case["chunk"])
        if case["window"]:
            lo = ((c - case["window"] + 1) * case["chunk"]).clamp(min=0)
    j = torch.arange(keys, device="cuda")
    seen = (j >= lo[..., None]) & (j < hi[..., None])                     # [B, n, keys]
    x = x.view(bsz, kv, h // kv, n, keys).masked_fill_(~seen[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    x = x.sub_(m).exp_()
    l = x.sum(-1)
    o = torch.matmul(x.view(bsz, kv, -1, keys), held(s["v8"], s["sv"], s["places"][1]))
    o = o.view(bsz, kv, -1, n, D) / l[..., None]
    lse = m[..., 0] + l.log()
    there = (i < new[:, None]).reshape(-1)                                # of [B, n]
    # every sequence's surplus rows go to one row behind the last token
    to = torch.where(there, rows.reshape(-1), torch.full_like(rows.reshape(-1), t))
    out = torch.zeros(t + 1, h, D, dtype=torch.bfloat16, device="cuda")
    out_lse = torch.zeros(t + 1, h, device="cuda")
    out[to] = o.permute(0, 3, 1, 2, 4).reshape(-1, h, D).bfloat16()
    out_lse[to] = lse.permute(0, 3, 1, 2).reshape(-1, h)
    return out[:t], out_lse[:t]


def _grouped(case, v):
    """A weight [G, cols] as one that multiplies [G, rows / G, cols]."""
    return v.view(case["groups"], 1, -1)


def _plain_norm(s):
    case, x = s["case"], s["x"].float()
    m = x.mean(1, keepdim=True)
    d = x - m
    r = torch.rsqrt(d.square().mean(1, keepdim=True) + 1e-6)
    y = (d * r).view(case["groups"], -1, case["cols"]) * _grouped(case, s["w"])
    return (y + _grouped(case, s["b"])).view_as(x).to(s["x"].dtype), m[:, 0], r[:, 0]


def _plain_norm_bwd(s):
    case = s["case"]
    xh = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    dy = s["dy"].float()
    by = lambda v: v.view(case["groups"], -1, case["cols"])
    dw, db = (by(dy) * by(xh)).sum(1), by(dy).sum(1)
    g = (by(dy) * _grouped(case, s["w"])).view_as(xh)
    dx = g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)
    return (dx * s["rstd"][:, None]).to(s["x"].dtype), dw, db


# --------------------------------------------------------------- the calls
def run(state):
    s, kind = state, state["case"]["kind"]
    if own:
        import paper_2609_23153_amd as sa
    if kind == "append":
        if own:
            q = sa.sparse_attn_cache_append(s["k"], s["v"], s["k8"], s["sk"], s["v8"], s["sv"],
                                            s["pages"], s["q_start"], s["kv_len"], rope=s["rope"],
                                            rope_row=s["rope_row"], q=s["q"])
        else:
            q = _plain_append(s)
        return dict(q=q, k=s["k8"].view(torch.float8_e4m3fn), v=s["v8"].view(torch.float8_e4m3fn),
                    sk=s["sk"], sv=s["sv"])
    if kind == "attend":
        if own:
            c = s["case"]
            o, lse = sa.sparse_attn_fwd_cache(
                s["q"], s["k8"], s["sk"], s["v8"], s["sv"], s["pages"], s["q_start"], s["kv_len"],
                causal=(c["chunk"], c["window"]) if c["chunk"] else None)
        else:
            o, lse = _plain_attend(s)
        return dict(o=o, lse=lse)
    if kind == "norm":
        if own:
            y, mean, rstd = sa.sparse_attn_layer_norm(s["x"], s["w"], s["b"], eps=1e-6)
        else:
            y, mean, rstd = _plain_norm(s)
        return dict(y=y, mean=mean, rstd=rstd)
    if own:
        dx, dw, db = sa.sparse_attn_layer_norm_bwd(s["dy"], s["x"], s["mean"], s["rstd"], s["w"])
    else:
        dx, dw, db = _plain_norm_bwd(s)
    return dict(dx=dx, dw=dw, db=db)


# ------------------------------------------------- the definitions in 64 bits
def _exact_append(case, s):
    total, new = _lengths(case)
    rope = s["rope"].double() if s["rope"] is not None else None

    def turned(x, row):
        x = x.double()
        if rope is not None:
            r = rope.shape[1]
            z = torch.view_as_complex(x[..., :2 * r].reshape(*x.shape[:2], r, 2).contiguous())
            w = torch.view_as_complex(rope[row].contiguous())
            x[..., :2 * r] = torch.view_as_real(z * w[:, None]).flatten(2)
        return x

    def encode(x):
        return x.float().to(torch.float8_e4m3fn)

    q_out = torch.empty_like(s["q"], dtype=torch.float64)
    kc, vc = (s[n].view(torch.float8_e4m3fn).clone() for n in ("k8", "v8"))
    sk, sv = s["sk"].double(), s["sv"].double()
    at = 0
    for b, (n, m) in enumerate(zip(total, new)):
        row = torch.arange(n - m, n, device="cuda")
        if s["rope_row"] is not None:
            row = s["rope_row"][at:at + m].long()
        k, v = turned(s["k"][at:at + m], row), s["v"][at:at + m].double()
        q_out[at:at + m] = turned(s["q"][at:at + m], row)
        for j in range((n - m) // PAGE, (n - 1) // PAGE + 1):
            page = int(s["pages"][b, j])
            a, z = max(n - m, j * PAGE), min(n, (j + 1) * PAGE)
            s0 = a - j * PAGE
            for x, c, sc, place in ((k, kc, sk, s["places"][0]), (v, vc, sv, s["places"][1])):
                part = x[a - (n - m):z - (n - m)].transpose(0, 1)            # [Hkv, tokens, 128]
                amax = part.abs().amax((1, 2))
                e = torch.ceil(torch.log2(amax / 448)).clamp(min=TINY)
                e = torch.where(amax > 448 * torch.exp2(e), e + 1, e)
                e = torch.where((amax <= 448 * torch.exp2(e - 1)) & (e > TINY), e - 1, e)
                scale = torch.exp2(e)
                tile = c[page][:, place].double()                           # [Hkv, 64, 128]
                if s0:
                    scale = torch.maximum(scale, sc[page])
                    tile[:, :s0] *= (sc[page] / scale)[:, None, None]
                tile[:, s0:s0 + z - a] = part / scale[:, None, None]
                c.view(torch.uint8)[page, :, place.reshape(-1)] = \
                    encode(tile).view(torch.uint8).flatten(1)
                sc[page] = scale
        at += m
    return dict(q=q_out, k=kc.double(), v=vc.double(), sk=sk, sv=sv)


def _exact_attend(case, s):
    total, new = _lengths(case)
    h, kv = case["heads"], case["kv_heads"]
    g = h // kv
    o = torch.empty(sum(new), h, D, dtype=torch.float64, device="cuda")
    lse = torch.empty(sum(new), h, dtype=torch.float64, device="cuda")
    at = 0
    for b, (n, m) in enumerate(zip(total, new)):
        pg = s["pages"][b, :-(-n // PAGE)].long()
        pos = torch.arange(n - m, n, device="cuda")
        j = torch.arange(n, device="cuda")
        seen = torch.ones(m, n, dtype=torch.bool, device="cuda")
        if case["chunk"]:
            ago = pos[:, None] // case["chunk"] - j[None] // case["chunk"]
            seen = (ago >= 0) & (ago < (case["window"] or n + 1))
        for i in range(kv):
            val = lambda c, sc, place: (s[c][pg, i][:, place].view(torch.float8_e4m3fn).double()
                                        * s[sc][pg, i].double()[:, None, None]).view(-1, D)[:n]
            k, v = val("k8", "sk", s["places"][0]), val("v8", "sv", s["places"][1])
            step = max(1, 2 ** 27 // n)
            for x in range(i * g, i * g + g):
                for r in range(0, m, step):
                    z = s["q"][at + r:at + min(r + step, m), x].double() @ k.T / math.sqrt(D)
                    z = z.masked_fill(~seen[r:r + step], -math.inf)
                    to = torch.logsumexp(z, 1)
                    lse[at + r:at + min(r + step, m), x] = to
                    o[at + r:at + min(r + step, m), x] = torch.exp(z - to[:, None]) @ v
        at += m
    return dict(o=o, lse=lse)


def _exact_norm(case, s):
    n = case["groups"]
    x = s["x"].double().view(n, -1, case["cols"])
    var, mean = torch.var_mean(x, 2, correction=0)
    if case["kind"] == "norm":
        rstd = (var + 1e-6) ** -0.5
        y = (x - mean[..., None]) * (rstd[..., None] * s["w"].double()[:, None])
        return dict(y=(y + s["b"].double()[:, None]).view_as(s["x"]), mean=mean.view(-1),
                    rstd=rstd.view(-1))
    rstd = s["rstd"].double().view(n, -1, 1)
    xh = (x - s["mean"].double().view(n, -1, 1)) * rstd
    dy = s["dy"].double().view_as(x)
    up = dy * s["w"].double()[:, None]
    along = torch.linalg.vecdot(up, xh, dim=2)[..., None] / case["cols"]
    dx = rstd * (up - up.mean(2, keepdim=True) - along * xh)
    return dict(dx=dx.view_as(s["x"]), dw=torch.linalg.vecdot(dy, xh, dim=1), db=dy.sum(1))


def exact(case, seed):
    if case["kind"].startswith("norm"):
        return _exact_norm(case, _prepare_norm(case, seed))
    s = _prepare_cache(case, seed)
    return (_exact_append if case["kind"] == "append" else _exact_attend)(case, s)
