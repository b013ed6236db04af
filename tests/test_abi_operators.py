"""Refusals of the layer-norm and cache calls: every bad argument is turned
down on the host before any HIP call (so these run without a GPU)."""
import ctypes

import pytest
import torch

import paper_2609_23153_amd as sa

P = ctypes.c_void_p(1 << 20)     # aligned, never dereferenced: every call fails its checks
ODD = ctypes.c_void_p((1 << 20) + 1)
MIS = ctypes.c_void_p((1 << 20) + 2)
WS = 1 << 40
INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3


def norm(dtype=0, x=P, ldx=64, rows=4, cols=64, groups=1, w=None, b=None, eps=1e-6, y=P, ldy=64,
         mean=None, rstd=None):
    return sa.library().sparse_attn_layer_norm(dtype, x, ldx, rows, cols, groups, w, b, eps, y, ldy,
                                               mean, rstd, None)


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=2), INVALID), (dict(dtype=-1), INVALID), (dict(x=None), INVALID),
    (dict(y=None), INVALID), (dict(x=ODD), INVALID), (dict(x=MIS, dtype=1), INVALID),
    (dict(ldx=63), INVALID), (dict(ldy=63), INVALID), (dict(rows=-1), INVALID),
    (dict(cols=0), INVALID), (dict(groups=0), INVALID), (dict(groups=3), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(w=MIS), INVALID), (dict(b=MIS), INVALID), (dict(mean=MIS), INVALID),
    (dict(rstd=MIS), INVALID), (dict(ldx=65), INVALID),  # y is x with another stride
    (dict(cols=16385, ldx=16385, ldy=16385), UNSUPPORTED),
    (dict(rows=65536, groups=65536), UNSUPPORTED), (dict(rows=1 << 41), UNSUPPORTED),
])
def test_layer_norm_refuses(kw, want):
    assert norm(**kw) == want


def norm_bwd(dtype=0, dy=P, lddy=64, x=P, ldx=64, mean=P, rstd=P, rows=4, cols=64, groups=1, w=None,
             dx=P, lddx=64, dw=P, db=P, ws=P, ws_bytes=WS):
    return sa.library().sparse_attn_layer_norm_bwd(dtype, dy, lddy, x, ldx, mean, rstd, rows, cols,
                                                   groups, w, dx, lddx, dw, db, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=7), INVALID), (dict(dy=None), INVALID), (dict(x=None), INVALID),
    (dict(dx=None), INVALID), (dict(mean=None), INVALID), (dict(rstd=None), INVALID),
    (dict(lddy=60), INVALID), (dict(lddx=0), INVALID), (dict(rows=5, groups=2), INVALID),
    (dict(ws=None), INVALID), (dict(ws=None, dw=None), INVALID), (dict(ws=MIS), INVALID),
    (dict(dw=MIS), INVALID), (dict(db=ODD), INVALID), (dict(ws_bytes=16), WORKSPACE),
    (dict(lddx=72), INVALID), (dict(cols=20000, lddy=20000, ldx=20000, lddx=20000), UNSUPPORTED),
])
def test_layer_norm_bwd_refuses(kw, want):
    assert norm_bwd(**kw) == want


def test_layer_norm_workspace():
    size = sa.library().sparse_attn_layer_norm_bwd_workspace_size
    assert size(0, 64, 1) == 2 * 64 * 4         # one (empty) team
    assert size(-1, 64, 1) == size(4, 0, 1) == size(4, 64, 3) == size(4, 64, 0) == 0
    assert size(1 << 30, 5120, 1) < 1 << 30     # teams are bounded


@pytest.mark.parametrize("bad", [
    dict(x=torch.zeros(4, 8, dtype=torch.float16)), dict(x=torch.zeros(2, 4, 8)),
    dict(x=torch.zeros(8, 4).t()), dict(weight=torch.ones(7)),
    dict(weight=torch.ones(8, dtype=torch.bfloat16)), dict(bias=torch.ones(3, 8)),
    dict(weight=torch.ones(2, 8), bias=torch.ones(8)), dict(y=torch.zeros(4, 9)),
    dict(y=torch.zeros(4, 8, dtype=torch.bfloat16)),
])
def test_layer_norm_binding_refuses(bad):
    args = dict(x=torch.zeros(4, 8))
    args.update(bad)
    with pytest.raises(ValueError):
        sa.sparse_attn_layer_norm(**args)


@pytest.mark.parametrize("bad", [
    dict(dy=torch.zeros(4, 7)), dict(dy=torch.zeros(4, 8, dtype=torch.bfloat16)),
    dict(mean=torch.zeros(5)), dict(rstd=torch.zeros(4, dtype=torch.float64)), dict(groups=3),
    dict(weight=torch.ones(2, 8), groups=1), dict(dx=torch.zeros(3, 8)),
])
def test_layer_norm_bwd_binding_refuses(bad):
    args = dict(dy=torch.zeros(4, 8), x=torch.zeros(4, 8), mean=torch.zeros(4), rstd=torch.ones(4))
    args.update(bad)
    with pytest.raises(ValueError):
        sa.sparse_attn_layer_norm_bwd(**args)


# ------------------------------------------------------------- paged cache
def cache_desc(**kw):
    d = sa.SparseAttnCacheDesc()
    f = dict(batch=2, heads=8, kv_heads=4, head_dim=128, tokens=6, num_pages=5, max_pages=3,
             pages_stride=3, q_stride=(1024, 128), k_stride=(512, 128), v_stride=(512, 128),
             o_stride=(1024, 128), softmax_scale=0.0, causal_chunk=0, causal_window=0)
    f.update(kw)
    for name, value in f.items():
        if isinstance(value, tuple):
            getattr(d, name)[:] = value
        else:
            setattr(d, name, value)
    return d


BAD_CACHE_DESCS = [
    (dict(batch=0), INVALID), (dict(heads=6), INVALID), (dict(kv_heads=0), INVALID),
    (dict(tokens=-1), INVALID), (dict(num_pages=0), INVALID), (dict(max_pages=0), INVALID),
    (dict(pages_stride=2), INVALID), (dict(head_dim=64), UNSUPPORTED),
    (dict(causal_chunk=-1), INVALID), (dict(causal_window=3), INVALID),
    (dict(softmax_scale=-1.0), INVALID), (dict(softmax_scale=float("nan")), INVALID),
    (dict(max_pages=1 << 24, pages_stride=1 << 24), UNSUPPORTED),
    (dict(tokens=(1 << 27) + 1), UNSUPPORTED), (dict(batch=1 << 22), UNSUPPORTED),
    (dict(tokens=(1 << 25) + 1), UNSUPPORTED), (dict(batch=(1 << 19) + 1), UNSUPPORTED),
    (dict(o_stride=(0, 128)), INVALID), (dict(o_stride=(1024, 120)), INVALID),   # rows overlap
]


def append(desc=None, k=P, v=P, rope=P, rope_rows=9, rope_dim=128, rope_row=None, q=P, q_out=P,
           k8=P, sk=P, v8=P, sv=P, pages=P, q_start=P, kv_len=P, **kw):
    d = cache_desc(**kw)
    return sa.library().sparse_attn_cache_append(
        None if desc == "null" else ctypes.byref(d), k, v, rope, rope_rows, rope_dim, rope_row, q,
        q_out, k8, sk, v8, sv, pages, q_start, kv_len, None)


@pytest.mark.parametrize("kw,want", BAD_CACHE_DESCS + [
    (dict(desc="null"), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID),
    (dict(k=MIS), INVALID), (dict(v=MIS), INVALID), (dict(q=None), INVALID),
    (dict(q_out=None), INVALID), (dict(q=MIS), INVALID), (dict(q_out=MIS), INVALID),
    (dict(q_stride=(1024, 136)), INVALID),           # q_out is q with other strides
    (dict(q_stride=(1020, 128)), INVALID), (dict(o_stride=(1024, 4)), INVALID),
    (dict(k_stride=(-512, 128)), INVALID), (dict(v_stride=(512, 129)), INVALID),
    (dict(rope=MIS), INVALID), (dict(rope_dim=130), INVALID), (dict(rope_dim=12), INVALID),
    (dict(rope_dim=0), INVALID), (dict(rope_rows=-1), INVALID), (dict(rope_row=ODD), INVALID),
    (dict(k8=None), INVALID), (dict(v8=MIS), INVALID), (dict(sk=None), INVALID),
    (dict(sv=ODD), INVALID), (dict(pages=None), INVALID), (dict(pages=MIS), INVALID),
    (dict(q_start=None), INVALID), (dict(kv_len=None), INVALID),
])
def test_cache_append_refuses(kw, want):
    assert append(**kw) == want


def cache_args():
    """Tensors of a valid append (on the CPU: never launched)."""
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    return dict(k=bf(6, 4, 128), v=bf(6, 4, 128), k8=torch.zeros(5, 4, 8192, dtype=torch.uint8),
                sk=torch.ones(5, 4), v8=torch.zeros(5, 4, 8192, dtype=torch.uint8),
                sv=torch.ones(5, 4), pages=i32(2, 3), q_start=i32(3), kv_len=i32(2))


BAD_CACHE_TENSORS = [
    dict(k8=torch.zeros(5, 4, 8192)), dict(k8=torch.zeros(5, 4, 4096, dtype=torch.uint8)),
    dict(v8=torch.zeros(4, 4, 8192, dtype=torch.uint8)), dict(sk=torch.ones(5, 3)),
    dict(sv=torch.ones(5, 4, dtype=torch.float64)), dict(pages=torch.zeros(2, 3)),
    dict(pages=torch.zeros(3, 2, dtype=torch.int32).t()), dict(kv_len=torch.zeros(3, dtype=torch.int32)),
    dict(q_start=torch.zeros(2, dtype=torch.int32)), dict(kv_len=torch.zeros(2, dtype=torch.int64)),
]


@pytest.mark.parametrize("bad", BAD_CACHE_TENSORS + [
    dict(k=torch.zeros(6, 4, 128)), dict(k=torch.zeros(6, 4, 64, dtype=torch.bfloat16)),
    dict(v=torch.zeros(5, 4, 128, dtype=torch.bfloat16)),
    dict(k=torch.zeros(6, 3, 128, dtype=torch.bfloat16), v=torch.zeros(6, 3, 128, dtype=torch.bfloat16)),
    dict(q=torch.zeros(6, 6, 128, dtype=torch.bfloat16)),
    dict(q=torch.zeros(5, 8, 128, dtype=torch.bfloat16)),
    dict(q_out=torch.zeros(6, 8, 128, dtype=torch.bfloat16)),
    dict(rope=torch.zeros(9, 64)), dict(rope=torch.zeros(9, 72, 2)), dict(rope=torch.zeros(9, 6, 2)),
    dict(rope=torch.zeros(9, 64, 2, dtype=torch.float64)),
    dict(rope_row=torch.zeros(6, dtype=torch.int32)),
    dict(rope=torch.zeros(9, 64, 2), rope_row=torch.zeros(5, dtype=torch.int32)),
    dict(rope=torch.zeros(9, 64, 2), rope_row=torch.zeros(6, dtype=torch.int64)),
])
def test_cache_append_binding_refuses(bad):
    args = cache_args()
    args.update(bad)
    with pytest.raises(ValueError):
        sa.sparse_attn_cache_append(**args)


def fwd_cache(desc=None, q=P, k8=P, sk=P, v8=P, sv=P, pages=P, q_start=P, kv_len=P,
              o=ctypes.c_void_p(1 << 21), lse=P, ws=P, ws_bytes=WS, **kw):
    d = cache_desc(**kw)
    return sa.library().sparse_attn_fwd_cache(
        None if desc == "null" else ctypes.byref(d), q, k8, sk, v8, sv, pages, q_start, kv_len, o,
        lse, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,want", BAD_CACHE_DESCS + [
    (dict(desc="null"), INVALID), (dict(q=None), INVALID), (dict(o=None), INVALID),
    (dict(o=P), INVALID),                            # o is q
    (dict(q=MIS), INVALID), (dict(o=MIS), INVALID), (dict(lse=MIS), INVALID),
    (dict(ws=None), INVALID), (dict(ws=MIS), INVALID), (dict(ws_bytes=8), WORKSPACE),
    (dict(q_stride=(1024, 12)), INVALID), (dict(o_stride=(-8, 128)), INVALID),
    (dict(k8=MIS), INVALID), (dict(v8=None), INVALID), (dict(sk=ODD), INVALID),
    (dict(sv=None), INVALID), (dict(pages=None), INVALID), (dict(q_start=MIS), INVALID),
    (dict(kv_len=None), INVALID),
])
def test_fwd_cache_refuses(kw, want):
    assert fwd_cache(**kw) == want


def test_fwd_cache_workspace():
    size = lambda **kw: sa.library().sparse_attn_fwd_cache_workspace_size(ctypes.byref(cache_desc(**kw)))
    assert size(heads=6) == 0 and size(head_dim=64) == 0
    assert sa.library().sparse_attn_fwd_cache_workspace_size(None) == 0
    assert size() >= 16 and size(tokens=0) >= 16
    assert size(tokens=1 << 25) > 0 and size(tokens=(1 << 25) + 1) == 0
    assert size(batch=1 << 19) > 0 and size(batch=(1 << 19) + 1) == 0
    # parts are bounded: one long sequence, 512 workgroups
    long = dict(batch=1, tokens=1, max_pages=1 << 20, pages_stride=1 << 20)
    assert size(**long) == 512 // 4 * 8 * (128 * 4 + 8)
    assert size(**long, kv_heads=1) == 512 * 8 * (128 * 4 + 8)


@pytest.mark.parametrize("bad", BAD_CACHE_TENSORS + [
    dict(q=torch.zeros(6, 8, 128)), dict(q=torch.zeros(6, 6, 128, dtype=torch.bfloat16)),
    dict(o=torch.zeros(5, 8, 128, dtype=torch.bfloat16)), dict(o=torch.zeros(6, 8, 128)),
    dict(lse=torch.zeros(8, 6)), dict(lse=torch.zeros(6, 8, dtype=torch.float64)),
])
def test_fwd_cache_binding_refuses(bad):
    args = cache_args()
    del args["k"], args["v"]
    args["q"] = torch.zeros(6, 8, 128, dtype=torch.bfloat16)
    args.update(bad)
    with pytest.raises(ValueError):
        sa.sparse_attn_fwd_cache(**args)
