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
