"""Outputs of the cache calls whose rows would lie on each other are refused on
the host; layouts that keep them apart pass (shown by the check that comes after,
a workspace that is too small: nothing is launched)."""
import pytest

import test_abi_operators as T

# (token, head) strides, tokens, heads
OVERLAP = [((128, 128), 6, 8), ((256, 128), 6, 8), ((896, 128), 6, 8), ((128, 640), 6, 8),
           ((1016, 128), 6, 8), ((128, 760), 6, 8), ((120, 1024), 6, 8), ((0, 128), 6, 8),
           ((1024, 0), 6, 8), ((0, 0), 6, 8), ((256, 256), 2, 2), ((1024, 64), 2, 8),
           ((120, 1024), 6, 4), ((1 << 40, 1 << 39), 3, 4), ((1 << 62, 1 << 60), 2, 8)]
APART = [((1024, 128), 6, 8), ((2048, 128), 6, 8), ((1536, 256), 6, 4), ((128, 768), 6, 8), ((136, 816), 6, 8),
         ((128, 1 << 40), 6, 8), ((1 << 40, 128), 6, 8), ((0, 128), 1, 8), ((0, 0), 1, 1),
         ((384, 256), 6, 2), ((128, 0), 6, 1), ((128, 8), 6, 1), ((8, 128), 1, 8), ((1024, 128), 0, 8),
         ((1 << 62, 1 << 58), 2, 8)]


def shape(strides, tokens, heads):
    return dict(o_stride=strides, tokens=tokens, heads=heads, kv_heads=1 if heads < 4 else heads // 4,
                batch=1, max_pages=4, pages_stride=4)


@pytest.mark.parametrize("strides,tokens,heads", OVERLAP)
def test_rows_that_overlap_are_refused(strides, tokens, heads):
    kw = shape(strides, tokens, heads)
    assert T.fwd_cache(**kw) == T.INVALID
    assert T.append(q_out=T.ctypes.c_void_p(1 << 22), **kw) == T.INVALID
    assert T.append(q_stride=strides, **kw) == T.INVALID       # in place alike


@pytest.mark.parametrize("strides,tokens,heads", APART)
def test_rows_apart_pass(strides, tokens, heads):
    assert T.fwd_cache(ws_bytes=8, **shape(strides, tokens, heads)) == T.WORKSPACE
