"""fp64 reference of the layer norm over rows and of its gradients.

Test infrastructure only: plain NumPy, written from the definition
y = (x - mean) rstd w + b, rstd = (var + eps)^(-1/2); the library's code never
imports it.  Rows form equal groups of consecutive rows, each with its own
weight and bias row.
"""
import numpy as np


def _per_row(w, rows, cols, none):
    """[cols] or [groups, cols] weights (None: `none`) as [rows, cols]."""
    if w is None:
        return np.full((rows, cols), none, dtype=np.float64)
    w = np.asarray(w, dtype=np.float64).reshape(-1, cols)
    return np.repeat(w, rows // w.shape[0], axis=0)


def layer_norm(x, weight=None, bias=None, eps=1e-6):
    """(y, mean, rstd) of x [rows, cols]."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    mean = x.sum(1) / cols
    d = x - mean[:, None]
    rstd = 1.0 / np.sqrt((d * d).sum(1) / cols + eps)
    y = d * rstd[:, None] * _per_row(weight, rows, cols, 1.0) + _per_row(bias, rows, cols, 0.0)
    return y, mean, rstd


def layer_norm_bwd(dy, x, mean, rstd, weight=None, groups=1):
    """(dx, dweight [groups, cols], dbias [groups, cols]) for upstream dy, the
    statistics being those of x."""
    dy, x = np.asarray(dy, dtype=np.float64), np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    xh = (x - np.asarray(mean, dtype=np.float64)[:, None]) * np.asarray(rstd, np.float64)[:, None]
    g = dy * _per_row(weight, rows, cols, 1.0)
    dx = (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    dx = dx * np.asarray(rstd, np.float64)[:, None]
    split = lambda t: t.reshape(groups, rows // groups, cols).sum(1)
    return dx, split(dy * xh), split(dy)
