"""Pins of the fp64 layer-norm reference: torch's own norm and its autograd in
float64, and the gradients against central differences."""
import numpy as np
import pytest
import torch

from oracle import layer_norm as R


@pytest.mark.parametrize("rows,cols,groups", [(6, 5, 1), (6, 17, 3), (1, 1, 1), (4, 128, 2)])
def test_matches_torch_in_float64(rows, cols, groups):
    g = torch.Generator().manual_seed(rows * 100 + cols)
    x = torch.randn(rows, cols, generator=g, dtype=torch.float64, requires_grad=True)
    w = torch.randn(groups, cols, generator=g, dtype=torch.float64, requires_grad=True)
    b = torch.randn(groups, cols, generator=g, dtype=torch.float64, requires_grad=True)
    dy = torch.randn(rows, cols, generator=g, dtype=torch.float64)
    n = torch.nn.functional.layer_norm(x, (cols,), eps=1e-3).view(groups, -1, cols)
    y = (n * w[:, None] + b[:, None]).view(rows, cols)
    y.backward(dy)
    ry, mean, rstd = R.layer_norm(x.detach(), w.detach(), b.detach(), 1e-3)
    assert np.allclose(ry, y.detach(), rtol=1e-12, atol=1e-12)
    dx, dw, db = R.layer_norm_bwd(dy, x.detach(), mean, rstd, w.detach(), groups)
    for got, want in ((dx, x.grad), (dw, w.grad), (db, b.grad)):
        assert np.allclose(got, want, rtol=1e-10, atol=1e-12)


def test_gradients_against_differences():
    rng = np.random.default_rng(3)
    x, dy = rng.standard_normal((4, 7)), rng.standard_normal((4, 7))
    w, b = rng.standard_normal((2, 7)), rng.standard_normal((2, 7))
    loss = lambda x, w, b: (R.layer_norm(x, w, b, 1e-3)[0] * dy).sum()
    _, mean, rstd = R.layer_norm(x, w, b, 1e-3)
    grads = R.layer_norm_bwd(dy, x, mean, rstd, w, 2)
    args, h = [x, w, b], 1e-6
    for a, grad in zip(range(3), grads):
        for i in np.ndindex(*args[a].shape):
            up, down = [v.copy() for v in args], [v.copy() for v in args]
            up[a][i] += h
            down[a][i] -= h
            # central differences: error ~ h^2 f''' + eps / h ~ 1e-9
            assert abs((loss(*up) - loss(*down)) / (2 * h) - grad[i]) < 1e-7


def test_constant_row_and_default_weights():
    y, mean, rstd = R.layer_norm(np.full((2, 8), 3.0), eps=0.25)
    assert np.array_equal(y, np.zeros((2, 8))) and np.array_equal(mean, [3.0, 3.0])
    assert np.array_equal(rstd, [2.0, 2.0])
