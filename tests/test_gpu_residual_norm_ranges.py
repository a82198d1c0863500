"""Norms between blocks of numbers far from 1, as far as their squares are a float's, with the bars of test_gpu_residual_norm.py, which are relative to the
magnitudes that are added up (needs an MI355X)."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import test_gpu_residual_norm as rn  # noqa: E402
import test_gpu_residual_norm_from_h as rh_  # noqa: E402
from test_gpu_residual_norm import Case, dol  # noqa: E402,F401

# factors of u and of x, scale, eps: with eps = 0 rstd is as large as the row is small
RANGES = [(1e16, 1.0, 0.5, 1e-6), (1e14, 1.0, 0.5, 1e-6), (1.0, 1e16, 0.5, 1e-6), (1e16, 1e16, 0.5, 1e-6), (1e16, 1e16, 1e16, 1e-6), (1e-14, 1.0, 0.5, 0.0),
          (1e-15, 1.0, 0.5, 1e-36), (1e-15, 1e-15, 1e-15, 0.0), (1.0, 1e-16, 1e-16, 0.0), (1e-16, 1e16, 1e16, 0.0)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("cols", [2, 64, 300, 4096, 20000])
@pytest.mark.parametrize("of_u,of_x,scale,eps", RANGES)
def test_far_from_one(dol, monkeypatch, of_u, of_x, scale, eps, cols, dtype):
    monkeypatch.setattr(rn, "EPS", eps)
    c = Case(21, cols, getattr(torch, dtype), gates=7, scale=scale, seed=cols)
    c.u, c.x = (c.u.float() * of_u).to(c.dtype), (c.x.float() * of_x).to(c.dtype)
    h, y, ru, rh = rn.forward(dol, c)
    rn.check_forward(c, h, y, ru, rh)
    for grad_h in (c.grad_h, None):
        rn.check_backward(c, ru, rh, grad_h, c.grad_y, rn.backward(dol, c, ru, rh, grad_h, c.grad_y))
        rh_.check(c, h, ru, rh, grad_h, c.grad_y, rh_.backward(dol, c, h, ru, rh, grad_h, c.grad_y))
