"""Gradients of the norms between blocks from h as the forward call has left it, against the definition in 64 bits at that h (needs an MI355X).

Bars as in test_gpu_residual_norm.py, where hhat counts with the magnitude of h itself.  In float the definition at x holds as well: h's own rounding is one
step in |x| + |scale gate v|, of which those bars allow sixteen.
"""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_residual_norm import HALF, U, Case, check_backward, dol, forward, spread_gate, view, within  # noqa: E402,F401


def backward(dol, c, h, ru, rh, grad_h, grad_y, grad_x=None, grad_u=None, **kw):
    gx, gu = c.like() if grad_x is None else grad_x, c.like() if grad_u is None else grad_u
    ggu = torch.full((c.cols,), 5.0, device="cuda") if c.post else None
    ggy = torch.full((c.cols,), 5.0, device="cuda")
    gg = c.like(c.gate.shape[0]) if c.gate is not None else None
    dol.residual_norm_backward(c.u, c.gamma_u, c.gate, c.gamma_y, h, ru if c.post else None, rh, grad_h, grad_y, gx, gu, ggu, gg, ggy, norm_u=c.post,
                               scale=c.scale, **kw)
    return gx, gu, ggu, gg, ggy


def check(c, h, ru, rh, grad_h, grad_y, got):
    u = c.u.double()
    zero = torch.zeros_like(u)
    gy, gh = (zero if g is None else g.double() for g in (grad_y, grad_h))
    one = torch.ones(c.cols, dtype=torch.float64, device="cuda")
    gamma_y, gamma_u = (one if g is None else g.double() for g in (c.gamma_y, c.gamma_u))
    rr, rs = ru.double()[:, None] if c.post else 1.0, rh.double()[:, None]
    uhat, a, k = u * rr, gamma_y * gy, c.scale * spread_gate(c) * torch.ones_like(u)
    hh = zero if h is None else h.double() * rs
    dh = gh + rs * (a - hh * (a * hh).mean(1, keepdim=True))
    sdh = gh.abs() + rs * (a.abs() + hh.abs() * (a * hh).abs().mean(1, keepdim=True))
    dv, sdv = k * dh, k.abs() * sdh
    du, sdu = dv, sdv
    if c.post:
        du = rr * (gamma_u * dv - uhat * (gamma_u * dv * uhat).mean(1, keepdim=True))
        sdu = rr * ((gamma_u * sdv).abs() + uhat.abs() * (gamma_u * sdv * uhat).abs().mean(1, keepdim=True))
    w, R = HALF[c.dtype], (2 * math.sqrt(c.cols) + 4) * U
    each, rows = 16 * (R + U), 4 * math.sqrt(c.rows) * U
    sets = [(got[0], dh, sdh, w, 0), (got[1], du, sdu, w, 0), (got[4], (gy * hh).sum(0), (gy * hh).abs().sum(0), 0, rows)]
    if c.post:
        sets.append((got[2], (dv * uhat).sum(0), (sdv * uhat).abs().sum(0), 0, rows))
    if c.gate is not None:
        n = c.gate.shape[0]
        sets.append((got[3],) + tuple(t.view(n, -1, c.cols).sum(1) for t in (c.scale * dh * gamma_u * uhat, (c.scale * sdh * gamma_u * uhat).abs())) + (w, rows))
    for k, (g, value, size, half, more) in enumerate(sets):
        within(g, value, size * (each + more) * (1 + half) + half * value.abs() + 1e-37, "gradient %d" % k)


def run_and_check(dol, c):
    h, _, ru, rh = forward(dol, c)
    got = backward(dol, c, h, ru, rh, c.grad_h, c.grad_y)
    check(c, h, ru, rh, c.grad_h, c.grad_y, got)
    if c.dtype == torch.float32:
        check_backward(c, ru, rh, c.grad_h, c.grad_y, got)
    return h, ru, rh, got


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("cols", [1, 3, 17, 32, 100, 300, 1111, 4096, 8192, 8200, 20000])
def test_rows_of_any_length(dol, cols, post, dtype):
    for rows, gates in ((1, 0), (37, 1), (40, 8), (24, 24)):
        run_and_check(dol, Case(rows, cols, getattr(torch, dtype), gates=gates, post=post, seed=cols + gates))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,gates,cols", [(3136, 64, 32), (1000, 500, 72), (999, 3, 700), (5000, 1, 72)])
def test_gates(dol, rows, gates, cols, dtype):
    run_and_check(dol, Case(rows, cols, getattr(torch, dtype), gates=gates, seed=rows))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("cols", [72, 257, 4096, 20000])
def test_strides_and_in_place(dol, cols, dtype):
    """Gradients in the place of h and of others, rows of any stride with NaN beside them, without one of the two gradients that come in."""
    t = getattr(torch, dtype)
    c = Case(33, cols, t, gates=11, stream=cols != 257, gammas=cols != 72)
    h, ru, rh, want = run_and_check(dol, c)
    for xn, un in (("h", "u"), ("grad_y", "h"), ("h", "grad_h")):
        d = Case(33, cols, t, gates=11, stream=cols != 257, gammas=cols != 72)
        d.h = h.clone()
        got = backward(dol, d, d.h, ru, rh, d.grad_h, d.grad_y, getattr(d, xn), getattr(d, un))
        assert all(a is None or torch.equal(a, b) for a, b in zip(got, want))
    d = Case(33, cols, t, gates=11, stream=cols != 257, gammas=cols != 72)
    for name, v in (("u", c.u), ("gate", c.gate), ("grad_h", c.grad_h), ("grad_y", c.grad_y), ("h", h)):
        s, b = view(v, 9, 1)
        b.fill_(math.nan)
        setattr(d, name, s.copy_(v))
    assert all(a is None or torch.equal(a, b) for a, b in zip(backward(dol, d, d.h, ru, rh, d.grad_h, d.grad_y), want))
    for gh, gy, hh in ((c.grad_h, None, h), (c.grad_h, None, None), (None, c.grad_y, h)):
        check(c, hh if gy is not None else None, ru, rh, gh, gy, backward(dol, c, hh, ru, rh, gh, gy))


def test_the_same_bits_on_another_stream_and_in_a_graph(dol):
    c = Case(600, 1500, torch.bfloat16, gates=6)
    h, ru, rh, _ = run_and_check(dol, c)
    ws = torch.empty(dol.residual_norm_workspace(c.u, c.gate), dtype=torch.uint8, device="cuda")
    captured = backward(dol, c, h, ru, rh, c.grad_h, c.grad_y, workspace=ws)
    gx, gu, ggu, gg, ggy = captured
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        dol.residual_norm_backward(c.u, c.gamma_u, c.gate, c.gamma_y, h, ru, rh, c.grad_h, c.grad_y, gx, gu, ggu, gg, ggy, scale=c.scale, workspace=ws)
    for k in range(3):
        for t in (c.grad_h, c.grad_y):
            t.copy_(torch.randn(t.shape, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        eager = backward(dol, c, h, ru, rh, c.grad_h, c.grad_y)
        torch.cuda.synchronize()
        other = backward(dol, c, h, ru, rh, c.grad_h, c.grad_y, stream=side)
        torch.cuda.synchronize()
        for a, b, d in zip(eager, captured, other):
            assert torch.equal(a, b) and torch.equal(a, d)


def test_refusals(dol):
    c = Case(8, 40, torch.float32, gates=4)
    r = torch.ones(8, device="cuda")
    gx, gu = c.like(), c.like()
    for h, kw, why in ((None, {}, "h is NULL"), (c.like(7), {}, "h is 7 x 40"), (c.u.bfloat16(), {}, "h is of another type"), (c.u.clone(), dict(rstd_h=None), "rstd_h"),
                       (c.u.clone(), dict(rstd_u=None), "rstd_u"), (c.u.clone(), dict(grad_x=None, grad_u=None), "no gradient")):
        a = dict(rstd_u=r, rstd_h=r, grad_h=c.grad_h, grad_y=c.grad_y, grad_x=gx, grad_u=gu, grad_gamma_u=None, grad_gate=None, grad_gamma_y=None)
        a.update(kw)
        with pytest.raises(dol.DolError, match=why):
            dol.residual_norm_backward(c.u, None, c.gate, None, h, **a)
    torch.cuda.synchronize()
    assert all(float(t.min()) == 5.0 == float(t.max()) for t in (gx, gu))
