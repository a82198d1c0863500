"""Calls of linear layers and of norms between blocks that the other tests do not make (needs an MI355X).

Bars of the linear layer's as in test_gpu_linear.py.  Against the exact z, from which z as the call is given it is off by e_z (L + 2^-8 |z|, with z_rest
L + 2^-23 |z|), each dz is off by |g| e_z more, the second derivative of an activation function being below 1 (gelu's is 0.8 at 0); relu's slope is that of a
z of the same sign, which rounding leaves.
"""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import test_gpu_linear as lin  # noqa: E402
from test_gpu_linear import U, W8, act_of, dol, make, within  # noqa: E402,F401


def check_at_exact_z(c, act, rest, got):
    x, w, g = c["x"].double(), c["w"].double(), c["g"].double()
    z = x @ w.t()
    e = 16 * U * (x.abs() @ w.t().abs())
    if c["b"] is not None:
        z = z + c["b"].double()
        e = e + U * z.abs()
    half = W8 if c["x"].dtype == torch.bfloat16 else 0.0
    e = e + (2.0 ** -23 if rest is not None else half) * z.abs()
    slope = act_of(z, act)[1]
    dz = g * slope
    off = torch.zeros_like(g) if act in ("none", "relu") else 16 * U * (1 + z * z) * g.abs() * (1 + slope.abs()) + g.abs() * e
    keep = 1 if act != "relu" else (z.abs() > e).double()           # (relu: what lies nearer to 0 than z is off may be on either side)
    off = off + (0 if act != "relu" else (1 - keep) * g.abs())
    for name, t, a, d, k in (("grad_x", got[0], w, dz, off), ("grad_weight", got[1], x, dz.t(), off.t())):
        size = d.abs() @ a.abs()
        rounding = (half if x.shape[0] > 512 else W8 * half) if act != "none" else 0.0
        bar, want = size * (16 * U + rounding) + k @ a.abs() * (1 + half), d @ a
        within(t, want, bar + half * (want.abs() + bar) + 1e-37, name)
    within(got[2], dz.sum(0), dz.abs().sum(0) * 16 * U + off.sum(0) + 1e-37, "grad_bias")


@pytest.mark.parametrize("n,d,m", [(1, 300, 70), (5, 200, 70), (40, 2101, 2100), (64, 300, 33), (130, 200, 70), (600, 64, 128), (1000, 513, 300)])
@pytest.mark.parametrize("act", ["relu", "silu", "gelu"])
def test_bf16_gradients_with_and_without_what_rounding_z_left(dol, n, d, m, act):
    """Without z_rest the gradients are those at z as it was rounded; either way at the exact z within what z is off there."""
    c = make(n, d, m, torch.bfloat16, seed=n + m)
    for kept in (False, True):
        y, z, rest = lin.forward(dol, c, act, rest=kept)
        assert (rest is not None) == kept
        got = lin.backward(dol, c, act, z, rest)
        lin.check_backward(c, act, z, rest, got)
        check_at_exact_z(c, act, rest, got)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("gates", [1, 3])
def test_no_rows_leave_a_gate_without_gradient(dol, gates, dtype):
    """Sums over no rows are zeros, a gate's as well as gammas', in rows of any distance."""
    t = getattr(torch, dtype)
    u, gate = torch.empty(0, 40, dtype=t, device="cuda"), torch.ones(gates, 40, dtype=t, device="cuda")
    buf = torch.full((gates, 47), 5.0, dtype=t, device="cuda")
    gg, sums = buf[:, 3:43], [torch.full((40,), 5.0, device="cuda") for _ in range(2)]
    none = sums[0][:0]
    dol.residual_norm(u, u, None, gate, None, u, u)
    for first in ((u, u, None, gate, None), (u, None, gate, None, u)):
        gg.fill_(5.0)
        dol.residual_norm_backward(*first, none, none, u, u, u, u, sums[0], gg, sums[1])
        assert not gg.any() and not sums[0].any() and not sums[1].any()
    assert bool((buf[:, :3] == 5).all()) and bool((buf[:, 43:] == 5).all())
    gg.fill_(5.0)
    dol.residual_norm_backward(u, u, None, gate, None, none, none, u, u, u, u, None, gg, None)
    assert not gg.any()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows", [5, 300])
def test_operands_and_results_as_columns_of_one_buffer(dol, rows, dtype):
    """The same bits as in buffers of their own, and every other column as it was; a result that shares a column is refused, in place it is taken."""
    t = getattr(torch, dtype)
    c = make(rows, 40, 40, t, seed=rows)
    y, z, rest = lin.forward(dol, c, "silu")
    gx, gw, gb = lin.backward(dol, c, "silu", z, rest)
    buf = torch.full((rows, 300), 7.0, dtype=t, device="cuda")
    x, r, g, y2, z2, gx2 = (buf[:, 41 * k:41 * k + 40] for k in range(6))
    for to, v in ((x, c["x"]), (r, c["r"]), (g, c["g"])):
        to.copy_(v)
    dol.linear(x, c["w"], y2, bias=c["b"], act="silu", residual=r, z=z2, z_rest=None if rest is None else rest.clone())
    gw2, gb2 = torch.empty_like(gw), torch.empty_like(gb)
    dol.linear_backward(x, c["w"], g, gx2, gw2, grad_bias=gb2, act="silu", z=z2, z_rest=rest)
    for a, b in ((y, y2), (z, z2), (gx, gx2), (gw, gw2), (gb, gb2)):
        assert torch.equal(a, b)
    with pytest.raises(dol.DolError, match="y is x"):
        dol.linear(x, c["w"], buf[:, 1:41], act="silu", residual=r)
    dol.linear(x, c["w"], r, bias=c["b"], act="silu", residual=r)
    assert torch.equal(r, y)
    r.copy_(c["r"])
    # x, u, grad_h, grad_y and h, y, grad_x, grad_u
    h, v, ru, rh = torch.empty_like(y), torch.empty_like(y), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    dol.residual_norm(c["r"], c["g"], None, None, None, h, v, ru, rh)
    dol.residual_norm(r, g, None, None, None, y2, z2, ru, rh)
    assert torch.equal(h, y2) and torch.equal(v, z2)
    a, b = torch.empty_like(y), torch.empty_like(y)
    dol.residual_norm_backward(c["r"], c["g"], None, None, None, ru, rh, h, v, a, b, None, None, None)
    dol.residual_norm_backward(r, g, None, None, None, ru, rh, y2, z2, gx2, x, None, None, None)
    assert torch.equal(a, gx2) and torch.equal(b, x)
    with pytest.raises(dol.DolError, match="own"):
        dol.residual_norm_backward(r, g, None, None, None, ru, rh, y2, z2, buf[:, 42:82], x, None, None, None)
    dol.residual_norm_backward(r, g, None, None, None, ru, rh, y2, z2, z2, r, None, None, None)
    assert torch.equal(a, z2) and torch.equal(b, r)
    for to in (x, r, g, y2, z2, gx2):
        to.fill_(7.0)
    assert bool((buf == 7).all())


# one for each form of the forward call in float: few rows, and tiles in one share of k or several
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,d,m", [(1, 300, 70), (64, 300, 33), (65, 300, 1100), (300, 100, 300), (300, 777, 150), (1500, 100, 1500), (257, 65, 3)])
def test_infinities_forward_do_not_go_by_the_number_of_rows(dol, n, d, m, dtype):
    """z is infinite, NaN and finite where the sums in 64 bits are, whatever computes it: infinities of either sign beside numbers of many bits, large ones
    among them, a zero, each other and a NaN."""
    t = getattr(torch, dtype)
    c = make(n, d, m, t, seed=n)
    x, w = c["x"], c["w"]
    w[0] *= 1e4
    x[0, 5], x[n - 1, 7], x[n // 2, d - 1] = float("inf"), float("-inf"), float("inf")
    w[m - 1, 3], w[1, 5], w[2, 5], w[2, 9] = float("-inf"), 0.0, float("-inf"), float("inf")
    x[n // 3, 20] = float("nan")
    y, z, _ = lin.forward(dol, dict(c, r=None), "none")
    want = x.double().cpu() @ w.double().cpu().t() + c["b"].double().cpu()
    got = z.double().cpu()
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.isinf(), want.isinf())
    assert torch.equal(got[want.isinf()], want[want.isinf()]) and torch.equal(y.isnan(), z.isnan())
    finite = want.isfinite()
    xs, ws = (v.double().cpu().nan_to_num(0.0, 0.0, 0.0) for v in (x, w))
    L = 16 * U * (xs.abs() @ ws.abs().t()) + U * want.abs()
    half = W8 if dtype == "bfloat16" else 0.0
    assert bool(((got - want).abs() <= L + half * (want.abs() + L) + 1e-37)[finite].all())


@pytest.mark.parametrize("n,d,m", [(100, 100, 100), (600, 200, 130), (1, 2100, 2100), (40, 2101, 2100), (64, 64, 70)])
def test_infinities_in_float_stay_in_their_gradients(dol, n, d, m):
    c = make(n, d, m, torch.float32, seed=6)
    c["x"][n - 1, 5], c["w"][m - 1, 3] = float("inf"), float("-inf")
    gx, gw, gb = lin.backward(dol, c, "none", None, None)
    off = torch.zeros(n, d, dtype=torch.bool, device="cuda")
    off[:, 3] = True
    assert torch.equal(~gx.isfinite(), off) and bool(gb.isfinite().all())
    off = torch.zeros(m, d, dtype=torch.bool, device="cuda")
    off[:, 5] = True
    assert torch.equal(~gw.isfinite(), off)
