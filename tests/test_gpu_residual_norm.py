"""dol_residual_norm and its gradients against the definition in 64 bits, through the binding (needs an MI355X).

Bars, u = 2^-24 a step of float, w = 2^-8 half a step of bf16 (0 in float), sums of n terms in 32 bits off by 4 sqrt(n) u of their magnitudes at most
(a thread's terms one after the other, then a tree):
  rstd       its sum's, halved by the root, and 4 roundings                     R = (2 sqrt(cols) + 4) u of it
  h          |x| u + |scale gate v| (R + 6 u), and w |h|
  y          |y| (R + 6 u) + what h's own error is in y, and w |y|
  gradients  each element from a dozen products of numbers that are off by R or less (the formula in 64 bits is given the same rstd), means of
             rows off by 4 sqrt(cols) u of their magnitudes: 16 (R + u) of the magnitudes that are added up, and w of the result; hhat counts
             with the magnitudes of what it is made of, |x| + |scale gate v|
  sums       over rows 4 sqrt(rows) u more of the magnitudes
"""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = 2.0 ** -24
HALF = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}
EPS = 1e-6


@pytest.fixture(scope="module")
def dol():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2410_03348_amd import binding
    return binding


def view(t, pad, shift):
    """The same values in a buffer of wider rows, from an element that only its type aligns; and the buffer."""
    if t is None:
        return None, None
    rows, cols = t.shape
    buf = torch.full((rows * (cols + pad) + shift + 8,), 7.0, dtype=t.dtype, device="cuda")
    v = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    v.copy_(t)
    return v, buf


class Case:
    def __init__(self, rows, cols, dtype, gates=0, post=True, stream=True, gammas=True, scale=0.7, seed=0, pad=0, shift=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape):
            return torch.randn(shape, generator=gen, device="cuda")

        self.rows, self.cols, self.dtype, self.post, self.scale = rows, cols, dtype, post, scale
        self.pad, self.shift = pad, shift
        size = torch.rand(rows, 1, generator=gen, device="cuda") * 2 + 0.2
        self.x = self.place((normal(rows, cols) * size).to(dtype)) if stream else None
        self.u = self.place((normal(rows, cols) * size).to(dtype))
        self.gate = self.place(normal(gates, cols).to(dtype)) if gates else None
        self.gamma_u = normal(cols) if post and gammas else None
        self.gamma_y = normal(cols) if gammas else None
        self.grad_h, self.grad_y = self.place(normal(rows, cols).to(dtype)), self.place(normal(rows, cols).to(dtype))

    def place(self, t):
        return view(t, self.pad, self.shift)[0]

    def like(self, rows=None):
        return self.place(torch.full((self.rows if rows is None else rows, self.cols), 5.0, dtype=self.dtype, device="cuda"))


def wide(t, n=None):
    return None if t is None else t.double()


def spread_gate(c):
    return 1.0 if c.gate is None else c.gate.double().repeat_interleave(c.rows // c.gate.shape[0], dim=0)


def within(got, want, bar, what):
    assert got.shape == want.shape
    off = (got.double() - want).abs() - bar
    assert not bool(off.isnan().any()) and (off.numel() == 0 or float(off.max()) <= 0), "%s: %g over its bar" % (what, float(off.max()))


def forward(dol, c, h=None, y=None, **kw):
    h, y = c.like() if h is None else h, c.like() if y is None else y
    ru, rh = (torch.full((c.rows,), 5.0, device="cuda") for _ in range(2))
    dol.residual_norm(c.x, c.u, c.gamma_u, c.gate, c.gamma_y, h, y, ru if c.post else None, rh, norm_u=c.post, scale=c.scale, eps=EPS, **kw)
    return h, y, ru, rh


def check_forward(c, h, y, ru, rh):
    w, R = HALF[c.dtype], (2 * math.sqrt(c.cols) + 4) * U
    u = c.u.double()
    v = u
    if c.post:
        rstd = (u.pow(2).mean(1) + EPS).rsqrt()
        within(ru, rstd, rstd * R, "rstd_u")
        v = u * rstd[:, None] * (1.0 if c.gamma_u is None else c.gamma_u.double())
    t = c.scale * spread_gate(c) * v
    x = 0.0 * u if c.x is None else c.x.double()
    want = x + t
    err = x.abs() * U + t.abs() * (R + 6 * U)
    within(h, want, err + w * (want.abs() + err) + 1e-37, "h")
    rstd = (want.pow(2).mean(1) + EPS).rsqrt()
    # h's errors in its norm: sum h dh / sum h^2, at most their roots' ratio
    hh = err.pow(2).mean(1).sqrt() * rstd
    within(rh, rstd, rstd * (R + hh), "rstd_h")
    g = 1.0 if c.gamma_y is None else c.gamma_y.double()
    wy = want * rstd[:, None] * g
    ey = wy.abs() * (R + hh[:, None] + 6 * U) + (err * rstd[:, None] * g).abs()
    within(y, wy, ey + w * (wy.abs() + ey) + 1e-37, "y")


def backward(dol, c, ru, rh, grad_h, grad_y, grad_x=None, grad_u=None, stream=None):
    gx, gu = c.like() if grad_x is None else grad_x, c.like() if grad_u is None else grad_u
    ggu = torch.full((c.cols,), 5.0, device="cuda") if c.post else None
    ggy = torch.full((c.cols,), 5.0, device="cuda")
    gg = c.like(c.gate.shape[0]) if c.gate is not None else None
    size = dol.residual_norm_workspace(c.u, c.gate)
    guard = torch.full((size + 2048,), 77, dtype=torch.uint8, device="cuda")
    dol.residual_norm_backward(c.x, c.u, c.gamma_u, c.gate, c.gamma_y, ru if c.post else None, rh, grad_h, grad_y, gx, gu, ggu, gg, ggy, norm_u=c.post,
                               scale=c.scale, workspace=guard[1024:1024 + size], stream=stream)
    if stream is None:
        assert bool((guard[:1024] == 77).all()) and bool((guard[1024 + size:] == 77).all())
    return gx, gu, ggu, gg, ggy


def exact_backward(c, ru, rh, grad_h, grad_y):
    """The formulas of the gradients in 64 bits, from the rstd that the call is given; with each result the magnitudes that make it up."""
    u = c.u.double()
    gy = 0.0 * u if grad_y is None else grad_y.double()
    gh = 0.0 * u if grad_h is None else grad_h.double()
    one = torch.ones(c.cols, dtype=torch.float64, device="cuda")
    gamma_y, gamma_u = (one if g is None else g.double() for g in (c.gamma_y, c.gamma_u))
    uhat = u * ru.double()[:, None] if c.post else u
    a = gamma_y * gy
    rs = rh.double()[:, None]
    k = c.scale * spread_gate(c) * torch.ones_like(u)
    x = 0.0 * u if c.x is None else c.x.double()
    hh, sh = (x + k * gamma_u * uhat) * rs, (x.abs() + (k * gamma_u * uhat).abs()) * rs
    dh = gh + rs * (a - hh * (a * hh).mean(1, keepdim=True))
    sdh = gh.abs() + rs * (a.abs() + sh * (a * sh).abs().mean(1, keepdim=True))
    dv, sdv = k * dh, k.abs() * sdh
    if c.post:
        rr = ru.double()[:, None]
        du = rr * (gamma_u * dv - uhat * (gamma_u * dv * uhat).mean(1, keepdim=True))
        sdu = rr * ((gamma_u * sdv).abs() + uhat.abs() * (gamma_u * sdv * uhat).abs().mean(1, keepdim=True))
    else:
        du, sdu = dv, sdv
    out = {"x": (dh, sdh), "u": (du, sdu), "gamma_y": ((gy * hh).sum(0), (gy * sh).abs().sum(0)),
           "gamma_u": ((dv * uhat).sum(0), (sdv * uhat).abs().sum(0))}
    if c.gate is not None:
        n = c.gate.shape[0]
        dg, sdg = c.scale * dh * gamma_u * uhat, (c.scale * sdh * gamma_u * uhat).abs()
        out["gate"] = tuple(t.view(n, -1, c.cols).sum(1) for t in (dg, sdg))
    return out


def check_backward(c, ru, rh, grad_h, grad_y, got):
    want = exact_backward(c, ru, rh, grad_h, grad_y)
    w, R = HALF[c.dtype], (2 * math.sqrt(c.cols) + 4) * U
    each, rows = 16 * (R + U), 4 * math.sqrt(c.rows) * U
    for name, g, half, more in (("x", got[0], w, 0), ("u", got[1], w, 0), ("gamma_u", got[2], 0, rows), ("gate", got[3], w, rows), ("gamma_y", got[4], 0, rows)):
        if g is None:
            continue
        value, size = want[name]
        within(g, value, size * (each + more) * (1 + half) + half * value.abs() + 1e-37, "grad_" + name)


def run_and_check(dol, c):
    h, y, ru, rh = forward(dol, c)
    check_forward(c, h, y, ru, rh)
    check_backward(c, ru, rh, c.grad_h, c.grad_y, backward(dol, c, ru, rh, c.grad_h, c.grad_y))


# rows to every form: 4 threads to a row up to a whole workgroup, and the form for longer ones
COLS = [1, 3, 8, 17, 32, 33, 64, 100, 128, 255, 256, 300, 512, 777, 1024, 1111, 2048, 2500, 4096, 5000, 8192, 8200, 16384, 16389, 40000]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("cols", COLS)
def test_rows_of_any_length(dol, cols, dtype):
    for rows, gates in ((1, 0), (37, 1)):
        run_and_check(dol, Case(rows, cols, getattr(torch, dtype), gates=gates, seed=cols))


# rows, gates: one for all, one for a sample of few rows or many, one for each row, sets that do not fill a workgroup's groups
SETS = [(1, 1), (2, 2), (64, 1), (64, 2), (64, 32), (64, 64), (3136, 64), (1000, 500), (999, 3), (4096, 8), (5000, 1), (1200, 1200), (3000, 600)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("rows,gates", SETS)
@pytest.mark.parametrize("cols", [32, 72, 700])
def test_gates(dol, rows, gates, cols, post, dtype):
    run_and_check(dol, Case(rows, cols, getattr(torch, dtype), gates=gates, post=post, seed=rows + gates))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,gates,cols", [(6, 3, 20000), (70, 2, 20000), (5, 5, 20000), (3, 0, 20000)])
def test_gates_of_long_rows(dol, rows, gates, cols, dtype):
    for post in (True, False):
        run_and_check(dol, Case(rows, cols, getattr(torch, dtype), gates=gates, post=post, seed=rows))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("cols,pad,shift", [(100, 1, 0), (100, 0, 1), (257, 7, 3), (4096, 3, 1), (4096, 64, 8), (20000, 5, 1)])
def test_strides_and_alignment(dol, cols, pad, shift, dtype):
    c = Case(40, cols, getattr(torch, dtype), gates=4, seed=pad, pad=pad, shift=shift)
    run_and_check(dol, c)
    # what lies around a result stays as it is
    h, hb = view(torch.zeros(c.rows, cols, dtype=c.dtype, device="cuda"), pad, shift)
    y, yb = view(torch.zeros(c.rows, cols, dtype=c.dtype, device="cuda"), pad, shift)
    _, _, ru, rh = forward(dol, c, h, y)
    gx, gxb = view(torch.zeros(c.rows, cols, dtype=c.dtype, device="cuda"), pad, shift)
    gu, gub = view(torch.zeros(c.rows, cols, dtype=c.dtype, device="cuda"), pad, shift)
    backward(dol, c, ru, rh, c.grad_h, c.grad_y, gx, gu)
    for v, b in ((h, hb), (y, yb), (gx, gxb), (gu, gub)):
        v.fill_(7.0)
        assert bool((b == 7).all())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("cols", [48, 3000, 20000])
def test_parts_that_are_left_out(dol, cols, dtype):
    t = getattr(torch, dtype)
    for kw in (dict(stream=False), dict(gammas=False), dict(stream=False, gammas=False, post=False, scale=1.0)):
        c = Case(21, cols, t, **kw)
        run_and_check(dol, c)
        h, y, ru, rh = forward(dol, c)
        only_y, only_h = c.like(), c.like()
        dol.residual_norm(c.x, c.u, c.gamma_u, c.gate, c.gamma_y, None, only_y, norm_u=c.post, scale=c.scale, eps=EPS)
        dol.residual_norm(c.x, c.u, c.gamma_u, c.gate, None, only_h, None, norm_u=c.post, scale=c.scale, eps=EPS)
        assert torch.equal(only_y, y) and torch.equal(only_h, h)
        for gh, gy in ((c.grad_h, None), (None, c.grad_y), (None, None)):
            check_backward(c, ru, rh, gh, gy, backward(dol, c, ru, rh, gh, gy))
        gx = c.like()
        dol.residual_norm_backward(c.x, c.u, c.gamma_u, c.gate, c.gamma_y, ru if c.post else None, rh, c.grad_h, c.grad_y, gx, None, None, None, None,
                                   norm_u=c.post, scale=c.scale)
        assert torch.equal(gx, backward(dol, c, ru, rh, c.grad_h, c.grad_y)[0])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("cols", [72, 4096, 20000])
def test_in_place(dol, cols, dtype):
    c = Case(33, cols, getattr(torch, dtype), gates=11)
    h, y, ru, rh = forward(dol, c)
    for hn, yn in (("x", "u"), ("u", "x")):
        d = Case(33, cols, getattr(torch, dtype), gates=11)
        hh, yy, _, _ = forward(dol, d, getattr(d, hn), getattr(d, yn))
        assert torch.equal(hh, h) and torch.equal(yy, y)
    want = backward(dol, c, ru, rh, c.grad_h, c.grad_y)
    for xn, un in (("grad_h", "grad_y"), ("grad_y", "u"), ("u", "x"), ("x", "grad_h")):
        d = Case(33, cols, getattr(torch, dtype), gates=11)
        got = backward(dol, d, ru, rh, d.grad_h, d.grad_y, getattr(d, xn), getattr(d, un))
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("cols", [1, 2, 5, 7, 9, 13, 20, 31, 129, 250, 361, 1111, 2101, 7463, 8193])
def test_ends_of_rows(dol, cols, dtype):
    """Where a row's last vector is read shifted: with NaN beside every row, and in place, the same bits."""
    t = getattr(torch, dtype)
    c = Case(70, cols, t, gates=14)
    h, y, ru, rh = forward(dol, c)
    check_forward(c, h, y, ru, rh)
    want = backward(dol, c, ru, rh, c.grad_h, c.grad_y)
    check_backward(c, ru, rh, c.grad_h, c.grad_y, want)
    d = Case(70, cols, t, gates=14)
    for name in ("x", "u", "gate", "grad_h", "grad_y"):
        v, b = view(getattr(c, name), 9, 1)
        b.fill_(math.nan)
        setattr(d, name, v.copy_(getattr(c, name)))
    got = backward(dol, d, ru, rh, d.grad_h, d.grad_y, d.grad_h, d.grad_y)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    hh, yy, ru2, rh2 = forward(dol, d, d.x, d.u)
    assert torch.equal(hh, h) and torch.equal(yy, y) and torch.equal(ru2, ru) and torch.equal(rh2, rh)


def test_differences(dol):
    """Gradients against differences of the forward call itself, in float."""
    c = Case(12, 96, torch.float32, gates=4, seed=2)
    h, y, ru, rh = forward(dol, c)
    gx, gu, ggu, gg, ggy = backward(dol, c, ru, rh, c.grad_h, c.grad_y)

    def loss():
        h, y, _, _ = forward(dol, c)
        return float((h.double() * c.grad_h.double()).sum() + (y.double() * c.grad_y.double()).sum())

    gen = torch.Generator(device="cuda").manual_seed(5)
    for t, g in ((c.x, gx), (c.u, gu), (c.gamma_u, ggu), (c.gate, gg), (c.gamma_y, ggy)):
        d = torch.randn(t.shape, generator=gen, device="cuda")
        kept, step = t.clone(), 2.0 ** -7
        t.copy_(kept + step * d)
        up = loss()
        t.copy_(kept - step * d)
        down = loss()
        t.copy_(kept)
        want = float((g.double() * d.double()).sum())
        # h and y off by some 2^-21 of 1 to 3 in 2 304 places, weighed by 1: 2^-21 * 3 * sqrt(2304) = 7e-5, over two steps 4.4e-3; the third derivative
        # (some 30 |d|^3 / |row|^3 of the same sums) times step^2 / 6 is below 1e-3 of the sum's size
        assert abs((up - down) / (2 * step) - want) <= 4.4e-3 + 5e-3 * (abs(want) + float(g.double().norm() * d.double().norm()) / math.sqrt(g.numel()))


def test_rows_of_zeros_and_of_what_is_not_finite(dol):
    c = Case(9, 200, torch.float32, gates=9)
    for t in (c.x, c.u):
        t[2] = 0.0
    c.u[4, 7], c.x[5, 0] = math.inf, math.nan
    h, y, ru, rh = forward(dol, c)
    assert float(ru[2]) == pytest.approx(1e3, rel=1e-6) and float(h[2].abs().max()) == 0.0 and float(y[2].abs().max()) == 0.0
    got = backward(dol, c, ru, rh, c.grad_h, c.grad_y)
    # rows that are not finite leave the others as they are
    keep = [0, 1, 2, 3, 6, 7, 8]
    d = Case(9, 200, torch.float32, gates=9)
    for t in (d.x, d.u):
        t[2] = 0.0
    h2, y2, ru2, rh2 = forward(dol, d)
    want = backward(dol, d, ru2, rh2, d.grad_h, d.grad_y)
    for a, b in ((h, h2), (y, y2), (got[0], want[0]), (got[1], want[1]), (got[3], want[3])):
        assert torch.equal(a[keep], b[keep])
    assert bool(y[5].isnan().all()) and bool(got[0][5].isnan().all())


def test_no_rows(dol):
    u = torch.empty(0, 40, device="cuda")
    g = [torch.full((40,), 5.0, device="cuda") for _ in range(2)]
    dol.residual_norm(u, u, None, None, None, u, u)
    dol.residual_norm_backward(u, u, None, None, None, g[0][:0], g[0][:0], u, u, u, u, g[0], None, g[1])
    assert all(float(t.abs().max()) == 0.0 for t in g)


def test_refusals(dol):
    c = Case(8, 40, torch.float32, gates=4)
    h, y, r = c.like(), c.like(), torch.ones(8, device="cuda")
    for kw, why in ((dict(gate=torch.ones(3, 40, device="cuda")), "divide"), (dict(gate=torch.ones(4, 41, device="cuda")), "gate has"),
                    (dict(gate=c.gate.bfloat16()), "type"), (dict(h=c.like(7)), "not 8 x 40"), (dict(x=c.u.bfloat16()), "type"),
                    (dict(h=None, y=None), "neither"), (dict(norm_u=False, gamma_u=c.gamma_u), "without norm_u"), (dict(eps=-1.0), "at least 0"),
                    (dict(eps=math.nan), "at least 0")):
        a = dict(x=c.x, gamma_u=None, gate=c.gate, gamma_y=None, h=h, y=y)
        a.update(kw)
        with pytest.raises(dol.DolError, match=why):
            dol.residual_norm(a.pop("x"), c.u, a.pop("gamma_u"), a.pop("gate"), a.pop("gamma_y"), a.pop("h"), a.pop("y"), **a)
    ok = dict(rstd_u=r, rstd_h=r, grad_h=c.grad_h, grad_y=c.grad_y, grad_x=c.like(), grad_u=c.like(), grad_gamma_u=None, grad_gate=None, grad_gamma_y=None)
    for kw, why in ((dict(rstd_h=None), "rstd_h"), (dict(rstd_u=None), "rstd_u"), (dict(grad_gate=c.like(8)), "grad_gate is"),
                    (dict(grad_x=None, grad_u=None), "no gradient"), (dict(norm_u=False, grad_gamma_u=torch.ones(40, device="cuda")), "without norm_u"),
                    (dict(workspace=torch.empty(256, dtype=torch.uint8, device="cuda")), "workspace")):
        a = dict(ok)
        a.update(kw)
        with pytest.raises(dol.DolError, match=why):
            dol.residual_norm_backward(c.x, c.u, None, c.gate, None, **a)
    with pytest.raises(dol.DolError, match="without gate"):
        dol.residual_norm_backward(c.x, c.u, None, None, None, **dict(ok, grad_gate=c.like(4)))
    for kw in (dict(gamma_y=torch.ones(41, device="cuda")), dict(gamma_y=torch.ones(40, device="cuda", dtype=torch.bfloat16))):
        with pytest.raises(AssertionError):
            dol.residual_norm(c.x, c.u, None, c.gate, h=h, y=y, **kw)
    torch.cuda.synchronize()
    assert all(float(t.float().min()) == 5.0 == float(t.float().max()) for t in (h, y, ok["grad_x"], ok["grad_u"]))


@pytest.mark.parametrize("cols", [64, 1500, 20000])
def test_the_same_bits_on_any_stream_and_in_a_graph(dol, cols):
    c = Case(600, cols, torch.bfloat16, gates=6)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()

    def buffers():
        return (c.like(), c.like(), torch.zeros(600, device="cuda"), torch.zeros(600, device="cuda"), c.like(), c.like(),
                torch.zeros(cols, device="cuda"), c.like(6), torch.zeros(cols, device="cuda"),
                torch.empty(dol.residual_norm_workspace(c.u, c.gate), dtype=torch.uint8, device="cuda"))

    def both(b, stream=None):
        dol.residual_norm(c.x, c.u, c.gamma_u, c.gate, c.gamma_y, b[0], b[1], b[2], b[3], scale=c.scale, stream=stream)
        dol.residual_norm_backward(c.x, c.u, c.gamma_u, c.gate, c.gamma_y, b[2], b[3], c.grad_h, c.grad_y, b[4], b[5], b[6], b[7], b[8], scale=c.scale,
                                   workspace=b[9], stream=stream)

    eager, captured, other = buffers(), buffers(), buffers()
    both(captured)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        both(captured)
    for k in range(3):
        for t in (c.x, c.u, c.grad_h, c.grad_y):
            t.copy_(torch.randn(t.shape, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        both(other, side)
        both(eager)
        torch.cuda.synchronize()
        for a, b, d in zip(eager[:9], captured[:9], other[:9]):
            assert torch.equal(a, b) and torch.equal(a, d)
