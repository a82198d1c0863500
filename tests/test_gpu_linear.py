"""dol_linear and its gradients against the definition in 64 bits, through the binding (needs an MI355X).

Bars, u = 2^-24 a step of float, w = 2^-8 half a step of bf16 (0 in float):
  z          L = 16 u sum |x w| (its products exact or to 2^-24, sums in 32 bits some sqrt(n) u of their magnitudes), and w |z|; with z_rest 2^-23 |z|
  act(z)     16 u (1 + z^2) of it for the function itself (the exponential's argument is off by u of z or z^2), and 1.2 L, its steepest slope
  y          that, u of what is added, and w |y|
  dz         from the z that the call is given: 16 u (1 + z^2) (1 + |dz|); rounded to bf16 w of it, in two planes (up to 512 rows) w^2
  gradients  the sums of dz's bars and of 16 u of their magnitudes, and w of the result
"""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U, W8 = 2.0 ** -24, 2.0 ** -8
ACTS = ["none", "relu", "silu", "gelu"]


@pytest.fixture(scope="module")
def dol():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2410_03348_amd import binding
    return binding


def act_of(z, act):
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    cdf = torch.special.ndtr(z)
    return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)


def view(t, pad, shift, value=7.0):
    """The same values in a buffer of wider rows, from an element that only its type aligns; and the buffer."""
    rows, cols = t.shape
    buf = torch.full((rows * (cols + pad) + shift + 8,), value, dtype=t.dtype, device="cuda")
    v = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    v.copy_(t)
    return v, buf


def make(n, d, m, dtype, seed=0, bias=True, residual=True):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    return dict(x=normal(n, d).to(dtype), w=(normal(m, d) / math.sqrt(d)).to(dtype), b=normal(m) * 0.5 if bias else None,
                r=normal(n, m).to(dtype) if residual else None, g=normal(n, m).to(dtype))


def within(got, want, bar, what):
    assert got.shape == want.shape
    off = (got.double() - want).abs() - bar
    assert not bool(off.isnan().any()) and (off.numel() == 0 or float(off.max()) <= 0), "%s: %g over its bar" % (what, float(off.max()))


def guarded(n):
    buf = torch.full((n + 2048,), 77, dtype=torch.uint8, device="cuda")
    return buf, buf[1024:1024 + n]


def untouched(buf, n):
    return bool((buf[:1024] == 77).all()) and bool((buf[1024 + n:] == 77).all())


def decoded(z, rest):
    """z in 64 bits, with what rounding it to bf16 left."""
    if rest is None:
        return z.double()
    return (z.float().view(torch.int32) + rest.int()).view(torch.float32).double()


def forward(dol, c, act, keep=True, rest=True, y=None, z=None):
    x, w = c["x"], c["w"]
    n, m = x.shape[0], w.shape[0]
    y = torch.full((n, m), 5.0, dtype=x.dtype, device="cuda") if y is None else y
    z = (torch.full((n, m), 5.0, dtype=x.dtype, device="cuda") if z is None else z) if keep else None
    rest = torch.full((n, m), 5, dtype=torch.int16, device="cuda") if keep and rest and x.dtype == torch.bfloat16 else None
    size = dol.linear_workspace(x, w)
    buf, ws = guarded(size)
    dol.linear(x, w, y, bias=c["b"], act=act, residual=c["r"], z=z, z_rest=rest, workspace=ws)
    assert untouched(buf, size)
    return y, z, rest


def check_forward(c, act, y, z, rest):
    x, w = c["x"].double(), c["w"].double()
    half = W8 if c["x"].dtype == torch.bfloat16 else 0.0
    want = x @ w.t()
    L = 16 * U * (x.abs() @ w.t().abs())
    if c["b"] is not None:
        want = want + c["b"].double()
        L = L + U * want.abs()
    if z is not None:
        within(z, want, L + half * (want.abs() + L) + 1e-37, "z")
        if rest is not None:
            within(decoded(z, rest), want, L + 2.0 ** -23 * want.abs() + 1e-37, "z and its rest")
    v, _ = act_of(want, act)
    bar = 1.2 * L + 16 * U * (1 + want * want) * v.abs()
    if c["r"] is not None:
        v = v + c["r"].double()
        bar = bar + U * (v.abs() + c["r"].double().abs())
    within(y, v, bar + half * (v.abs() + bar) + 1e-37, "y")


def backward(dol, c, act, z, rest, gx=None, gw=None, which="xwb"):
    x, w = c["x"], c["w"]
    gx = (torch.full_like(x, 5.0, memory_format=torch.contiguous_format) if gx is None else gx) if "x" in which else None
    gw = (torch.full_like(w, 5.0, memory_format=torch.contiguous_format) if gw is None else gw) if "w" in which else None
    gb = torch.full((w.shape[0],), 5.0, device="cuda") if "b" in which else None
    size = dol.linear_workspace(x, w, True)
    buf, ws = guarded(size)
    dol.linear_backward(x, w, c["g"], gx, gw, grad_bias=gb, act=act, z=z, z_rest=rest, workspace=ws)
    assert untouched(buf, size)
    return gx, gw, gb


def check_backward(c, act, z, rest, got):
    x, w, g = c["x"].double(), c["w"].double(), c["g"].double()
    bf = c["x"].dtype == torch.bfloat16
    zd = torch.zeros_like(g) if act == "none" else decoded(z, rest)
    _, slope = act_of(zd, act)
    dz = g * slope
    err = torch.zeros_like(g) if act in ("none", "relu") else 16 * U * (1 + zd * zd) * g.abs() * (1 + slope.abs())
    half = W8 if bf else 0.0
    for name, t, a, e, k in (("grad_x", got[0], w, dz, err), ("grad_weight", got[1], x, dz.t(), err.t())):
        if t is None:
            continue
        size = e.abs() @ a.abs()
        rounding = (half if x.shape[0] > 512 else W8 * half) if act != "none" else 0.0
        bar = size * (16 * U + rounding) + k @ a.abs() * (1 + half)
        want = e @ a
        within(t, want, bar + half * (want.abs() + bar) + 1e-37, name)
    if got[2] is not None:
        within(got[2], dz.sum(0), dz.abs().sum(0) * 16 * U + err.sum(0) + 1e-37, "grad_bias")


def run_and_check(dol, c, act):
    y, z, rest = forward(dol, c, act, keep=act != "none")
    check_forward(c, act, y, z, rest)
    got = backward(dol, c, act, z, rest)
    check_backward(c, act, z, rest, got)
    return (y, z, rest) + got


SIZES = [(1, 1, 1), (1, 3, 5), (1, 4096, 64), (2, 64, 16), (3, 1000, 17), (16, 300, 33), (17, 64, 100), (31, 777, 10), (32, 129, 65), (33, 8, 200), (64, 1568, 128),
         (60, 70000, 3), (65, 64, 64), (65, 1, 1), (100, 100, 100), (128, 64, 320), (129, 63, 257), (300, 2000, 70), (513, 96, 129), (640, 128, 64), (1000, 65, 511)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,d,m", SIZES)
def test_sizes(dol, n, d, m, dtype):
    for act, bias, residual in (("none", True, True), ("gelu", True, False), ("silu", False, True)):
        run_and_check(dol, make(n, d, m, getattr(torch, dtype), seed=n + d + m, bias=bias, residual=residual), act)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,d,m", [(5, 200, 70), (130, 200, 70), (600, 64, 128)])
@pytest.mark.parametrize("act", ACTS)
def test_activation_functions(dol, n, d, m, act, dtype):
    run_and_check(dol, make(n, d, m, getattr(torch, dtype), seed=n), act)


# every tile, and both sides of the rules that choose them
TILES = [("bfloat16", 4096, 256, 4096, "256x256x64"), ("bfloat16", 4000, 700, 3900, "256x256x64"), ("bfloat16", 2000, 64, 2000, "128x128x64"), ("bfloat16", 700, 128, 700, "64x64x64"),
         ("float32", 2560, 64, 2048, "128x256x32"), ("float32", 1500, 100, 1500, "128x128x32"), ("float32", 300, 100, 300, "64x64x64"),
         ("bfloat16", 16, 100, 100, "few_kernel 16x16"), ("bfloat16", 256, 100, 8200, "few_kernel 16x16"), ("bfloat16", 3, 1000, 3001, "few_kernel 16x16"),
         ("bfloat16", 17, 1000, 1100, "64x64x64"), ("bfloat16", 257, 100, 100, "64x64x64"), ("float32", 1, 100, 100, "few_kernel 16x16"),
         ("float32", 50, 100, 100, "few_kernel 16x16"), ("float32", 64, 1000, 2500, "few_kernel 64x16"), ("float32", 33, 200, 8200, "few_kernel 64x32"),
         ("float32", 200, 100, 2000, "few_kernel 64x16"), ("float32", 32, 300, 8200, "few_kernel 32x64"), ("float32", 17, 2000, 4100, "few_kernel 32x16"),
         ("float32", 65, 1000, 1100, "64x64x64")]


@pytest.mark.parametrize("dtype,n,d,m,name", TILES)
def test_forward_tiles(dol, dtype, n, d, m, name):
    c = make(n, d, m, getattr(torch, dtype), seed=n)
    assert dol.linear_kernel(c["x"], c["w"]).endswith(name)
    check_forward(c, "gelu", *forward(dol, c, "gelu"))


BACK_TILES = [("bfloat16", 4096, 2048, 4096, "256x256x64"), ("bfloat16", 4000, 2048, 2048, "128x128x64"), ("bfloat16", 600, 128, 200, "64x64x64"),
              ("bfloat16", 512, 1024, 2048, "128x128x32"), ("bfloat16", 100, 100, 100, "64x64x64"),
              ("bfloat16", 1, 2100, 2100, "few_back_kernel 16"), ("bfloat16", 16, 1509, 3003, "few_back_kernel 16"), ("bfloat16", 30, 4160, 1100, "few_back_kernel 32"),
              ("bfloat16", 64, 130, 40000, "few_back_kernel 64"), ("bfloat16", 64, 30000, 150, "few_back_kernel 64"), ("bfloat16", 65, 2100, 2100, "128x128x32"),
              ("float32", 3, 2100, 2100, "few_back_kernel 16"), ("float32", 17, 1509, 3003, "few_back_kernel 32"), ("float32", 50, 70, 60100, "few_back_kernel 64"),
              ("float32", 64, 30000, 150, "few_back_kernel 64"), ("bfloat16", 3, 5, 900001, "few_back_kernel 16"), ("bfloat16", 18, 9, 500003, "few_back_kernel 32"),
              ("float32", 3, 3, 1500001, "few_back_kernel 16"), ("float32", 33, 7, 700001, "few_back_kernel 64"), ("float32", 2048, 256, 4096, "128x256x32"), ("float32", 1000, 300, 500, "128x128x32"), ("float32", 100, 100, 100, "64x64x64")]


@pytest.mark.parametrize("dtype,n,d,m,name", BACK_TILES)
@pytest.mark.parametrize("act", ["none", "silu"])
def test_backward_tiles(dol, dtype, n, d, m, name, act):
    c = make(n, d, m, getattr(torch, dtype), seed=n)
    assert dol.linear_kernel(c["x"], c["w"], True).endswith(name)
    run_and_check(dol, c, act)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n", [3, 40, 150, 600])
@pytest.mark.parametrize("pad,shift", [(1, 0), (8, 0), (3, 1), (64, 8)])
def test_strides_and_alignment(dol, n, pad, shift, dtype):
    """Rows of any stride, from any element; what lies between the rows of operands is NaN, of results stays as it is."""
    c = make(n, 128, 200, getattr(torch, dtype), seed=pad)
    plain = run_and_check(dol, c, "silu")
    for k in ("x", "w", "r", "g"):
        c[k] = view(c[k], pad, shift, float("nan"))[0]
    outs = [view(torch.zeros(*s, dtype=c["x"].dtype, device="cuda"), pad, shift) for s in ((n, 200), (n, 200), (n, 128), (200, 128))]
    y, z, rest = forward(dol, c, "silu", y=outs[0][0], z=outs[1][0])
    got = backward(dol, c, "silu", z, rest, outs[2][0], outs[3][0])
    check_forward(c, "silu", y, z, rest)
    check_backward(c, "silu", z, rest, got)
    assert rest is None or torch.equal(rest, plain[2])
    for v, b in outs:
        v.fill_(7.0)
        assert bool((b == 7).all())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,d,m", [(7, 100, 40), (200, 130, 90), (700, 64, 128)])
def test_each_gradient_by_itself_and_the_same_bits_twice(dol, n, d, m, dtype):
    c = make(n, d, m, getattr(torch, dtype), seed=4)
    y, z, rest, gx, gw, gb = run_and_check(dol, c, "gelu")
    for a, b in zip((y, z, rest), forward(dol, c, "gelu")):
        assert a is None or torch.equal(a, b)
    assert torch.equal(y, forward(dol, c, "gelu", keep=False)[0]) and torch.equal(z, forward(dol, c, "gelu", rest=False)[1])
    for k, want in (("x", gx), ("w", gw), ("b", gb)):
        got = backward(dol, c, "gelu", z, rest, which=k)
        assert torch.equal(got["xwb".index(k)], want)
    none = [backward(dol, c, "none", None, None, which=k)["xwb".index(k)] for k in "xwb"]
    for a, b in zip(none, backward(dol, c, "none", z, rest)):           # z is ignored without an activation function
        assert torch.equal(a, b)
    own = dict(c, r=c["r"].clone())
    assert torch.equal(forward(dol, own, "gelu", y=own["r"])[0], y)     # y in the residual's place


def test_what_rounding_z_leaves(dol):
    """Steps across powers of two, zero, the smallest and largest numbers, and what is not finite."""
    vals = [0.0, -0.0, 1.0, 1.99999988, 2.0, -1.00390625, 1.001953125, 255.99998, 3.4e38, -3.3961775e38, 1e-38, 1e-40, -1e-45, 1e-30, 0.333333343]
    b = torch.tensor(vals + [math.inf, -math.inf, math.nan], device="cuda")
    n = b.numel()
    x, w = torch.zeros(2, 8, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, 8, dtype=torch.bfloat16, device="cuda")
    y, z, rest = torch.empty(2, n, dtype=torch.bfloat16, device="cuda"), torch.empty(2, n, dtype=torch.bfloat16, device="cuda"), torch.empty(2, n, dtype=torch.int16, device="cuda")
    dol.linear(x, w, y, bias=b, z=z, z_rest=rest)
    got, want = decoded(z, rest)[1], b.double()
    m = len(vals)
    assert bool(((got[:m] - want[:m]).abs() <= 2.0 ** -23 * want[:m].abs()).all())
    assert float(got[m]) == math.inf and float(got[m + 1]) == -math.inf and math.isnan(float(got[m + 2]))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_against_differences(dol, dtype):
    """The gradients against central differences of what the forward call gives for float, of the definition in 64 bits for bf16."""
    c = make(20, 24, 30, getattr(torch, dtype), seed=31)
    y, z, rest, gx, gw, gb = run_and_check(dol, c, "silu")
    bf = dtype == "bfloat16"

    def value(x, w, b):
        if bf:
            v = act_of(x.double() @ w.double().t() + b.double(), "silu")[0]
        else:
            v = torch.empty_like(y)
            dol.linear(x, w, v, bias=b, act="silu")
        return float((v.double() * c["g"].double()).sum())

    gen = torch.Generator(device="cuda").manual_seed(5)
    h = 2.0 ** -7
    for _ in range(4):
        dx, dw, db = (torch.randn(q.shape, generator=gen, device="cuda") * s for q, s in ((c["x"], 1.0), (c["w"], 0.2), (c["b"], 1.0)))
        x, w, b = c["x"].float(), c["w"].float(), c["b"]
        num = (value(x + h * dx, w + h * dw, b + h * db) - value(x - h * dx, w - h * dw, b - h * db)) / (2 * h)
        ana = float((gx.double() * dx).sum() + (gw.double() * dw).sum() + (gb.double() * db).sum())
        # the third derivative of 600 terms (z moves by some 2 h a term, silu''' below 1: 8 h^2 / 6 each, adding up as random signs do), the roundings
        # of the losses over h, and in bf16 half a step of 480 + 720 gradients of some 5
        assert abs(num - ana) <= 3 * 8 / 6 * math.sqrt(600) * h * h + 600 * 8 * U / h + (3 * W8 * 5 * math.sqrt(1200) if bf else 0.0)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n", [20, 200])
def test_nan_stays_in_its_row(dol, n, dtype):
    c = make(n, 64, 96, getattr(torch, dtype), seed=8)
    y, z, rest, gx, _, _ = run_and_check(dol, c, "silu")
    c["x"][11, 3] = float("nan")
    y2, z2, rest2 = forward(dol, c, "silu")
    gx2, gw2, gb2 = backward(dol, c, "silu", z2, rest2)
    others = torch.arange(n, device="cuda") != 11
    assert bool(y2[11].isnan().all()) and torch.equal(y2[others], y[others]) and torch.equal(gx2[others], gx[others]) and bool(gx2[11].isnan().all())
    assert bool(gw2.isnan().all()) and bool(gb2.isnan().all())


@pytest.mark.parametrize("n,d,m", [(100, 100, 100), (600, 200, 130), (1, 2100, 2100), (40, 2101, 2100), (64, 64, 70)])
def test_an_infinity_stays_in_its_sums(dol, n, d, m):
    """bf16: results forward are infinite where the sums are; gradients may be NaN there, and nowhere else."""
    c = make(n, d, m, torch.bfloat16, seed=6)
    c["x"][n - 1, 5], c["w"][m - 1, 3] = math.inf, math.inf
    y, z, rest = forward(dol, c, "none")
    gx, gw, gb = backward(dol, c, "none", z, rest)
    want = c["x"].double().cpu() @ c["w"].double().cpu().T
    assert torch.equal(z.isnan().cpu(), want.isnan()) and torch.equal(z.isinf().cpu(), want.isinf())
    off = torch.zeros(n, d, dtype=torch.bool, device="cuda")
    off[:, 3] = True
    assert torch.equal(~gx.isfinite(), off) and bool(gb.isfinite().all())
    off = torch.zeros(m, d, dtype=torch.bool, device="cuda")
    off[:, 5] = True
    assert torch.equal(~gw.isfinite(), off)


def test_on_another_stream_and_in_a_graph(dol):
    """Replayed graphs beside eager work, two graphs one after the other that share a workspace, and eager gradients of the same operands alive."""
    for n in (8, 300):
        c = make(n, 64, 300, torch.bfloat16, seed=41)
        a = run_and_check(dol, c, "gelu")
        y, z, rest, gx, gw, gb = outs = [torch.empty_like(q) for q in a]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        dol.linear(c["x"], c["w"], y, bias=c["b"], act="gelu", residual=c["r"], z=z, z_rest=rest, stream=side)
        dol.linear_backward(c["x"], c["w"], c["g"], gx, gw, grad_bias=gb, act="gelu", z=z, z_rest=rest, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        for p, q in zip(a, outs):
            assert torch.equal(p, q)
        ws = torch.empty(max(dol.linear_workspace(c["x"], c["w"]), dol.linear_workspace(c["x"], c["w"], True)), dtype=torch.uint8, device="cuda")
        first, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(first):
            dol.linear(c["x"], c["w"], y, bias=c["b"], act="gelu", residual=c["r"], z=z, z_rest=rest, workspace=ws)
        with torch.cuda.graph(second):
            dol.linear_backward(c["x"], c["w"], c["g"], gx, gw, grad_bias=gb, act="gelu", z=z, z_rest=rest, workspace=ws)
        for k in range(3):
            c["x"].copy_(torch.randn_like(c["x"].float()))
            first.replay()
            second.replay()
            for p, q in zip(run_and_check(dol, c, "gelu"), outs):
                assert torch.equal(p, q)
            torch.cuda.synchronize()


def test_no_rows(dol):
    c = make(4, 16, 20, torch.float32)
    gw, gb = torch.full_like(c["w"], 3.0), torch.full_like(c["b"], 3.0)
    e = torch.empty(0, 20, device="cuda")
    dol.linear(c["x"][:0], c["w"], e, bias=c["b"], act="silu", z=e)
    dol.linear_backward(c["x"][:0], c["w"], e, c["x"][:0], gw, grad_bias=gb, act="silu", z=e)
    assert not gw.any() and not gb.any()


def test_refusals(dol):
    c = make(8, 16, 20, torch.float32)
    x, w, g = c["x"], c["w"], c["g"]
    y, z = torch.full((8, 20), 9.0, device="cuda"), torch.full((8, 20), 9.0, device="cuda")
    rests = torch.zeros(8, 20, dtype=torch.int16, device="cuda")
    for a, kw, why in (((x[:, :15], w, y), {}, "ESHAPE"), ((x.bfloat16(), w, y), {}, "types"), ((x, w[:0], y), {}, "one out"), ((x, w, y[:, :19]), {}, "y is"),
                       ((x, w, y.bfloat16()), {}, "another type"), ((x, w, y), dict(residual=g[:7]), "residual is"), ((x, w, y), dict(z=z[:, 1:]), "z is"),
                       ((x, w, y), dict(z_rest=rests), "z_rest"), ((x, w, y), dict(z=z, z_rest=rests), "z_rest")):
        with pytest.raises(dol.DolError, match=why):
            dol.linear(*a, **kw)
    big = make(300, 16, 20, torch.float32)
    with pytest.raises(dol.DolError, match="workspace has 16 bytes"):
        dol.linear(big["x"], w, big["g"], workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(dol.DolError, match="aligned"):
        dol.linear(big["x"], w, big["g"], workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda")[16:])
    gx, gw = torch.full_like(x, 9.0), torch.full_like(w, 9.0)
    for a, kw, why in (((x, w, g, None, None), {}, "no gradient"), ((x, w, g[:7], gx, gw), {}, "grad_y is"), ((x, w, g, gx[:7], gw), {}, "grad_x is"),
                       ((x, w, g, gx, gw[:, :15]), {}, "grad_weight is"), ((x, w, g, gx.bfloat16(), gw), {}, "another type"),
                       ((x, w, g, gx, gw), dict(act="silu"), "z is NULL"), ((x, w, g, gx, gw), dict(act="silu", z=z[:7]), "z is"),
                       ((x, w, g, gx, gw), dict(act="silu", z=z, z_rest=rests), "z_rest")):
        with pytest.raises(dol.DolError, match=why):
            dol.linear_backward(*a, **kw)
    for bad in (x.double(), x.cpu(), x.t(), x[0]):
        with pytest.raises(AssertionError):
            dol.linear(bad, w, y)
    with pytest.raises(AssertionError):
        dol.linear(x, w, y, bias=torch.zeros(19, device="cuda"))
    with pytest.raises(KeyError):
        dol.linear(x, w, y, act="tanh")
    torch.cuda.synchronize()
    assert all(bool((t == 9).all()) for t in (y, z, gx, gw))
