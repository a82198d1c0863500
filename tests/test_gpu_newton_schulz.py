"""dol_newton_schulz against its definition in 64 bits (needs an MI355X).

Bars: an error of size e in an iterate grows at most four times in each later step (the largest slope of s (a + b s^2 + c s^4) for singular
values up to 1.2 is 3.9), so errors of eps |X_t| made in each step end within eps sum_t 4^(steps - t) |X_t|, norms being Frobenius norms.
float: eps = 16 * 2^-24, and beside that no more than four times what the same steps in 32-bit numpy are off by.  bf16: eps = 8 * 2^-12
(A and B rounded to 11 bits, |b| + 2 |c| < 9), the result's rounding 2^-8 beside it.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

COEFFICIENTS = (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module")
def dol():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2410_03348_amd import binding
    return binding


def iterates(g, steps=5, k=COEFFICIENTS, eps=1e-7, dtype=np.float64):
    """X_0 .. X_steps in the wide orientation."""
    g = np.asarray(g, np.float64)
    x = g.T if g.shape[0] > g.shape[1] else g
    x = (x / (np.sqrt((x * x).sum()) + eps)).astype(dtype)
    a, b, c = (dtype(np.float32(v)) for v in k)
    out = [x]
    for _ in range(steps):
        gram = x @ x.T
        x = a * x + (b * gram + c * (gram @ gram)) @ x
        out.append(x)
    return out


def check(got, g, steps=5, k=COEFFICIENTS, eps=1e-7):
    bf = g.dtype == torch.bfloat16
    g, got = g.cpu().double().numpy(), got.cpu().double().numpy()
    xs = iterates(g, steps, k, eps)
    want = xs[-1].T if g.shape[0] > g.shape[1] else xs[-1]
    assert got.shape == want.shape and np.isfinite(got).all()
    err = np.linalg.norm(got - want)
    e = 8 * 2.0 ** -12 if bf else 16 * 2.0 ** -24
    bar = e * sum(4.0 ** (steps - t) * np.linalg.norm(x) for t, x in enumerate(xs)) + (2.0 ** -8 * np.linalg.norm(want) if bf else 0.0)
    assert err <= bar, (err, bar)
    if not bf:
        plain = iterates(g, steps, k, eps, np.float32)[-1]
        plain = np.linalg.norm((plain.T if g.shape[0] > g.shape[1] else plain) - want)
        assert err <= 4 * plain + 2.0 ** -22 * np.linalg.norm(want), (err, plain)
    return err / max(np.linalg.norm(want), 1e-300)


def normal(shape, dtype, seed=0, scale=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (9, 1), (10, 128), (16, 16), (64, 64), (65, 63), (3, 1000), (128, 128), (129, 300), (300, 129),
                                       (257, 512), (512, 1024), (1000, 777), (1100, 1030), (2000, 100)])
def test_sizes(dol, rows, cols, dtype):
    g = normal((rows, cols), getattr(torch, dtype), seed=rows + cols)
    out = torch.empty_like(g)
    size = dol.newton_schulz_workspace(g)
    guard = torch.full((size + 2048,), 77, dtype=torch.uint8, device="cuda")
    dol.newton_schulz(g, out, workspace=guard[1024:1024 + size])
    assert bool((guard[:1024] == 77).all()) and bool((guard[1024 + size:] == 77).all())
    rel = check(out, g)
    if dtype == "bfloat16":
        assert rel <= 3.6e-3        # 2.4e-3 as the operator says, half as much again for small matrices


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_spectra(dol, dtype):
    """Matrices of one direction, of few, of ones that fade, of equal ones; the result's singular values are those of the polynomial."""
    u, _ = np.linalg.qr(np.random.default_rng(0).standard_normal((200, 200)))
    v, _ = np.linalg.qr(np.random.default_rng(1).standard_normal((300, 200)))
    k = np.arange(200)
    for s in (np.where(k < 1, 1.0, 0.0), np.where(k < 4, 1.0, 1e-3), 1.0 / (1 + k), 10.0 ** (-6.0 * k / 200), np.ones(200)):
        g = torch.from_numpy(((u * s) @ v.T)).to("cuda").to(getattr(torch, dtype))
        out = torch.empty_like(g)
        dol.newton_schulz(g, out)
        check(out, g)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_scale_of_g_does_not_matter(dol, dtype):
    """Squares of elements from 1e-30 to 1e30 are summed without running over or vanishing; eps counts as it should."""
    for scale in (1e-30, 1e-18, 1e-4, 1e10, 1e30):
        g = normal((70, 90), getattr(torch, dtype), seed=5, scale=scale)
        out = torch.empty_like(g)
        dol.newton_schulz(g, out, eps=0.0)
        check(out, g, eps=0.0)
    g = normal((70, 90), getattr(torch, dtype), seed=6)
    out = torch.empty_like(g)
    dol.newton_schulz(g, out, eps=50.0)
    check(out, g, eps=50.0)
    dol.newton_schulz(torch.zeros_like(g), out)
    assert not out.any()
    g[3, 4] = float("nan")
    dol.newton_schulz(g, out)
    assert bool(torch.isnan(out).all())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_steps_and_coefficients(dol, dtype):
    g = normal((90, 120), getattr(torch, dtype), seed=7)
    out = torch.empty_like(g)
    for steps, k in ((1, COEFFICIENTS), (2, COEFFICIENTS), (12, COEFFICIENTS), (8, (15 / 8, -10 / 8, 3 / 8)), (10, (1.5, -0.5, 0.0)), (3, (1.0, 0.0, 0.0))):
        dol.newton_schulz(g, out, steps=steps, coefficients=k)
        check(out, g, steps, k)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,cols", [(33, 70), (70, 33), (512, 300)])
def test_batches_strides_and_in_place(dol, rows, cols, dtype):
    dtype = getattr(torch, dtype)
    buf = normal((3, rows + 2, cols + 5), dtype, seed=9)
    g = buf[:, 1:rows + 1, 3:cols + 3]
    keep = buf.clone()
    single = torch.empty(rows, cols, dtype=dtype, device="cuda")
    out = torch.full((3, rows, cols + 1), 7.0, dtype=dtype, device="cuda")
    dol.newton_schulz(g, out[:, :, :cols])
    assert bool((out[:, :, cols] == 7).all())
    for k in range(3):
        check(out[k, :, :cols], g[k])
        dol.newton_schulz(g[k], single)
        e = (single.double() - out[k, :, :cols].double()).norm() / single.double().norm()
        assert float(e) <= (1e-2 if dtype == torch.bfloat16 else 2e-5)         # another tile may sum in another order
    dol.newton_schulz(g, g)
    assert torch.equal(g, out[:, :, :cols])
    inside = torch.zeros_like(buf, dtype=torch.bool)
    inside[:, 1:rows + 1, 3:cols + 3] = True
    assert torch.equal(buf[~inside], keep[~inside])


def test_same_bits_other_stream_and_graph(dol):
    g = normal((300, 500), torch.bfloat16, seed=11)
    a, b = torch.empty_like(g), torch.empty_like(g)
    dol.newton_schulz(g, a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    dol.newton_schulz(g, b, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a, b)
    ws = torch.empty(dol.newton_schulz_workspace(g), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dol.newton_schulz(g, b, workspace=ws)
    for _ in range(3):
        b.fill_(3.0)
        ws.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a, b)


def test_empty_and_refusals(dol):
    g = normal((8, 12), torch.float32)
    out = torch.full_like(g, 5.0)
    for shape in ((0, 4), (4, 0), (0, 4, 4), (3, 0, 4)):
        e = torch.empty(shape, device="cuda")
        dol.newton_schulz(e, e)
    for kw, match in ((dict(steps=0), "0 steps"), (dict(steps=65), "65 steps"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"),
                      (dict(coefficients=(30.0, 5.0, 1.0)), "pass 64"), (dict(coefficients=(float("nan"), 0.0, 0.0)), "pass 64")):
        with pytest.raises(dol.DolError, match=match):
            dol.newton_schulz(g, out, **kw)
    with pytest.raises(dol.DolError, match="ESHAPE"):
        dol.newton_schulz(g, out[:4])
    with pytest.raises(dol.DolError, match="types"):
        dol.newton_schulz(g, out.bfloat16())
    with pytest.raises(dol.DolError, match="overlap"):
        dol.newton_schulz(torch.stack([g, g]), out.expand(2, 8, 12))
    with pytest.raises(dol.DolError, match="workspace"):
        dol.newton_schulz(g.repeat(20, 20), out.repeat(20, 20), workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    for bad in (g.double(), g.cpu(), g.t(), g[0]):
        with pytest.raises(AssertionError):
            dol.newton_schulz(bad, out)
    assert bool((out == 5).all())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,cols", [(33, 70), (70, 33), (300, 200)])
def test_matrices_side_by_side(dol, rows, cols, dtype):
    """Views of [rows, batch, cols]: one row of each matrix after the other."""
    dtype = getattr(torch, dtype)
    g = normal((3, rows, cols), dtype, seed=10)
    want = torch.empty_like(g)
    dol.newton_schulz(g, want)
    there, out = (torch.empty(rows, 3, cols, dtype=dtype, device="cuda").transpose(0, 1) for _ in range(2))
    there.copy_(g)
    dol.newton_schulz(there, out)
    for k in range(3):
        check(out[k], g[k])
    assert torch.equal(out, want)


def check_on_device(got, g, steps=5):
    """The bars of check, for a batch of matrices, with products in 64 bits on the device; float beside the same steps in 32 bits there."""
    bf, tall = g.dtype == torch.bfloat16, g.shape[1] > g.shape[2]

    def turned(x):
        return x.transpose(1, 2).contiguous() if tall else x

    def steps_of(x):
        x = x / (x.norm(dim=(1, 2), keepdim=True) + 1e-7)
        a, b, c = (float(np.float32(v)) for v in COEFFICIENTS)
        out = [x]
        for _ in range(steps):
            gram = torch.stack([torch.mm(q, q.t().contiguous()) for q in x])
            x = torch.stack([a * q + torch.mm(b * p + c * torch.mm(p, p), q) for p, q in zip(gram, x)])
            out.append(x)
        return out

    xs = steps_of(turned(g.double()))
    want = xs[-1]
    assert bool(torch.isfinite(got).all())
    err = (turned(got.double()) - want).norm(dim=(1, 2))
    e = 8 * 2.0 ** -12 if bf else 16 * 2.0 ** -24
    bar = e * sum(4.0 ** (steps - t) * x.norm(dim=(1, 2)) for t, x in enumerate(xs)) + (2.0 ** -8 * want.norm(dim=(1, 2)) if bf else 0.0)
    assert bool((err <= bar).all()), (err / bar).max()
    if bf:
        assert bool((err <= 3.6e-3 * want.norm(dim=(1, 2))).all()), (err / want.norm(dim=(1, 2))).max()
    else:
        plain = (steps_of(turned(g))[-1].double() - want).norm(dim=(1, 2))
        assert bool((err <= 4 * plain + 2.0 ** -22 * want.norm(dim=(1, 2))).all()), (err / plain).max()


# Every tile of both products, wide and (in its last step turned) tall, square, a matrix and several; sides that no tile divides.
FORMS = [("float32", 1, 1100, 1030, 64, 64), ("float32", 10, 500, 1000, 128, 128), ("float32", 10, 1000, 500, 128, 128), ("float32", 1, 1700, 1750, 128, 128),
         ("float32", 43, 500, 511, 256, 256), ("float32", 43, 511, 500, 256, 256), ("float32", 1, 4000, 4095, 256, 256), ("bfloat16", 14, 300, 320, 64, 64),
         ("bfloat16", 20, 500, 490, 128, 128), ("bfloat16", 20, 490, 500, 128, 128), ("bfloat16", 20, 500, 1000, 128, 256), ("bfloat16", 20, 1000, 500, 128, 256),
         ("bfloat16", 1, 2300, 2400, 64, 128), ("bfloat16", 1, 2400, 2300, 64, 128), ("bfloat16", 43, 511, 500, 256, 256), ("bfloat16", 1, 4095, 4000, 256, 256),
         ("bfloat16", 1, 4000, 4000, 256, 256)]


@pytest.mark.parametrize("dtype,batch,rows,cols,symmetric,apply", FORMS)
def test_forms(dol, dtype, batch, rows, cols, symmetric, apply):
    g = normal((batch, rows, cols), getattr(torch, dtype), seed=rows + cols)
    assert dol.newton_schulz_kernel(g) == "ns_symmetric_kernel %dx%d, ns_apply_kernel %dx%d" % (symmetric, symmetric, apply, apply)
    out = torch.full((batch, rows, cols + 3), 7.0, dtype=g.dtype, device="cuda")
    size = dol.newton_schulz_workspace(g)
    guard = torch.full((size + 2048,), 77, dtype=torch.uint8, device="cuda")
    dol.newton_schulz(g, out[:, :, :cols], workspace=guard[1024:1024 + size])
    assert bool((guard[:1024] == 77).all()) and bool((guard[1024 + size:] == 77).all()) and bool((out[:, :, cols:] == 7).all())
    check_on_device(out[:, :, :cols], g)
    dol.newton_schulz(g, g)
    assert torch.equal(g, out[:, :, :cols])
