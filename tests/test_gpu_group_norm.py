"""dol_group_norm and its gradients against the definition in 64 bits, element by element (needs an MI355X).

Bars: u = 2^-24.  A deviation x - mean errs by some u (|x| + mean |x|), that is q = rstd max |x| times the same in units of the spread; sums,
rstd and the exponentials add tens of u relative to what they are made of.  Results in bf16 are rounded once, 2^-8.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U, W8 = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def dol():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2410_03348_amd import binding
    return binding


def act_and_slope(z, act):
    if act == "silu":
        s = 1 / (1 + np.exp(-z))
        return z * s, s * (1 + z * (1 - s))
    if act == "gelu":
        from scipy.special import ndtr
        return z * ndtr(z), ndtr(z) + z * np.exp(-z * z / 2) / np.sqrt(2 * np.pi)
    if act == "relu":
        return np.maximum(z, 0), (z > 0).astype(np.float64)
    return z, np.ones_like(z)


def reference(x, gamma, beta, groups, eps, act, dy):
    x = x.cpu().double().numpy()
    b, p, c = x.shape
    ga = np.ones(c) if gamma is None else gamma.cpu().double().numpy()
    be = np.zeros(c) if beta is None else beta.cpu().double().numpy()
    dy = dy.cpu().double().numpy()

    def spread(v):          # [b, groups] to [b, 1, c]
        return np.repeat(v, c // groups, axis=1)[:, None, :]

    def mean_of(v):
        return v.reshape(b, p, groups, -1).mean(axis=(1, 3))

    mean = mean_of(x)
    dev = x - spread(mean)
    rstd = 1 / np.sqrt(mean_of(dev * dev) + eps)
    r = spread(rstd)
    xh = dev * r
    z = ga * xh + be
    y, slope = act_and_slope(z, act)
    dz = dy * slope
    dh = dz * ga
    dx = r * (dh - spread(mean_of(dh)) - xh * spread(mean_of(dh * xh)))
    top = spread(np.abs(x).reshape(b, p, groups, -1).max(axis=(1, 3)))
    q = 1 + r * top
    t = np.abs(ga * dy) * (1 + np.abs(ga)) * q * (1 + np.abs(z))
    bars = dict(mean=16 * U * mean_of(np.abs(x)), rstd=rstd * 32 * U * (1 + rstd * np.abs(x).reshape(b, p, groups, -1).max(axis=(1, 3))),
                y=32 * U * (1 + np.abs(z)) * (np.abs(ga) * q * (1 + np.abs(xh)) + np.abs(be)),
                grad_x=64 * U * r * (t * (1 + np.abs(xh)) + spread(mean_of(t)) + np.abs(xh) * spread(mean_of(t * (1 + np.abs(xh))))) * (1 + np.abs(xh)),
                grad_gamma=64 * U * ((1 + np.abs(ga)) * np.abs(dy) * q * (1 + np.abs(z)) * (1 + np.abs(xh))).sum(axis=(0, 1)),
                grad_beta=64 * U * ((1 + np.abs(ga)) * np.abs(dy) * q * (1 + np.abs(z))).sum(axis=(0, 1)))
    return dict(mean=mean, rstd=rstd, y=y, grad_x=dx, grad_gamma=(dz * xh).sum(axis=(0, 1)), grad_beta=dz.sum(axis=(0, 1)), z=z), bars


def make(b, p, c, dtype, seed=0, offset=0.5):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn(b, p, c, generator=gen, device="cuda") * (torch.rand(c, generator=gen, device="cuda") + 0.5)
         + torch.randn(c, generator=gen, device="cuda") * offset).to(dtype)
    gamma, beta = torch.rand(c, generator=gen, device="cuda") + 0.5, torch.randn(c, generator=gen, device="cuda") * 0.3
    dy = torch.randn(b, p, c, generator=gen, device="cuda").to(dtype)
    return x, gamma, beta, dy


def run_and_check(dol, x, gamma, beta, groups, dy, act="silu", eps=1e-5, y=None, dx=None):
    b, p, c = x.shape
    bf = x.dtype == torch.bfloat16
    want, bars = reference(x, gamma, beta, groups, eps, act, dy)
    if act == "relu":       # a z that rounds to the other side of 0 has the other slope: no gradient comes in there
        dy = dy.masked_fill(torch.from_numpy(np.abs(want["z"]) < 1e-2).cuda(), 0.0)
        want, bars = reference(x, gamma, beta, groups, eps, act, dy)
    y = torch.empty_like(x) if y is None else y
    dx = torch.empty_like(x) if dx is None else dx
    got = dict(y=y, mean=torch.empty(b, groups, device="cuda"), rstd=torch.empty(b, groups, device="cuda"), grad_x=dx,
               grad_gamma=torch.full((c,), 7.0, device="cuda"), grad_beta=torch.full((c,), 7.0, device="cuda"))
    for backward in (False, True):
        size = dol.group_norm_workspace(x, groups, backward)
        guard = torch.full((size + 2048,), 77, dtype=torch.uint8, device="cuda")
        ws = guard[1024:1024 + size]
        if backward:
            dol.group_norm_backward(x, gamma, beta, groups, got["mean"], got["rstd"], dy, dx, got["grad_gamma"], got["grad_beta"], act=act, workspace=ws)
        else:
            dol.group_norm(x, gamma, beta, groups, y, got["mean"], got["rstd"], eps=eps, act=act, workspace=ws)
        assert bool((guard[:1024] == 77).all()) and bool((guard[1024 + size:] == 77).all())
    for name, bar in bars.items():
        g = got[name].cpu().double().numpy()
        bar = bar + (W8 * np.abs(want[name]) if bf and name in ("y", "grad_x") else 0.0) + 1e-37
        off = np.abs(g - want[name]) - bar
        assert g.shape == want[name].shape and off.max() <= 0, "%s: %g over its bar at %s" % (name, off.max(), np.unravel_index(off.argmax(), off.shape))
    return got


SIZES = [(1, 1, 1, 1), (2, 1, 8, 2), (1, 5, 3, 3), (64, 784, 32, 8), (3, 49, 84, 14), (2, 399, 84, 14), (2, 1024, 64, 8), (5, 100, 42, 14), (1, 4096, 16, 2),
         (2, 3000, 24, 3), (1, 20000, 6, 1), (2, 9000, 33, 11), (1, 700, 768, 1), (2, 64, 2048, 32), (1, 40, 5000, 1), (1, 9, 3001, 1), (70, 16, 24, 8),
         (300, 64, 64, 8)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("b,p,c,groups", SIZES)
def test_sizes(dol, b, p, c, groups, dtype):
    x, gamma, beta, dy = make(b, p, c, getattr(torch, dtype), seed=p + c)
    run_and_check(dol, x, gamma, beta, groups, dy)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("b,p,c,groups", [(3, 200, 48, 6), (1, 30000, 16, 4)])
def test_activation_functions(dol, b, p, c, groups, act, dtype):
    x, gamma, beta, dy = make(b, p, c, getattr(torch, dtype), seed=4)
    run_and_check(dol, x, gamma * 4, beta, groups, dy, act=act)
    run_and_check(dol, x, None, None, groups, dy, act=act)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("b,p,c,groups", [(2, 150, 40, 5), (1, 30000, 20, 5)])
def test_strides_and_in_place(dol, b, p, c, groups, dtype):
    """Channel slices of wider tensors at odd offsets; y over x and grad_x over grad_y; other elements stay as they are."""
    dtype = getattr(torch, dtype)
    x, gamma, beta, dy = make(b, p, c, dtype, seed=6)
    for lead, tail in ((1, 2), (4, 4), (8, 0)):
        bufs = [torch.full((b, p + 1, lead + c + tail), 7.0, dtype=dtype, device="cuda") for _ in range(4)]
        views = [q[:, :p, lead:lead + c] for q in bufs]
        views[0].copy_(x), views[1].copy_(dy)
        got = run_and_check(dol, views[0], gamma, beta, groups, views[1], act="silu", y=views[2], dx=views[3])
        for q, v in zip(bufs, views):
            q = q.clone()
            q[:, :p, lead:lead + c] = 7.0
            assert bool((q == 7).all())
    mean, rstd = torch.empty_like(got["mean"]), torch.empty_like(got["rstd"])
    gx, keep = dy.clone(), x.clone()
    y = x.clone()
    dol.group_norm(y, gamma, beta, groups, y, mean, rstd, act="silu")
    dol.group_norm_backward(keep, gamma, beta, groups, mean, rstd, gx, gx, None, None, act="silu")
    whole = run_and_check(dol, keep, gamma, beta, groups, dy)
    assert torch.equal(y, whole["y"]) and torch.equal(gx, whole["grad_x"])


@pytest.mark.parametrize("b,p,c,groups", [(2, 500, 32, 4), (1, 40000, 8, 2)])
def test_far_from_zero(dol, b, p, c, groups):
    """Activations whose mean is thousands of times their spread, and groups that do not vary at all."""
    x, gamma, beta, dy = make(b, p, c, torch.float32, seed=7, offset=0.0)
    run_and_check(dol, x * 0.01 + 100.0, gamma, beta, groups, dy)
    run_and_check(dol, x * 1e-12, gamma, beta, groups, dy, eps=0.0)
    run_and_check(dol, x * 1e12, gamma, beta, groups, dy)
    flat = torch.full_like(x, 3.0)
    got = run_and_check(dol, flat, gamma, beta, groups, dy)
    assert bool((got["mean"] == 3.0).all())
    x[0, 0, 0] = 1e4        # one point far out
    run_and_check(dol, x, gamma, beta, groups, dy)


def test_nan_stays_in_its_group(dol):
    for b, p, c, groups in ((3, 100, 32, 4), (1, 40000, 32, 4)):
        x, gamma, beta, dy = make(b, p, c, torch.float32, seed=8)
        clean = run_and_check(dol, x, gamma, beta, groups, dy)
        x[0, 7, 9] = float("nan")           # group 1 of sample 0
        y, mean, rstd = torch.empty_like(x), torch.empty_like(clean["mean"]), torch.empty_like(clean["rstd"])
        dol.group_norm(x, gamma, beta, groups, y, mean, rstd, act="silu")
        hit = torch.zeros_like(x, dtype=torch.bool)
        hit[0, :, 8:16] = True
        assert bool(torch.isnan(y[hit]).all()) and torch.equal(y[~hit], clean["y"][~hit])


@pytest.mark.parametrize("b,p,c,groups", [(2, 30, 12, 3), (1, 20000, 2, 1)])
def test_against_differences(dol, b, p, c, groups):
    x, gamma, beta, dy = make(b, p, c, torch.float32, seed=9)

    def value(x, gamma, beta):
        y, mean, rstd = torch.empty_like(x), torch.empty(b, groups, device="cuda"), torch.empty(b, groups, device="cuda")
        dol.group_norm(x, gamma, beta, groups, y, mean, rstd, act="gelu")
        return (y.double() * dy.double()).sum(), mean, rstd

    _, mean, rstd = value(x, gamma, beta)
    gx, gg, gb = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
    dol.group_norm_backward(x, gamma, beta, groups, mean, rstd, dy, gx, gg, gb, act="gelu")
    gen = torch.Generator(device="cuda").manual_seed(10)
    h = 2.0 ** -8
    for _ in range(3):
        d = [torch.randn(q.shape, generator=gen, device="cuda") for q in (x, gamma, beta)]
        num = (value(*(q + h * e for q, e in zip((x, gamma, beta), d)))[0] - value(*(q - h * e for q, e in zip((x, gamma, beta), d)))[0]) / (2 * h)
        ana = sum((q.double() * e.double()).sum() for q, e in zip((gx, gg, gb), d))
        # h^2 / 6 of a third derivative (z moves by some 4 h, so 64 of it) of each term, adding up at random, and roundings over h
        terms = float((b * p * c) ** 0.5)
        assert abs(float(num - ana)) <= terms * (64 / 6 * h * h * 4 + 64 * U / h)


def test_same_bits_other_stream_and_graph(dol):
    for b, p, c, groups in ((4, 300, 64, 8), (1, 50000, 32, 4)):
        x, gamma, beta, dy = make(b, p, c, torch.bfloat16, seed=12)
        want = run_and_check(dol, x, gamma, beta, groups, dy)
        got = {k: torch.empty_like(v) for k, v in want.items()}

        def both(**kw):
            dol.group_norm(x, gamma, beta, groups, got["y"], got["mean"], got["rstd"], act="silu", **kw)
            dol.group_norm_backward(x, gamma, beta, groups, got["mean"], got["rstd"], dy, got["grad_x"], got["grad_gamma"], got["grad_beta"], act="silu", **kw)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        both(stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(got[k], want[k]) for k in want)
        ws = torch.empty(max(dol.group_norm_workspace(x, groups), dol.group_norm_workspace(x, groups, True)), dtype=torch.uint8, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            both(workspace=ws)
        for _ in range(3):
            for v in got.values():
                v.fill_(3.0)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(got[k], want[k]) for k in want)


def test_image_dimensions(dol):
    """[batch, height, width, channels], also as the permuted view of a channels-last image tensor."""
    x, gamma, beta, dy = make(2, 35, 16, torch.float32, seed=13)
    want = run_and_check(dol, x, gamma, beta, 4, dy)
    image = x.view(2, 5, 7, 16).permute(0, 3, 1, 2).contiguous(memory_format=torch.channels_last).permute(0, 2, 3, 1)
    y, mean, rstd = torch.empty_like(image), torch.empty(2, 4, device="cuda"), torch.empty(2, 4, device="cuda")
    dol.group_norm(image, gamma, beta, 4, y, mean, rstd, act="silu")
    assert torch.equal(y.reshape(2, 35, 16), want["y"])
    with pytest.raises(AssertionError):
        dol.group_norm(image.transpose(1, 2), gamma, beta, 4, y.transpose(1, 2), mean, rstd)


def test_empty_and_refusals(dol):
    x, gamma, beta, dy = make(2, 6, 8, torch.float32)
    y = torch.full_like(x, 5.0)
    mean, rstd = torch.full((2, 2), 5.0, device="cuda"), torch.full((2, 2), 5.0, device="cuda")
    gg, gb = torch.full((8,), 5.0, device="cuda"), torch.full((8,), 5.0, device="cuda")
    e = x[:, :0]
    dol.group_norm(e, gamma, beta, 2, e, mean, rstd)
    dol.group_norm(x[:0], gamma, beta, 2, x[:0], mean[:0], rstd[:0])
    dol.group_norm_backward(x[:0], gamma, beta, 2, mean[:0], rstd[:0], x[:0], x[:0], gg, gb)
    assert not gg.any() and not gb.any()
    for args, kw, match in (((x, gamma, beta, 3, y, None, None), {}, "8 channels in 3 groups"), ((x, gamma, beta, 0, y, None, None), {}, "in 0 groups"),
                            ((x, gamma, beta, 2, y[:, :4], None, None), {}, "ESHAPE"), ((x, gamma, beta, 2, y.bfloat16(), None, None), {}, "another type"),
                            ((x, gamma, beta, 2, y, None, None), dict(eps=-1.0), "eps")):
        with pytest.raises(dol.DolError, match=match):
            dol.group_norm(*args, **kw)
    with pytest.raises(dol.DolError, match="no gradient"):
        dol.group_norm_backward(x, gamma, beta, 2, mean, rstd, dy, None, None, None)
    with pytest.raises(dol.DolError, match="workspace"):
        dol.group_norm_backward(x, gamma, beta, 2, mean, rstd, dy, y, gg, gb, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    for bad in (x.double(), x.cpu(), x[0], x.transpose(1, 2)):
        with pytest.raises(AssertionError):
            dol.group_norm(bad, gamma, beta, 2, y, None, None)
    with pytest.raises(KeyError):
        dol.group_norm(x, gamma, beta, 2, y, None, None, act="swish")
    assert bool((y == 5).all()) and bool((mean == 5).all())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("b,p,c,groups", [(3, 150, 40, 5), (2, 30000, 20, 5), (4, 1, 8, 2)])
def test_samples_side_by_side(dol, b, p, c, groups, dtype):
    """Views of [points, batch, channels]: samples interleaved, in the inputs and in what is written."""
    dtype = getattr(torch, dtype)
    x, gamma, beta, dy = make(b, p, c, dtype, seed=14)
    want = run_and_check(dol, x, gamma, beta, groups, dy)
    views = [torch.empty(p, b, c, dtype=dtype, device="cuda").transpose(0, 1) for _ in range(4)]
    views[0].copy_(x), views[1].copy_(dy)
    got = run_and_check(dol, views[0], gamma, beta, groups, views[1], y=views[2], dx=views[3])
    assert torch.equal(got["y"], want["y"]) and torch.equal(got["grad_x"], want["grad_x"])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("b,p,c,groups", [(2, 2000, 24, 3), (3, 1024, 256, 32), (130, 520, 32, 1), (2, 2047, 16, 4)])
def test_slabs_of_many_vectors_to_a_thread(dol, b, p, c, groups, dtype):
    """Slabs that take eight vectors of x and of grad_y to a thread, and sixteen of x."""
    x, gamma, beta, dy = make(b, p, c, getattr(torch, dtype), seed=p)
    for act in ("silu", "none"):
        run_and_check(dol, x, gamma, beta, groups, dy, act=act)


def test_more_slabs_than_a_launch_has_threads_for(dol):
    """65 535 samples of one point, 4 093 groups of eight channels; some of the samples against the definition."""
    b, c, groups = 65535, 8 * 4093, 4093
    if torch.cuda.mem_get_info()[0] < 90 << 30:
        pytest.skip("90 GB of memory")
    gen = torch.Generator(device="cuda").manual_seed(15)
    x = torch.empty(b, 1, c, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    dy = x.roll(1, 0)
    gamma, beta = torch.rand(c, generator=gen, device="cuda") + 0.5, torch.randn(c, generator=gen, device="cuda") * 0.3
    y, mean, rstd, dx = torch.zeros_like(x), torch.zeros(b, groups, device="cuda"), torch.zeros(b, groups, device="cuda"), torch.zeros_like(x)
    dol.group_norm(x, gamma, beta, groups, y, mean, rstd, act="silu")
    dol.group_norm_backward(x, gamma, beta, groups, mean, rstd, dy, dx, None, None, act="silu")
    at = [0, 1, 7, 1024, 30000, 65533, 65534]
    want, bars = reference(x[at], gamma, beta, groups, 1e-5, "silu", dy[at])
    for name, got in (("y", y), ("mean", mean), ("rstd", rstd), ("grad_x", dx)):
        off = np.abs(got[at].cpu().double().numpy() - want[name]) - bars[name] - (W8 * np.abs(want[name]) if name in ("y", "grad_x") else 0.0) - 1e-37
        assert off.max() <= 0, "%s: %g over its bar" % (name, off.max())
    assert bool((rstd > 0).all()) and bool(torch.isfinite(rstd).all())
