"""dol_cross_entropy and its gradients against the definition in 64 bits, through the binding (needs an MI355X).

Bars, from the rounding the operator states: u = 2^-24 (float) for sums and exponentials, w = 2^-8 for a number rounded to bf16.
  a logit        |dl| <= L = 16 u sum_k |x_ik w_vk|  (its products exact or to 2^-24; a sum of n terms in 32 bits errs by some sqrt(n) u of
                 their magnitudes, blocks of 16 and 32 at a time: 16 covers rows of 1 024)
  lse, loss      L + 8 u (1 + |lse|), the exponentials' own roundings and that of the result
  a gradient     its terms' magnitudes S times (2 max L + 32 u), and w (S + |result|) where dl and the result are bf16
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


def padded(t, pad, value=7.0):
    """The same values as a view into a wider tensor whose other columns hold `value`."""
    buf = torch.full((t.shape[0], t.shape[1] + pad), value, dtype=t.dtype, device="cuda")
    buf[:, :t.shape[1]] = t
    return buf, buf[:, :t.shape[1]]


def make(n, d, v, dtype, seed=0, bias=True, scale=2.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, d, generator=gen, device="cuda").to(dtype)
    w = (torch.randn(v, d, generator=gen, device="cuda") * scale / d ** 0.5).to(dtype)
    b = torch.randn(v, generator=gen, device="cuda") * 0.5 if bias else None
    t = torch.randint(0, v, (n,), generator=gen, device="cuda", dtype=torch.int32)
    g = torch.rand(n, generator=gen, device="cuda") * 2 - 0.5
    return x, w, b, t, g


def reference(x, w, b, t, g):
    """Everything in 64 bits on the host; also the magnitudes that the bars are made of."""
    x, w = x.detach().cpu().double().numpy(), w.detach().cpu().double().numpy()
    t, g = t.cpu().numpy(), g.cpu().double().numpy()
    v = w.shape[0]
    kept = (t >= 0) & (t < v)
    with np.errstate(all="ignore"):
        logits = x @ w.T + (0.0 if b is None else b.cpu().double().numpy())
        top = logits.max(axis=1)
        base = np.where(np.isfinite(top), top, 0.0)
        lse = base + np.log(np.exp(logits - base[:, None]).sum(axis=1))
        loss = np.where(kept, np.where(lse == -np.inf, np.inf, lse - logits[np.arange(len(t)), np.where(kept, t, 0)]), 0.0)
        counts = kept & (lse != -np.inf)
        dl = np.where(counts[:, None], np.exp(logits - lse[:, None]), 0.0)
    dl[np.flatnonzero(counts), t[counts]] -= 1.0
    dl = np.where(counts[:, None], dl * g[:, None], 0.0)
    xk = np.where(kept[:, None], x, 0.0)
    err_l = 16 * U * (np.abs(xk) @ np.abs(w).T)
    return dict(lse=lse, loss=loss, grad_x=dl @ w, grad_w=dl.T @ xk, grad_b=dl.sum(axis=0), kept=kept,
                size_x=np.abs(dl) @ np.abs(w), size_w=np.abs(dl).T @ np.abs(xk), size_b=np.abs(dl).sum(axis=0), err_l=err_l)


def within(got, want, bar, what):
    got = got.detach().cpu().double().numpy()
    assert got.shape == want.shape
    fine = np.isfinite(want)
    np.testing.assert_array_equal(got[~fine], want[~fine], err_msg=what)
    off = np.abs(got - want)[fine] - np.broadcast_to(bar, want.shape)[fine]
    assert off.size == 0 or off.max() <= 0, "%s: %g over its bar" % (what, off.max())


def run_and_check(dol, x, w, b, t, g, pad=0):
    n, d = x.shape
    v = w.shape[0]
    ref = reference(x, w, b, t, g)
    loss, lse = torch.full((n,), 9.0, device="cuda"), torch.full((n,), 9.0, device="cuda")
    gx_buf, gx = padded(torch.full_like(x, 5.0), pad)
    gw_buf, gw = padded(torch.full_like(w, 5.0), pad)
    gb = torch.full((v,), 5.0, device="cuda") if b is not None else None
    # workspaces of exactly the size asked for, between guards that nothing may touch
    for backward in (False, True):
        size = dol.cross_entropy_workspace(x, w, backward)
        guard = torch.full((size + 2048,), 77, dtype=torch.uint8, device="cuda")
        ws = guard[1024:1024 + size]
        if backward:
            dol.cross_entropy_backward(x, w, t, lse, g, gx, gw, bias=b, grad_bias=gb, workspace=ws)
        else:
            dol.cross_entropy(x, w, t, loss, lse, bias=b, workspace=ws)
        assert bool((guard[:1024] == 77).all()) and bool((guard[1024 + size:] == 77).all())
    top_l = ref["err_l"].max(axis=1, initial=0.0)
    kept = ref["kept"]
    bar = top_l + 8 * U * (1 + np.abs(np.where(np.isfinite(ref["lse"]), ref["lse"], 0.0)))
    within(lse[torch.from_numpy(kept).cuda()], ref["lse"][kept], bar[kept], "lse")
    within(loss, ref["loss"], 2 * bar, "loss")
    rel = 2 * ref["err_l"].max(initial=0.0) + 32 * U
    bf = x.dtype == torch.bfloat16
    within(gx, ref["grad_x"], ref["size_x"] * (rel + W8 * bf) + W8 * bf * np.abs(ref["grad_x"]) + 1e-37, "grad_x")
    within(gw, ref["grad_w"], ref["size_w"] * (rel + W8 * bf) + W8 * bf * np.abs(ref["grad_w"]) + 1e-37, "grad_weight")
    if gb is not None:
        within(gb, ref["grad_b"], ref["size_b"] * rel + 1e-37, "grad_bias")
    if pad:
        assert bool((gx_buf[:, d:] == 7).all()) and bool((gw_buf[:, d:] == 7).all())
    return loss, lse, gx, gw, gb


SIZES = [(1, 1, 1), (1, 16, 2), (64, 128, 10), (5, 7, 3), (129, 65, 257), (300, 64, 300), (257, 200, 1025), (40, 1024, 700), (700, 96, 129),
         (2, 33, 9000), (1500, 24, 40)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,d,v", SIZES)
def test_sizes(dol, n, d, v, dtype):
    x, w, b, t, g = make(n, d, v, getattr(torch, dtype), seed=n + d + v)
    run_and_check(dol, x, w, b, t, g)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("pad,shift", [(1, 0), (8, 0), (3, 1), (64, 8)])
def test_strides_and_alignment(dol, dtype, pad, shift):
    """Rows of any stride, from any element; the gradients' rows too, whose other columns stay as they are."""
    x, w, b, t, g = make(150, 128 + shift, 200, getattr(torch, dtype), seed=pad)
    x, w = padded(x, pad, float("nan"))[1][:, shift:], padded(w, pad, float("nan"))[1][:, shift:]
    run_and_check(dol, x, w, b, t, g, pad)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rows_left_out(dol, dtype):
    """Targets outside the classes: no loss, no gradient, and what such a row or its grad_loss holds reaches nobody."""
    x, w, b, t, g = make(200, 64, 90, getattr(torch, dtype), seed=3)
    t[::3] = -1
    t[1::7] = 90
    t[2::11] = 2 ** 31 - 1
    out = (t < 0) | (t >= 90)
    x[out] = float("nan")
    x[5 * 3] = float("inf")
    g[out] = float("nan")
    loss, lse, gx, gw, gb = run_and_check(dol, x, w, b, t, g)
    assert bool((loss[out] == 0).all()) and bool((gx[out] == 0).all())
    # and all of them
    t[:] = -5
    loss, lse, gx, gw, gb = run_and_check(dol, x, w, b, t, g)
    assert not loss.any() and not gx.any() and not gw.any() and not gb.any()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("v", [10, 300, 1000])
def test_classes_taken_out(dol, dtype, v):
    """A bias of -inf takes a class out: whole tiles of them, the target's own (loss +inf, gradient -g at the target), all of them."""
    x, w, b, t, g = make(70, 32, v, getattr(torch, dtype), seed=v)
    b[: v * 3 // 4] = float("-inf")
    b[v - 1] = float("-inf")
    loss, *_ = run_and_check(dol, x, w, b, t, g)
    assert bool(torch.isinf(loss).any())
    b[:] = float("-inf")
    loss, lse, gx, gw, gb = run_and_check(dol, x, w, b, t, g)
    assert bool((loss == float("inf")).all()) and bool((lse == float("-inf")).all()) and not gx.any() and not gw.any() and not gb.any()
    b[:] = torch.finfo(torch.float32).min           # the type's lowest value is a number
    b[v // 2] = 0.0
    run_and_check(dol, x, w, b, torch.full_like(t, v // 2), g)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_nan_stays_in_its_row(dol, dtype):
    x, w, b, t, g = make(150, 64, 400, getattr(torch, dtype), seed=8)
    clean = run_and_check(dol, x, w, b, t, g)[0].clone()
    x[77, 3] = float("nan")
    n = x.shape[0]
    loss, lse, gx, gw = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty_like(x), torch.empty_like(w)
    dol.cross_entropy(x, w, t, loss, lse, bias=b)
    dol.cross_entropy_backward(x, w, t, lse, g, gx, gw, bias=b)
    others = torch.arange(n, device="cuda") != 77
    assert bool(torch.isnan(loss[77])) and bool(torch.isnan(gx[77]).all()) and bool(torch.isfinite(gx[others]).all())
    assert torch.equal(loss[others], clean[others])


def test_large_logits_and_small_ones(dol):
    """Logits of thousands, where every other class underflows, and a table of tiny numbers, where every class is as likely."""
    x, w, b, t, g = make(100, 64, 500, torch.float32, seed=11, scale=800.0)
    run_and_check(dol, x, w, b, t, g)
    x, w, b, t, g = make(100, 64, 500, torch.float32, seed=12)
    run_and_check(dol, x, w * 1e-30, None, t, g)


def test_pieces_and_splits(dol):
    """More classes than one piece of dl holds, and rows enough to split the k of both products."""
    for dtype, n, d, v in ((torch.bfloat16, 8300, 64, 17000), (torch.float32, 5000, 40, 9000)):
        x, w, b, t, g = make(n, d, v, dtype, seed=2)
        t[::9] = -1
        run_and_check(dol, x, w, b, t, g)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_same_bits_twice_and_any_subset(dol, dtype):
    x, w, b, t, g = make(513, 72, 1500, getattr(torch, dtype), seed=21)
    a = run_and_check(dol, x, w, b, t, g)
    loss, lse, gx, gw, gb = (torch.empty_like(q) for q in a)
    dol.cross_entropy(x, w, t, loss, lse, bias=b)
    dol.cross_entropy_backward(x, w, t, lse, g, gx, None, bias=b)
    dol.cross_entropy_backward(x, w, t, lse, g, None, gw, bias=b)
    dol.cross_entropy_backward(x, w, t, lse, g, None, None, bias=b, grad_bias=gb)
    for p, q in zip(a, (loss, lse, gx, gw, gb)):
        assert torch.equal(p, q)


def test_against_differences(dol):
    """grad_x and grad_weight against central differences of the loss that the forward call gives."""
    x, w, b, t, g = make(6, 20, 30, torch.float32, seed=31)
    t[2] = -1

    def value(x, w, b):
        loss, lse = torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
        dol.cross_entropy(x, w, t, loss, lse, bias=b)
        return (loss.double() * g.double()).sum(), lse

    _, lse = value(x, w, b)
    gx, gw, gb = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    dol.cross_entropy_backward(x, w, t, lse, g, gx, gw, bias=b, grad_bias=gb)
    gen = torch.Generator(device="cuda").manual_seed(5)
    h = 2.0 ** -7
    for _ in range(4):
        dx, dw, db = (torch.randn(q.shape, generator=gen, device="cuda") for q in (x, w, b))
        num = (value(x + h * dx, w + h * dw, b + h * db)[0] - value(x - h * dx, w - h * dw, b - h * db)[0]) / (2 * h)
        ana = (gx.double() * dx).sum() + (gw.double() * dw).sum() + (gb.double() * db).sum()
        # differences err by h^2 of a third derivative (logits move by some 5 h: 125 h^2 / 6 of a loss of order 1 in each row) and by
        # the losses' roundings over h
        assert abs(float(num - ana)) <= 6 * 125 / 6 * h * h + 6 * 32 * U * 8 / h


def test_on_another_stream_and_in_a_graph(dol):
    x, w, b, t, g = make(300, 64, 700, torch.bfloat16, seed=41)
    a = run_and_check(dol, x, w, b, t, g)
    outs = [torch.empty_like(q) for q in a]
    loss, lse, gx, gw, gb = outs
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    dol.cross_entropy(x, w, t, loss, lse, bias=b, stream=side)
    dol.cross_entropy_backward(x, w, t, lse, g, gx, gw, bias=b, grad_bias=gb, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for p, q in zip(a, outs):
        assert torch.equal(p, q)
    wf = torch.empty(max(dol.cross_entropy_workspace(x, w), dol.cross_entropy_workspace(x, w, True)), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dol.cross_entropy(x, w, t, loss, lse, bias=b, workspace=wf)
        dol.cross_entropy_backward(x, w, t, lse, g, gx, gw, bias=b, grad_bias=gb, workspace=wf)
    for _ in range(3):
        for q in outs:
            q.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        for p, q in zip(a, outs):
            assert torch.equal(p, q)


def test_no_rows(dol):
    x, w, b, t, g = make(4, 16, 20, torch.float32)
    gw, gb, e = torch.full_like(w, 3.0), torch.full_like(b, 3.0), torch.empty(0, device="cuda")
    dol.cross_entropy(x[:0], w, t[:0], e, e, bias=b)
    dol.cross_entropy_backward(x[:0], w, t[:0], e, e, x[:0], gw, bias=b, grad_bias=gb)
    assert not gw.any() and not gb.any()


def test_refusals(dol):
    x, w, b, t, g = make(8, 16, 20, torch.float32)
    loss, lse = torch.full((8,), 9.0, device="cuda"), torch.full((8,), 9.0, device="cuda")
    with pytest.raises(dol.DolError, match="ESHAPE"):
        dol.cross_entropy(x[:, :15], w, t, loss, lse)
    with pytest.raises(dol.DolError, match="types"):
        dol.cross_entropy(x.bfloat16(), w, t, loss, lse)
    with pytest.raises(dol.DolError, match="classes"):
        dol.cross_entropy(x, w[:0], t, loss, lse)
    with pytest.raises(dol.DolError, match="workspace has 16 bytes"):
        dol.cross_entropy(x, w, t, loss, lse, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(dol.DolError, match="aligned"):
        dol.cross_entropy(x, w, t, loss, lse, workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda")[16:])
    with pytest.raises(dol.DolError, match="no gradient"):
        dol.cross_entropy_backward(x, w, t, lse, g, None, None)
    with pytest.raises(dol.DolError, match="ESHAPE"):
        dol.cross_entropy_backward(x, w, t, lse, g, x[:4], None)
    with pytest.raises(dol.DolError, match="another type"):
        dol.cross_entropy_backward(x, w, t, lse, g, x.bfloat16(), None)
    for bad in (x.double(), x.cpu(), x.t(), x[0]):
        with pytest.raises(AssertionError):
            dol.cross_entropy(bad, w, t, loss, lse)
    with pytest.raises(AssertionError):
        dol.cross_entropy(x, w, t.long(), loss, lse)
    assert bool((loss == 9).all()) and bool((lse == 9).all())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,d,v", [(1, 1, 1), (17, 255, 32), (17, 256, 33), (40, 1023, 32), (40, 1025, 32), (513, 2049, 4), (300, 16, 32), (9000, 130, 10)])
def test_few_classes(dol, n, d, v, dtype):
    """Both sides of where a head is small enough for a form of its own, and its odd sizes."""
    x, w, b, t, g = make(n, d, v, getattr(torch, dtype), seed=v)
    t[::7] = v
    run_and_check(dol, x, w, b, t, g)
    run_and_check(dol, x[:, :d], w, None, t, g, pad=3)


@pytest.mark.parametrize("dtype,v", [("float32", 10), ("bfloat16", 10), ("bfloat16", 300)])
def test_rows_without_a_class(dol, dtype, v):
    """A row whose logits are all -inf: lse -inf, loss +inf, and no part in any gradient, whatever it holds."""
    x, w, b, t, g = make(40, 64, v, getattr(torch, dtype), seed=3)
    w = w.abs() + 0.125
    out = []
    for fill in (0.0, float("-inf")):
        x[3] = fill
        t[3] = v if fill == 0.0 else 1
        loss, lse = torch.empty(40, device="cuda"), torch.empty(40, device="cuda")
        gx, gw, gb = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
        dol.cross_entropy(x, w, t, loss, lse, bias=b)
        dol.cross_entropy_backward(x, w, t, lse, g, gx, gw, bias=b, grad_bias=gb)
        out.append((gx, gw, gb))
    assert float(lse[3]) == float("-inf") and float(loss[3]) == float("inf") and not gx[3].any()
    assert all(torch.equal(p, q) for p, q in zip(*out))


def test_nearly_certain_rows_of_few_classes(dol):
    """p of the target within 2^-24 of one: loss and gradient are what the other classes leave, not zero."""
    x, w = torch.zeros(20, 8, device="cuda"), torch.zeros(10, 8, device="cuda")
    b = torch.zeros(10, device="cuda")
    b[4] = 20.0
    t = torch.full((20,), 4, dtype=torch.int32, device="cuda")
    loss, lse = torch.empty(20, device="cuda"), torch.empty(20, device="cuda")
    dol.cross_entropy(x, w, t, loss, lse, bias=b)
    want = float(np.log1p(9 * np.exp(-20.0)))
    assert abs(float(loss[0]) - want) <= 16 * U * want + 8 * U * want * 20


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("v", [1, 10, 16, 17, 32, 33])
def test_nan_reaches_its_row_and_the_sums(dol, dtype, v):
    """A NaN in x, in a bias or in a whole row of logits is no missing class: the row's loss, lse and grad_x are NaN, and so is what sums over
    it; other rows have what they had.  Left out, the row has no part in anything."""
    n = 40
    x, w, b, t, g = make(n, 64, v, getattr(torch, dtype), seed=v)
    clean = run_and_check(dol, x, w, b, t, g)
    x[7, 3] = float("nan")
    others = torch.arange(n, device="cuda") != 7
    got = [torch.empty_like(q) for q in clean]
    loss, lse, gx, gw, gb = got
    for bias in (b, None):
        dol.cross_entropy(x, w, t, loss, lse, bias=bias)
        dol.cross_entropy_backward(x, w, t, lse, g, gx, gw, bias=bias, grad_bias=gb)
        assert bool(torch.isnan(loss[7])) and bool(torch.isnan(lse[7])) and bool(torch.isnan(gx[7]).all())
        assert bool(torch.isnan(gw).all()) and bool(torch.isnan(gb).all()) and bool(torch.isfinite(gx[others]).all())
        if bias is not None:
            assert all(torch.equal(p[others], q[others]) for p, q in zip(got[:3], clean[:3]))
    t[7] = -1
    run_and_check(dol, x, w, b, t, g)
    b[v // 2] = float("nan")
    x[7, 3] = 0.0
    dol.cross_entropy(x, w, t, loss, lse, bias=b)
    dol.cross_entropy_backward(x, w, t, lse, g, gx, gw, bias=b, grad_bias=gb)
    assert bool(torch.isnan(loss[others]).all()) and bool(torch.isnan(lse).all()) and bool(torch.isnan(gx[others]).all()) and float(loss[7]) == 0


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,d,v", [(40, 64, 10), (40, 64, 33), (300, 64, 700), (2000, 128, 2000)])
def test_left_out_rows_beside_what_is_not_finite(dol, n, d, v, dtype):
    """dl of a row that is left out, or has no class, is 0 whatever the biases and weights are: all rows so, all sums are zeros; some rows
    so, their grad_x is zeros where a bias is NaN or infinite."""
    x, w, b, t, g = make(n, d, v, getattr(torch, dtype), seed=v)
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    gx, gw, gb = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    for bad in (float("nan"), float("inf")):
        bias = b.clone()
        bias[v // 3] = bad
        some = t.clone()
        some[::3] = -1
        dol.cross_entropy(x, w, some, loss, lse, bias=bias)
        dol.cross_entropy_backward(x, w, some, lse, g, gx, gw, bias=bias, grad_bias=gb)
        assert not gx[::3].any() and not loss[::3].any()
        weight = w.clone()
        weight[v // 3, 2] = bad
        for ww, bb in ((w, bias), (weight, b), (weight, bias)):
            dol.cross_entropy(x, ww, torch.full_like(t, -1), loss, lse, bias=bb)
            dol.cross_entropy_backward(x, ww, torch.full_like(t, -1), lse, g, None, gw, bias=bb, grad_bias=gb)
            assert not loss.any() and not gw.any() and not gb.any()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,d,v", [(40, 64, 10), (40, 64, 33), (300, 64, 700), (700, 64, 2600)])
def test_a_logit_of_infinity(dol, n, d, v, dtype):
    """The sum of the exponentials is inf and so is its log, for one such class or two in different tiles; the loss is inf, or NaN where the
    target's own logit is inf too.  The other exponentials vanish beside it: grad_bias is -g at the targets."""
    x, w, b, t, g = make(n, d, v, getattr(torch, dtype), seed=v)
    loss, lse, gb = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(v, device="cuda")
    t = (t % (v - 2)) + 1
    t[0] = 0
    for at in ((0,), (0, v - 1)):
        bias = b.clone()
        bias[list(at)] = float("inf")
        dol.cross_entropy(x, w, t, loss, lse, bias=bias)
        assert bool((lse == float("inf")).all()) and bool((loss[1:] == float("inf")).all()) and bool(torch.isnan(loss[0]))
        dol.cross_entropy_backward(x, w, t, lse, g, None, None, bias=bias, grad_bias=gb)
        want = torch.zeros(v, dtype=torch.float64, device="cuda").index_add_(0, t.long(), -g.double())
        size = torch.zeros(v, dtype=torch.float64, device="cuda").index_add_(0, t.long(), g.double().abs())
        rest = torch.ones(v, dtype=torch.bool, device="cuda")
        rest[list(at)] = False
        assert bool(torch.isnan(gb[list(at)]).all()) and bool(((gb.double() - want).abs() <= 32 * U * size)[rest].all())


@pytest.mark.parametrize("n,d,v", [(40, 64, 10), (40, 64, 33), (300, 64, 700), (2000, 128, 2000)])
def test_numbers_at_the_end_of_the_range(dol, n, d, v):
    """x, weight and grad_loss of 3.4e38, which bf16 does not hold: what 32 bits can say of the results is said."""
    top = 3.4e38
    x, w, b, t, g = make(n, d, v, torch.float32, seed=v)
    x[5, 0], g[5] = top, 0.5
    w[:, 0] = 2.0 ** -126 * torch.where(w[:, 0] > 0, 1.0, -1.0)
    run_and_check(dol, x, w, b, t, g)
    x, w, b, t, g = make(n, d, v, torch.float32, seed=v)
    w[3, 0], t[t == 3] = -top, 4
    x[:, 0] = 2.0 ** -126
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    dol.cross_entropy(x, w, t, loss, lse, bias=b)
    ref = reference(x, w, b, t, g)
    bar = ref["err_l"].max(axis=1) + 8 * U * (1 + np.abs(ref["lse"]))
    within(lse, ref["lse"], bar, "lse")
    within(loss, ref["loss"], 2 * bar, "loss")
    for dtype in (torch.float32, torch.bfloat16)[: 1 + (n <= 512)]:
        x, w, b, t, g = make(n, d, v, dtype, seed=v)
        g[5] = top
        run_and_check(dol, x * 2.0 ** -12, w * 2.0 ** -12, b, t, g)


# Every tile that logits and products can take, with several tiles and steps of k each way and remainders in all of them.
FORMS = [("float32", 2000, 130, 2000, "128x128x32", "128x128x32"), ("float32", 1000, 300, 5200, "128x256x32", "128x256x32"),
         ("float32", 300, 256, 3001, "64x64x64", "128x128x32"), ("bfloat16", 2000, 130, 2000, "128x128x64", "128x128x64"),
         ("bfloat16", 2001, 192, 1999, "128x128x64", "128x128x64"), ("bfloat16", 2500, 320, 8200, "256x256x64", "256x256x64"),
         ("bfloat16", 2500, 300, 8201, "256x256x64", "256x256x64"), ("bfloat16", 400, 130, 5000, "128x128x64", "128x128x32"),
         ("bfloat16", 511, 200, 24401, "256x256x64", "128x128x32"), ("bfloat16", 300, 64, 300, "64x64x64", "64x64x64")]


@pytest.mark.parametrize("dtype,n,d,v,logits,products", FORMS)
def test_forms(dol, dtype, n, d, v, logits, products):
    x, w, b, t, g = make(n, d, v, getattr(torch, dtype), seed=d)
    assert dol.cross_entropy_kernel(x, w) == "xent_sums_kernel " + logits
    assert dol.cross_entropy_kernel(x, w, True) == "xent_dlogits_kernel %s, xent_products_kernel %s" % (logits, products)
    t[::11] = -1
    got = run_and_check(dol, x, w, b, t, g)
    again = [torch.empty_like(q) for q in got]
    loss, lse, gx, gw, gb = again
    dol.cross_entropy(x, w, t, loss, lse, bias=b)
    dol.cross_entropy_backward(x, w, t, lse, g, gx, None, bias=b)
    dol.cross_entropy_backward(x, w, t, lse, g, None, gw, bias=b, grad_bias=gb)
    assert all(torch.equal(p, q) for p, q in zip(got, again))


@pytest.mark.parametrize("dtype,n,d,v,logits,products", FORMS)
def test_forms_with_masks_and_strides(dol, dtype, n, d, v, logits, products):
    """Rows left out that hold NaN, classes taken out (the target's own among them, and whole tiles of them), rows of other strides."""
    x, w, b, t, g = make(n, d, v, getattr(torch, dtype), seed=d + 1)
    t[::7] = -1
    t[3::29] = v
    out = (t < 0) | (t >= v)
    x[out], g[out] = float("nan"), float("nan")
    b[v // 3: v // 3 + 600] = float("-inf")
    b[v - 1] = float("-inf")
    x, w = padded(x, 3, float("nan"))[1], padded(w, 5, float("nan"))[1]
    assert dol.cross_entropy_kernel(x, w, True) == "xent_dlogits_kernel %s, xent_products_kernel %s" % (logits, products)
    loss, _, gx, _, _ = run_and_check(dol, x, w, b, t, g, pad=3)
    assert not loss[out].any() and not gx[out].any()
    assert bool(torch.isinf(loss).any()) == bool((~out & torch.isinf(b[t.clamp(0, v - 1).long()])).any())


@pytest.mark.parametrize("n,d,v", [(1, 50, 70), (64, 128, 360), (300, 64, 300), (512, 130, 5000), (511, 200, 24401)])
def test_dl_of_few_rows_in_two_planes(dol, n, d, v):
    """bf16 up to 512 rows: dl has 2^-17 of rounding in its two planes, so that the gradients err by that and by the rounding of the result."""
    x, w, b, t, g = make(n, d, v, torch.bfloat16, seed=v)
    ref = reference(x, w, b, t, g)
    loss, lse, gx, gw = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty_like(x), torch.empty_like(w)
    dol.cross_entropy(x, w, t, loss, lse, bias=b)
    dol.cross_entropy_backward(x, w, t, lse, g, gx, gw, bias=b)
    rel = 2 * ref["err_l"].max(initial=0.0) + 32 * U + 2.0 ** -17
    within(gx, ref["grad_x"], ref["size_x"] * rel + W8 * np.abs(ref["grad_x"]) + 1e-37, "grad_x")
    within(gw, ref["grad_w"], ref["size_w"] * rel + W8 * np.abs(ref["grad_w"]) + 1e-37, "grad_weight")


def rows_in_64_bits(x, w, b, t, at):
    """lse and loss of some rows (all of whose targets count), products in 64 bits on the device, and their bars."""
    xd, wd, t = x[at].double(), w.double(), t[at].long()
    logits = torch.mm(xd, wd.t().contiguous()) + (0 if b is None else b.double())
    lse = torch.logsumexp(logits, 1)
    bar = 16 * U * torch.mm(xd.abs(), wd.t().abs().contiguous()).max(1).values + 8 * U * (1 + lse.abs())
    return lse, lse - logits.gather(1, t[:, None])[:, 0], bar


def test_more_elements_than_a_round_of_workgroups(dol):
    """A million rows: what is laid out, and what is summed up of grad_x, takes its workgroups more than once."""
    n, d, v = (1 << 20) + 5, 72, 300
    x, w, b, t, g = make(n, d, v, torch.bfloat16, seed=1)
    t[::5] = -1
    loss, lse = torch.full((n,), 9.0, device="cuda"), torch.full((n,), 9.0, device="cuda")
    gx, gw, gb = torch.full_like(x, 9.0), torch.full_like(w, 9.0), torch.full_like(b, 9.0)
    dol.cross_entropy(x, w, t, loss, lse, bias=b)
    dol.cross_entropy_backward(x, w, t, lse, g, gx, gw, bias=b, grad_bias=gb)
    kept = torch.nonzero(t >= 0)[:, 0]
    want_lse, want, bar = rows_in_64_bits(x, w, b, t, kept)
    assert bool(((lse[kept].double() - want_lse).abs() <= bar).all()) and bool(((loss[kept].double() - want).abs() <= 2 * bar).all())
    assert not loss[::5].any() and not gx[::5].any()
    xd, wd = x[kept].double(), w.double()
    dl = torch.exp(torch.mm(xd, wd.t().contiguous()) + b.double() - want_lse[:, None])
    dl[torch.arange(kept.numel(), device="cuda"), t[kept].long()] -= 1
    dl *= g[kept].double()[:, None]
    rel = 2 * float(bar.max()) + 32 * U + W8
    for got, ref, size in ((gx[kept], torch.mm(dl, wd), torch.mm(dl.abs(), wd.abs())),
                           (gw, torch.mm(dl.t().contiguous(), xd), torch.mm(dl.abs().t().contiguous(), xd.abs()))):
        assert bool(((got.double() - ref).abs() <= rel * size + W8 * ref.abs() + 1e-37).all())
    assert bool(((gb.double() - dl.sum(0)).abs() <= (rel - W8) * dl.abs().sum(0)).all())


def test_more_tiles_than_a_launch_has_threads_for(dol):
    """2^22 rows into 2^17 classes: 2^23 tiles of 512 threads."""
    n, d, v = 1 << 22, 16, 1 << 17
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("60 GB of memory")
    x, w, b, t, g = make(n, d, v, torch.bfloat16, seed=2, bias=False)
    loss, lse = torch.full((n,), -9.0, device="cuda"), torch.full((n,), -9.0, device="cuda")
    dol.cross_entropy(x, w, t, loss, lse)
    at = torch.cat([torch.arange(0, n, n // 500, device="cuda"), torch.arange(n - 300, n, device="cuda")])
    want_lse, want, bar = rows_in_64_bits(x, w, None, t, at)
    assert bool(((lse[at].double() - want_lse).abs() <= bar).all()) and bool(((loss[at].double() - want).abs() <= 2 * bar).all())
    assert bool((lse > -9).all()) and bool(torch.isfinite(loss).all())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,d,v", [(40, 64, 10), (40, 64, 300), (300, 64, 3001), (2000, 130, 2000)])
def test_logits_far_from_zero(dol, n, d, v, dtype):
    """Masks of every finite size over part of the classes, whole tiles of them, and a class that stands far above or all others far below:
    exponentials of differences, whatever the logits themselves are."""
    x, w, b, t, g = make(n, d, v, getattr(torch, dtype), seed=n + v)
    for far in (-2e6, -1e8, -1e10, -1e20, -1e30, -1e37, -3e38):
        bias = b.clone()
        bias[: v * 3 // 4] = far
        run_and_check(dol, x, w, bias, torch.full_like(t, v - 1), g)
    t = t % (v - 1) + 1
    for far in (2e6, 1e8, 3e9, 1e10, 1e20, 1e30, 1e38, -1e8, -1e10, -1e20, -1e30, -1e38):
        bias = torch.full_like(b, min(0.0, 2 * far))
        bias[0] = far
        run_and_check(dol, x, w, bias, t, g)
