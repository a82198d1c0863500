"""dol_grad_norm and dol_clip_grads against the definition in 64 bits, through the binding (needs an MI355X).

Bars, u = 2^-24: squares and sums are in 64 bits (off by less than 2^-29 of the sum for the sizes here), so the norm is off by its rounding, u, and
2^-29; coef by its own rounding of the same kind; a float result by coef's rounding and the product's, 2 u, or half the smallest number, a bf16 one
by half a step, 2^-8, beside them.
"""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U, SLACK = 2.0 ** -24, 2.0 ** -29
HALF = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module")
def dol():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2410_03348_amd import binding
    return binding


def make(sizes, dtypes, seed=0, scale=1.0, shift=0):
    """Tensors of these sizes one behind the other in a buffer for each type, from element `shift` on: aligned to their elements alone."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    at, flat = {}, {}
    for n, t in zip(sizes, dtypes):
        at[t] = at.get(t, shift) + n
    for t, n in at.items():
        flat[t] = (torch.randn(n + 5, generator=gen, device="cuda") * scale).to(t)
    out, at = [], {t: shift for t in flat}
    for n, t in zip(sizes, dtypes):
        out.append(flat[t][at[t]:at[t] + n])
        at[t] += n
    return out, flat


def exact(tensors, max_norm, eps):
    norm = math.sqrt(sum(float(t.double().pow(2).sum()) for t in tensors))
    return norm, min(1.0, max_norm / (norm + eps)) if norm + eps else (math.nan if max_norm == 0 else 1.0)


def guarded(n):
    buf = torch.full((n + 2048,), 77, dtype=torch.uint8, device="cuda")
    return buf, buf[1024:1024 + n]


def check(dol, tensors, max_norm, eps=1e-6, out=None, stream=None):
    norm, coef = torch.full((1,), 9.0, device="cuda"), torch.full((1,), 9.0, device="cuda")
    want, ratio = exact(tensors, max_norm, eps)
    before = [t.double() for t in tensors]
    grads = dol.TensorList(tensors)
    lists = dol.TensorList(out) if out is not None else None
    buf, ws = guarded(dol.grad_norm_workspace(grads))
    dol.grad_norm(grads, norm, workspace=ws)
    assert abs(float(norm) - want) <= want * (U + SLACK)
    norm.fill_(9.0)
    dol.clip_grads(grads, max_norm, norm, coef, out=lists, eps=eps, workspace=ws)
    assert bool((buf[:1024] == 77).all()) and bool((buf[1024 + ws.numel():] == 77).all())
    assert abs(float(norm) - want) <= want * (U + SLACK)
    assert abs(float(coef) - ratio) <= ratio * (U + 2 * SLACK)
    for b, t, r in zip(before, tensors, out if out is not None else tensors):
        bar = (b * ratio).abs() * (HALF[r.dtype] + 2 * U + 4 * SLACK) + (2.0 ** -150 if r.dtype == torch.float32 else 2.0 ** -134)
        assert bool(((r.double() - b * ratio).abs() <= bar).all())
        if out is not None:
            assert bool((t.double() == b).all())
    return norm, coef


# both sides of what one workgroup holds (64 chunks of 1 024), and of the chunks themselves
SIZES = [[1], [7, 1], [1023, 1025], [8192], [8191, 8193], [3, 0, 24577, 2], [65536], [65537], [1] * 64, [1] * 65, [100001], [33] * 300, [512, 32, 32, 15680, 10], [1 << 21, 5, 70000]]


@pytest.mark.parametrize("dtypes", ["f", "b", "fb"])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "x".join(map(str, s[:4])))
@pytest.mark.parametrize("inplace", [True, False])
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_sizes(dol, sizes, dtypes, inplace, shift):
    types = [{"f": torch.float32, "b": torch.bfloat16}[dtypes[k % len(dtypes)]] for k in range(len(sizes))]
    tensors, _ = make(sizes, types, seed=len(sizes), shift=shift)
    want, _ = exact(tensors, 1.0, 0.0)
    out, flat = make(sizes, types, seed=5, shift=2) if not inplace else (None, {})
    guards = {t: (f[:2].clone(), f[-5:].clone()) for t, f in flat.items()}
    check(dol, tensors, 0.3 * want, out=out)
    for t, f in flat.items():           # what lies before the first tensor and behind the last
        assert bool((f[:2] == guards[t][0]).all()) and bool((f[-5:] == guards[t][1]).all())


@pytest.mark.parametrize("inplace", [True, False])
@pytest.mark.parametrize("large", [0, 100000])
def test_a_norm_that_is_allowed_leaves_every_bit(dol, inplace, large):
    tensors, _ = make([1000, 33, 9000 + large], [torch.float32, torch.bfloat16, torch.float32])
    before = [t.clone() for t in tensors]
    out = None if inplace else [torch.zeros_like(t) for t in tensors]
    _, coef = check(dol, tensors, 1e4, out=out)
    assert float(coef) == 1.0
    for b, r in zip(before, tensors if inplace else out):
        assert torch.equal(b, r)


def test_nothing(dol):
    check(dol, [], 1.0)
    check(dol, [torch.empty(0, device="cuda"), torch.empty(0, 3, device="cuda", dtype=torch.bfloat16)], 1.0)
    check(dol, [torch.zeros(5000, device="cuda")], 1.0)
    check(dol, [torch.ones(5000, device="cuda")], 0.0)


@pytest.mark.parametrize("scale", [1e-38, 1e-25, 1e25, 3e36])
def test_squares_past_a_floats_range(dol, scale):
    tensors, _ = make([5000, 77], [torch.float32, torch.bfloat16], scale=scale)
    want, _ = exact(tensors, 1.0, 0.0)
    check(dol, tensors, 0.5 * want, eps=0.0, out=[torch.empty_like(t) for t in tensors])


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("n", [60010, 70000])
def test_a_norm_that_is_not_finite(dol, value, n):
    tensors, _ = make([n, 33], [torch.float32, torch.bfloat16])
    tensors[0][60001] = value
    norm, coef = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    dol.clip_grads(dol.TensorList(tensors), 1.0, norm, coef)
    if math.isnan(value):
        assert math.isnan(float(norm)) and math.isnan(float(coef)) and all(bool(t.isnan().all()) for t in tensors)
    else:
        assert float(norm) == math.inf and float(coef) == 0.0
        assert math.isnan(float(tensors[0][60001])) and float(tensors[0].nan_to_num().abs().sum()) == 0.0 and float(tensors[1].abs().sum()) == 0.0


def test_tensors_in_another_order(dol):
    gen = torch.Generator(device="cuda").manual_seed(1)
    a, b = torch.randn(77, 130, generator=gen, device="cuda"), torch.randn(4, 5, 6, 7, generator=gen, device="cuda")
    tensors = [a.t(), b.permute(0, 2, 3, 1), torch.ones(1, 9, device="cuda")[:, :1]]
    out = [torch.empty_like(t, memory_format=torch.preserve_format) for t in tensors]
    check(dol, tensors, 1.0, out=out)
    with pytest.raises(AssertionError):
        dol.clip_grads(dol.TensorList(tensors), 1.0, torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda"),
                       out=dol.TensorList([t.contiguous() for t in tensors]))
    check(dol, tensors, 1.0)


def test_refused_lists(dol):
    a = torch.randn(1000, device="cuda")
    for bad in ([torch.zeros(3)], [torch.zeros(3, device="cuda", dtype=torch.float16)], [torch.zeros(4, 4, device="cuda")[:, :3]],
                [torch.zeros(1, device="cuda").expand(5)]):
        with pytest.raises(AssertionError):
            dol.TensorList(bad)
    norm, coef = torch.full((1,), 9.0, device="cuda"), torch.full((1,), 9.0, device="cuda")
    one, parts, twice, late = (dol.TensorList(x) for x in ([a[:500], a[500:]], [a[500:], a[:500]], [a[:500], a[:500]], [a[1:501], a[501:1000]]))
    other = dol.TensorList([torch.empty(500, device="cuda"), torch.empty(500, device="cuda")])
    before = a.clone()
    for grads, out, why in ((twice, None, "share"), (twice, other, "share"), (other, twice, "share"), (one, parts, "another"), (one, late, "ESHAPE"),
                            (one, dol.TensorList([a[:500]]), "ESHAPE"), (one, dol.TensorList([a[:500], a[500:].bfloat16()]), "ESHAPE"),
                            (dol.TensorList([a[:500]]), dol.TensorList([a[1:501]]), "another")):
        with pytest.raises(dol.DolError, match=why):
            dol.clip_grads(grads, 1.0, norm, coef, out=out)
    for most, eps in ((-1.0, 0.0), (math.nan, 0.0), (1.0, -1.0), (1.0, math.nan)):
        with pytest.raises(dol.DolError, match="at least 0"):
            dol.clip_grads(one, most, norm, coef, eps=eps)
    with pytest.raises(dol.DolError, match="workspace"):
        dol.clip_grads(dol.TensorList([torch.empty(70000, device="cuda")]), 1.0, norm, coef, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(a, before) and float(norm) == 9.0 and float(coef) == 9.0
    dol.grad_norm(twice, norm)
    want = math.sqrt(2.0) * float(a[:500].double().norm())
    assert abs(float(norm) - want) <= want * (U + SLACK)
    dol.clip_grads(one, 1.0, norm, coef, out=dol.TensorList([a[:500], a[500:]]))       # in place, by another list of the same buffers
    assert abs(float(a.double().norm()) - 1.0) < 1e-5
    one.destroy()
    with pytest.raises(dol.DolError, match="NULL"):
        dol.grad_norm(one, norm)


def test_more_elements_than_32_bits_count(dol):
    n = (1 << 31) + 8195
    t = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    at = [0, (1 << 31) - 1, 1 << 31, n - 1]
    for k in at:
        t[k] = 3.0
    norm, coef = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    dol.clip_grads(dol.TensorList([t]), 3.0, norm, coef, eps=0.0)
    assert float(norm) == 6.0 and float(coef) == 0.5
    for k in at:
        assert float(t[k]) == 1.5
        t[k] = 0.0
    assert int(t.count_nonzero()) == 0


@pytest.mark.parametrize("n", [3000, 300000])
def test_the_same_bits_on_any_stream_and_in_a_graph(dol, n):
    tensors, _ = make([n, 5, n // 4 + 1], [torch.float32, torch.bfloat16, torch.bfloat16], seed=3)
    out = [[torch.empty_like(t) for t in tensors] for _ in range(2)]
    grads, lists = dol.TensorList(tensors), [dol.TensorList(o) for o in out]
    norm, coef = (torch.zeros(2, 1, device="cuda") for _ in range(2))
    size = dol.grad_norm_workspace(grads)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        dol.clip_grads(grads, 2.0, norm[1], coef[1], out=lists[1], workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        dol.clip_grads(grads, 2.0, norm[1], coef[1], out=lists[1], workspace=ws)
    for k in range(4):
        for t in tensors:
            t.copy_(torch.randn_like(t.float()) * (0.001 if k == 2 else 1.0))
        graph.replay()
        dol.clip_grads(grads, 2.0, norm[0], coef[0], out=lists[0])
        torch.cuda.synchronize()
        assert torch.equal(norm[0], norm[1]) and torch.equal(coef[0], coef[1]) and all(torch.equal(a, b) for a, b in zip(*out))
        assert (float(coef[0]) == 1.0) == (k == 2)
    dol.clip_grads(grads, 2.0, norm[0], coef[0], out=lists[0], stream=side)
    torch.cuda.synchronize()
    assert torch.equal(norm[0], norm[1]) and all(torch.equal(a, b) for a, b in zip(*out))
