"""A recogniser trained under a Sum-N program: one step's gradients against the same model in 64 bits on the host, and a short training.

Bars.  The step is in 32 bits (u = 2^-24): a gradient is a sum over some thousand terms through three layers, each of which errs by some
u times the magnitudes that it adds up.  A relative error of 2^-24 x 256 = 1.5e-5 of the gradient's norm leaves two orders for the sums'
lengths and for cancellation.  The update is orthogonal up to the polynomial: its singular values lie in 0.6 .. 1.3 (five steps take any
value above 0.02 of the norm there)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def T():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2410_03348_amd import training
    return training


def plain(model, params, patches, target, labels):
    """Loss of one mini-batch by elementary operations, in 64 bits with autograd."""
    M, n, batch = model.images, model.n, model.batch
    h = patches @ params["w1"].T
    x = h.view(M, model.points, model.groups, -1)
    mean = x.mean((1, 3), keepdim=True)
    xhat = ((x - mean) / (((x - mean) ** 2).mean((1, 3), keepdim=True) + 1e-5).sqrt()).view_as(h)
    z = params["gamma"] * xhat + params["beta"]
    f = (z * torch.sigmoid(z)).reshape(M, -1)
    logp = torch.log_softmax(f @ params["w2"].T + params["b2"], 1)
    known = labels >= 0
    labelled = -logp[known].gather(1, labels[known, None].long()).mean()
    p = logp.exp().view(n, batch, 10)
    acc = p[0]
    for t in range(1, n):
        nxt = torch.zeros(batch, acc.shape[1] + 9, dtype=acc.dtype)
        for d in range(10):
            nxt = nxt + torch.nn.functional.pad(acc * p[t][:, d:d + 1], (d, 9 - d))
        acc = nxt
    return -acc.gather(1, target[:, None].long()).log().mean() + model.labels_weight * labelled


@pytest.mark.parametrize("n,batch,channels,groups,share", [(3, 64, 32, 8, 0.1), (2, 5, 12, 4, 0.5), (4, 33, 48, 1, 0.9)])
def test_gradients_of_a_step(T, n, batch, channels, groups, share):
    model = T.SumRecogniser(n_digits=n, batch=batch, channels=channels, groups=groups, labels_weight=0.5)
    images, sums, labels, _ = T.SyntheticDigits(seed=1).draw(n, batch, share, "cuda")
    labels[0] = 3                       # (at least one)
    patches = model.patches(images)
    model.target.copy_(sums)
    model.backward(patches, model.forward(patches, labels), labels)
    params = {k: v.cpu().double().requires_grad_() for k, v in model.params.items()}
    want = plain(model, params, patches.cpu().double(), sums.cpu(), labels.cpu())
    want.backward()
    program, labelled = model.losses()
    assert abs(program + labelled - float(want.detach())) <= 1.5e-5 * float(want.detach())
    for k, v in params.items():
        off = float((model.grads[k].cpu().double() - v.grad).norm() / v.grad.norm())
        assert off <= 1.5e-5, "%s: %g" % (k, off)


def test_update_is_orthogonal(T):
    model = T.SumRecogniser()
    images, sums, labels, _ = T.SyntheticDigits(seed=2).draw(model.n, model.batch, 0.3, "cuda")
    before = model.params["w1"].clone()
    model.step(model.patches(images), sums, labels)
    s = np.linalg.svd(model.updates["w1"].cpu().double().numpy(), compute_uv=False)
    m = np.linalg.svd(model.moments["w1"].cpu().double().numpy(), compute_uv=False)
    large = m > 0.02 * np.linalg.norm(m)
    assert large.any() and s[large].min() > 0.6 and s.max() < 1.3
    moved = float((model.params["w1"] - before).norm())
    np.testing.assert_allclose(moved, model.lr * 2 ** 0.5 * float(model.updates["w1"].norm()), rtol=1e-4)


def test_training_recognises_the_digits(T):
    """Labels of one digit in ten and the sums of all: the digits are told apart after a hundred steps, the losses near zero."""
    model, data = T.SumRecogniser(), T.SyntheticDigits()
    first = None
    for _ in range(100):
        images, sums, labels, digits = data.draw(model.n, model.batch, 0.1, "cuda")
        model.step(model.patches(images), sums, labels)
        first = first or model.losses()
    program, labelled = model.losses()
    assert float((model.p.argmax(2) == digits).float().mean()) > 0.95 and program < first[0] / 4 and labelled < first[1] / 4


def test_a_step_in_a_graph(T):
    """Two models from one seed: one steps eagerly, the other by replays of one captured step."""
    data = T.SyntheticDigits(seed=4)
    images, sums, labels, _ = data.draw(3, 64, 0.2, "cuda")
    eager, caught = T.SumRecogniser(seed=5), T.SumRecogniser(seed=5)
    patches = eager.patches(images)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        caught.step(patches, sums, labels)
    torch.cuda.current_stream().wait_stream(side)
    eager.step(patches, sums, labels)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        caught.step(patches, sums, labels)
    for _ in range(4):
        g.replay()
        eager.step(patches, sums, labels)
        torch.cuda.synchronize()
        for k in eager.params:
            torch.testing.assert_close(caught.params[k], eager.params[k], rtol=1e-5, atol=1e-6)


def test_calls_that_overlap_on_two_streams(T):
    """Calls without a workspace of the caller's, one on the current stream and one on a side stream with no wait between them: their workspaces
    are not the same memory, and each result is what the call alone gives."""
    from paper_2410_03348_amd import binding as dol
    side = torch.cuda.Stream()
    # the allocator gives the current stream a block back at once; a call on the side stream does not get it
    block = torch.empty(3 << 20, dtype=torch.uint8, device="cuda")
    at = block.data_ptr()
    del block
    address, n, keep = dol._workspace(None, 3 << 20, "cuda", side)
    assert not at <= address < at + n and not address <= at < address + n
    assert dol._workspace(None, 4096, "cuda", side.cuda_stream)[0] not in (None, at)
    del keep

    gen = torch.Generator(device="cuda").manual_seed(3)
    calls = []
    for k in range(2):
        x, w = torch.randn(700, 96, generator=gen, device="cuda"), torch.randn(900, 96, generator=gen, device="cuda") * 0.2
        t = torch.randint(0, 900, (700,), generator=gen, device="cuda", dtype=torch.int32)
        g, m = torch.rand(700, generator=gen, device="cuda"), torch.randn(200, 300, generator=gen, device="cuda")
        a = torch.randn(1, 40000, 16, generator=gen, device="cuda")
        out = [torch.empty(700, device="cuda"), torch.empty(700, device="cuda"), torch.empty_like(x), torch.empty_like(w), torch.empty_like(m),
               torch.empty_like(a), torch.empty(1, 2, device="cuda"), torch.empty(1, 2, device="cuda"), torch.empty_like(a), torch.empty(16, device="cuda")]

        def call(stream, x=x, w=w, t=t, g=g, m=m, a=a, out=out):
            loss, lse, gx, gw, u, y, mean, rstd, ga, gg = out
            dol.cross_entropy(x, w, t, loss, lse, stream=stream)
            dol.cross_entropy_backward(x, w, t, lse, g, gx, gw, stream=stream)
            dol.newton_schulz(m, u, stream=stream)
            dol.group_norm(a, None, None, 2, y, mean, rstd, act="silu", stream=stream)
            dol.group_norm_backward(a, None, None, 2, mean, rstd, y, ga, gg, None, act="silu", stream=stream)

        call(None)
        torch.cuda.synchronize()
        calls.append((call, out, [q.clone() for q in out]))
    torch.cuda.synchronize()
    for _ in range(5):
        for _, out, _ in calls:
            for q in out:
                q.zero_()
        torch.cuda.synchronize()
        calls[0][0](None)
        calls[1][0](side)
        torch.cuda.synchronize()
        for _, out, want in calls:
            assert all(torch.equal(p, q) for p, q in zip(out, want))
