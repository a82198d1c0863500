"""The recogniser with residual blocks between its norm and its head: linear layers, norms between blocks and clipped gradients as one step uses them.

Bars.  As for the recogniser without blocks: a step is in 32 bits (u = 2^-24), and a gradient a sum over some thousand terms through up to ten more
layers, each of which errs by some u times the magnitudes that it adds up: 2^-24 x 512 = 3e-5 of the gradient's norm.  A gate's and a post norm's
gradients add up terms that cancel (a row's norm has no gradient along the row), some tenfold: 3e-4."""
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


def norm(v, gamma):
    return v * (v.pow(2).mean(1, keepdim=True) + 1e-6).rsqrt() * gamma


def plain(model, w, patches, target, labels):
    """Loss of one mini-batch by elementary operations, in 64 bits with autograd."""
    M, n, batch = model.images, model.n, model.batch
    h = patches @ w["w1"].T
    x = h.view(M, model.points, model.groups, -1)
    xhat = ((x - x.mean((1, 3), keepdim=True)) / (x.var((1, 3), unbiased=False, keepdim=True) + 1e-5).sqrt()).view_as(h)
    s = torch.nn.functional.silu(w["gamma"] * xhat + w["beta"]).reshape(M * model.points, -1)
    for b in range(model.blocks):
        u = torch.nn.functional.silu(norm(s, w["norm%d" % b]) @ w["wa%d" % b].T + w["ba%d" % b]) @ w["wb%d" % b].T + w["bb%d" % b]
        s = s + (w["gate%d" % b] * norm(u, w["post%d" % b]) if b < model.blocks - 1 else u)
    f = s.reshape(M, -1)
    logp = torch.log_softmax(f @ w["w2"].T + w["b2"], 1)
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


@pytest.mark.parametrize("n,batch,channels,blocks,widen", [(3, 64, 32, 3, 4), (2, 5, 12, 1, 3), (2, 3, 20, 2, 1), (2, 33, 48, 4, 2)])
def test_gradients_of_a_step(T, n, batch, channels, blocks, widen):
    model = T.SumRecogniser(n_digits=n, batch=batch, channels=channels, groups=4, labels_weight=0.5, blocks=blocks, widen=widen)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for k, v in model.params.items():                   # no parameter at the value that leaves its neighbour out
        if not k.startswith("w"):
            v.add_(0.2 * torch.randn(v.shape, generator=gen, device="cuda"))
    images, sums, labels, _ = T.SyntheticDigits(seed=1).draw(n, batch, 0.5, "cuda")
    labels[0] = 3
    patches = model.patches(images)
    model.target.copy_(sums)
    model.backward(patches, model.forward(patches, labels), labels)
    params = {k: v.cpu().double().requires_grad_() for k, v in model.params.items()}
    want = plain(model, params, patches.cpu().double(), sums.cpu(), labels.cpu())
    want.backward()
    program, labelled = model.losses()
    assert abs(program + labelled - float(want.detach())) <= 3e-5 * float(want.detach())
    for k, v in params.items():
        off = float((model.grads[k].cpu().double() - v.grad).norm() / v.grad.norm())
        assert off <= (3e-4 if k.startswith(("gate", "post")) else 3e-5), "%s: %g" % (k, off)


def test_clipped_gradients(T):
    images, sums, labels, _ = T.SyntheticDigits(seed=2).draw(3, 64, 0.3, "cuda")
    free, held = T.SumRecogniser(blocks=2), T.SumRecogniser(blocks=2, max_norm=0.05)
    patches = free.patches(images)
    for m in (free, held):
        m.step(patches, sums, labels)
    norm = float(np.sqrt(sum(float(g.double().pow(2).sum()) for g in free.grads.values())))
    assert norm > 0.05 and abs(float(held.norm) - norm) <= 2e-7 * norm and abs(float(held.coef) * norm - 0.05) <= 1e-6
    for k, g in free.grads.items():
        torch.testing.assert_close(held.grads[k], g * held.coef, rtol=1e-6, atol=0)
    # vectors move by the clipped gradient, matrices as far as ever
    torch.testing.assert_close(held.params["beta"], -held.lr_vector * held.grads["beta"], rtol=1e-6, atol=0)
    torch.testing.assert_close(held.updates["wa1"], free.updates["wa1"], rtol=1e-3, atol=1e-5)


def test_steps_in_a_graph(T):
    """Two models from one seed: one steps eagerly, the other by replays of one captured step."""
    images, sums, labels, _ = T.SyntheticDigits(seed=4).draw(3, 64, 0.2, "cuda")
    eager, caught = (T.SumRecogniser(seed=5, blocks=3, max_norm=1.0) for _ in range(2))
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


def test_training_runs(T, capsys):
    T.main(steps=3, blocks=2, max_norm=1.0)
    lines = capsys.readouterr().out.splitlines()
    assert len(lines) == 2 and all("nan" not in line for line in lines)
