"""Training a digit recogniser under a Sum-N program, where some of the digits are labelled as well.

The network in front of a Dolphin program (Fig. 2 of the paper) and what trains it, on the library's calls:

    images [n, batch, side, side]  as patches [n * batch, points, patch * patch]
      h = patches w1^T                                           plain matrix product
      y = silu(group_norm(h))                                    dol.group_norm
      s = y as one row a point, and for each of `blocks`
        v = norm(s)                                              dol.residual_norm, with the end of the block before
        u = silu(v wa^T + ba) wb^T + bb                          dol.linear twice
        s <- s + gate * norm(u); the last: s + u                 dol.residual_norm; the residual of dol.linear
      f = s as one row an image
      loss and lse of the digits that have a label               dol.cross_entropy
      p = exp(f w2^T + b2 - lse)                                 the softmax, from the same lse
      sum of n digit Distributions, -log p[target], grad_p       dol.fold_apply2, one launch
    and back
      grad f, w2, b2 of the labels' loss                         dol.cross_entropy_backward
      the blocks' gradients                                      dol.linear_backward, dol.residual_norm_backward
      grad h, gamma, beta                                        dol.group_norm_backward
      all gradients times min(1, max_norm / their norm)          dol.clip_grads
      matrices: momentum, its orthogonalisation as the update    dol.newton_schulz

``step`` only issues asynchronous calls on the current stream.  What passes between the library's calls is in buffers that the constructor
allocates; logits, masks, torch's temporaries and the calls' workspaces come from torch's allocator, which has them again a step later.

    python -m paper_2410_03348_amd.training [--blocks N] [--max-norm X]     # trains on seeded synthetic digits and prints its course
"""
from __future__ import annotations

import argparse
import math
from typing import Optional

import numpy as np
import torch

from . import binding as dol
from .programs import sum_table_of

DIGITS = np.arange(10, dtype=np.int32)


class SumRecogniser:
    """n_digits images to a sample; labels_weight: of the labelled digits' mean loss beside the samples' mean -log p[sum]; blocks: residual
    blocks over the channels of each point, `widen` times as wide inside; max_norm: of all gradients together (None: as they come)."""

    def __init__(self, n_digits: int = 3, batch: int = 64, side: int = 28, patch: int = 4, channels: int = 32, groups: int = 8,
                 labels_weight: float = 1.0, lr: float = 0.02, lr_vector: float = 0.01, momentum: float = 0.9, seed: int = 0, device="cuda",
                 blocks: int = 0, widen: int = 4, max_norm: Optional[float] = None):
        assert side % patch == 0 and channels % groups == 0
        self.n, self.batch, self.side, self.patch, self.groups = n_digits, batch, side, patch, groups
        self.labels_weight, self.lr, self.lr_vector, self.momentum = labels_weight, lr, lr_vector, momentum
        self.images, self.points, self.channels = n_digits * batch, (side // patch) ** 2, channels
        self.width = self.points * channels
        self.blocks, self.max_norm = blocks, max_norm
        gen = torch.Generator().manual_seed(seed)

        def weight(rows, cols):
            return (torch.randn(rows, cols, generator=gen) / math.sqrt(cols)).to(device)

        def empty(*shape):
            return torch.empty(shape, device=device)

        self.params = {"w1": weight(channels, patch * patch), "gamma": torch.ones(channels, device=device),
                       "beta": torch.zeros(channels, device=device), "w2": weight(10, self.width), "b2": torch.zeros(10, device=device)}
        for b in range(blocks):
            wide = widen * channels
            self.params.update({"norm%d" % b: torch.ones(channels, device=device), "wa%d" % b: weight(wide, channels), "ba%d" % b: torch.zeros(wide, device=device),
                                "wb%d" % b: weight(channels, wide), "bb%d" % b: torch.zeros(channels, device=device)})
            if b < blocks - 1:          # the last one's result is added as it is
                self.params.update({"post%d" % b: torch.ones(channels, device=device), "gate%d" % b: torch.ones(1, channels, device=device)})
        self.grads = {k: torch.empty_like(v) for k, v in self.params.items()}
        matrices = [k for k in self.params if k.startswith("w")]
        self.moments = {k: torch.zeros_like(self.params[k]) for k in matrices}
        self.updates = {k: torch.empty_like(self.params[k]) for k in matrices}
        if max_norm is not None:
            self.all_grads, self.norm, self.coef = dol.TensorList(self.grads.values()), empty(1), empty(1)
        rows = self.images * self.points
        # a block's: its input, normed; inside, before and behind the activation function; its result; rstd's of its result and of its input
        self.inside = [dict(v=empty(rows, channels), z=empty(rows, widen * channels), t=empty(rows, widen * channels), u=empty(rows, channels),
                            s=empty(rows, channels), rstd_u=empty(rows), rstd_v=empty(rows)) for _ in range(blocks)]
        if blocks:
            self.grad_s, self.grad_u, self.grad_v, self.grad_t = (empty(rows, k * channels) for k in (1, 1, 1, widen))
        self.h, self.y = empty(self.images, self.points, channels), empty(self.images, self.points, channels)
        self.grad_f, self.grad_h = empty(self.images, self.width), empty(self.images, self.points, channels)
        self.mean, self.rstd = empty(self.images, groups), empty(self.images, groups)
        self.label_loss, self.lse, self.scale = empty(self.images), empty(self.images), empty(self.images)
        self.p, self.grad_p = empty(n_digits, batch, 10), empty(n_digits, batch, 10)
        # the program: the sum of the samples' digits, its loss and its gradients by one launch
        self.digits = [dol.Dist(DIGITS, self.p[t]) for t in range(n_digits)]
        tables, syms = [], DIGITS
        for _ in range(1, n_digits):
            tables.append(dol.FnTable.create_dense(sum_table_of(syms, DIGITS)))
            syms = tables[-1].out_syms
        self.target = torch.zeros(batch, dtype=torch.int32, device=device)
        self.out = dol.Dist.empty(syms, batch, device)
        self.fold = dol.Fold(self.digits, tables, out=self.out, target_col=self.target, grad_inputs=[self.grad_p[t] for t in range(n_digits)])

    def patches(self, images: torch.Tensor) -> torch.Tensor:
        """[n, batch, side, side] as [n * batch, points, patch * patch]."""
        k, s = self.patch, self.side // self.patch
        return images.reshape(self.images, s, k, s, k).transpose(2, 3).reshape(self.images, self.points, k * k).contiguous()

    def forward(self, patches: torch.Tensor, labels: torch.Tensor) -> torch.Tensor:
        """The digits' Distributions into self.p; labels int32 [n * batch], -1 where a digit has none.  Returns the features."""
        w = self.params
        torch.matmul(patches, w["w1"].T, out=self.h)
        dol.group_norm(self.h, w["gamma"], w["beta"], self.groups, self.y, self.mean, self.rstd, act="silu")
        f = self.through_blocks(self.y.view(-1, self.channels)).view(self.images, self.width)
        dol.cross_entropy(f, w["w2"], labels, self.label_loss, self.lse, bias=w["b2"])
        torch.exp(torch.addmm(w["b2"], f, w["w2"].T).sub_(self.lse[:, None]), out=self.p.view(self.images, 10))
        return f

    def through_blocks(self, s: torch.Tensor) -> torch.Tensor:
        """The stream of activations [images * points, channels] behind the last block."""
        w = self.params
        for b, m in enumerate(self.inside):
            if b == 0:
                dol.residual_norm(None, s, None, None, w["norm0"], None, m["v"], rstd_h=m["rstd_v"], norm_u=False)
            dol.linear(m["v"], w["wa%d" % b], m["t"], bias=w["ba%d" % b], act="silu", z=m["z"])
            if b == self.blocks - 1:
                dol.linear(m["t"], w["wb%d" % b], m["s"], bias=w["bb%d" % b], residual=s)
            else:
                dol.linear(m["t"], w["wb%d" % b], m["u"], bias=w["bb%d" % b])
                after = self.inside[b + 1]
                dol.residual_norm(s, m["u"], w["post%d" % b], w["gate%d" % b], w["norm%d" % (b + 1)], m["s"], after["v"], m["rstd_u"], after["rstd_v"])
            s = m["s"]
        return s

    def back_through_blocks(self, s: torch.Tensor, grad: torch.Tensor) -> torch.Tensor:
        """The gradient of the stream s in front of the blocks from that behind them; the blocks' own into self.grads."""
        w, g = self.params, self.grads
        grad_u = grad
        for b in reversed(range(self.blocks)):
            m = self.inside[b]
            dol.linear_backward(m["t"], w["wb%d" % b], grad_u, self.grad_t, g["wb%d" % b], grad_bias=g["bb%d" % b])
            dol.linear_backward(m["v"], w["wa%d" % b], self.grad_t, self.grad_v, g["wa%d" % b], grad_bias=g["ba%d" % b], act="silu", z=m["z"])
            if b == 0:
                dol.residual_norm_backward(None, s, None, None, w["norm0"], None, m["rstd_v"], grad, self.grad_v, None, self.grad_s, None, None, g["norm0"],
                                           norm_u=False)
            else:
                before = self.inside[b - 1]
                x = self.inside[b - 2]["s"] if b > 1 else s
                dol.residual_norm_backward(x, before["u"], w["post%d" % (b - 1)], w["gate%d" % (b - 1)], w["norm%d" % b], before["rstd_u"], m["rstd_v"], grad,
                                           self.grad_v, self.grad_s, self.grad_u, g["post%d" % (b - 1)], g["gate%d" % (b - 1)], g["norm%d" % b])
                grad_u = self.grad_u
            grad = self.grad_s
        return grad

    def backward(self, patches: torch.Tensor, f: torch.Tensor, labels: torch.Tensor):
        """Gradients of mean -log p[sum] + labels_weight * the labelled digits' mean loss into self.grads."""
        w, g = self.params, self.grads
        dol.fold_apply2(self.fold)
        labelled = labels >= 0
        torch.div(labelled, labelled.sum().clamp_(min=1), out=self.scale).mul_(self.labels_weight)
        dol.cross_entropy_backward(f, w["w2"], labels, self.lse, self.scale, self.grad_f, g["w2"], bias=w["b2"], grad_bias=g["b2"])
        p, gp = self.p.view(self.images, 10), self.grad_p.view(self.images, 10)
        gl = p * (gp - (p * gp).sum(1, keepdim=True)) / self.batch          # the program's gradient of the logits
        self.grad_f.addmm_(gl, w["w2"])
        g["w2"].addmm_(gl.T, f)
        g["b2"].add_(gl.sum(0))
        grad_y = self.back_through_blocks(self.y.view(-1, self.channels), self.grad_f.view(-1, self.channels))
        dol.group_norm_backward(self.h, w["gamma"], w["beta"], self.groups, self.mean, self.rstd, grad_y.view_as(self.h), self.grad_h,
                                g["gamma"], g["beta"], act="silu")
        torch.matmul(self.grad_h.view(-1, self.channels).T, patches.view(-1, self.patch ** 2), out=g["w1"])

    def update(self):
        """Matrices by their orthogonalised momentum, at a size that does not depend on the gradient's; vectors by the gradient."""
        if self.max_norm is not None:
            dol.clip_grads(self.all_grads, self.max_norm, self.norm, self.coef)
        for k, w in self.params.items():
            if k in self.moments:
                m = self.moments[k].mul_(self.momentum).add_(self.grads[k])
                dol.newton_schulz(m, self.updates[k])
                w.sub_(self.updates[k], alpha=self.lr * math.sqrt(max(1.0, w.shape[0] / w.shape[1])))
            else:
                w.sub_(self.grads[k], alpha=self.lr_vector)

    def step(self, patches: torch.Tensor, target: torch.Tensor, labels: torch.Tensor):
        """One update from one mini-batch; target int32 [batch]: the samples' sums."""
        self.target.copy_(target)
        f = self.forward(patches, labels)
        self.backward(patches, f, labels)
        self.update()

    def losses(self):
        """(mean -log p[sum], mean loss of the labelled digits) of the last mini-batch, on the host; label_loss is 0 without a label."""
        at = self.out.prob[:, :self.out.n_sym].gather(1, self.target[:, None].long())[:, 0]
        return float(-at.clamp(min=torch.finfo(torch.float32).tiny).log().mean()), float((self.label_loss * self.scale).sum())


class SyntheticDigits:
    """Ten random prototypes of images and noise around them, drawn on the host."""

    def __init__(self, side: int = 28, noise: float = 0.5, seed: int = 0):
        self.gen = torch.Generator().manual_seed(seed)
        self.noise = noise
        self.prototypes = torch.randn(10, side, side, generator=self.gen)

    def draw(self, n_digits: int, batch: int, labelled: float, device):
        """(images [n, batch, side, side], sums int32 [batch], labels int32 [n * batch], of which a share `labelled` is not -1, digits)."""
        digits = torch.randint(0, 10, (n_digits, batch), generator=self.gen)
        images = self.prototypes[digits]
        images = images + self.noise * torch.randn(images.shape, generator=self.gen)
        known = torch.rand(n_digits * batch, generator=self.gen) < labelled
        labels = torch.where(known, digits.reshape(-1), torch.tensor(-1)).to(torch.int32)
        return images.to(device), digits.sum(0).to(torch.int32).to(device), labels.to(device), digits.to(device)


def main(steps: int = 41, blocks: int = 0, max_norm: Optional[float] = None):
    model, data = SumRecogniser(blocks=blocks, max_norm=max_norm), SyntheticDigits()
    for t in range(steps):
        images, sums, labels, digits = data.draw(model.n, model.batch, 0.1, "cuda")
        model.step(model.patches(images), sums, labels)
        if t % 10 == 0 or t == steps - 1:
            program, labelled = model.losses()
            right = float((model.p.argmax(2) == digits).float().mean())
            print("step %3d  -log p[sum] %.4f  labelled digits %.4f  digits recognised %.3f" % (t, program, labelled, right), flush=True)


if __name__ == "__main__":
    options = argparse.ArgumentParser(description="Train a recogniser of synthetic digits under a Sum-N program.")
    options.add_argument("--blocks", type=int, default=0, help="residual blocks")
    options.add_argument("--max-norm", type=float, default=None, help="of all gradients together")
    chosen = options.parse_args()
    main(blocks=chosen.blocks, max_norm=chosen.max_norm)
