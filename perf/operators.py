"""The work of training the network whose outputs become a program's Distributions, as sized cases: the loss over its classes, the
orthogonalised update of its weights, the normalised activation between its layers.

A case is a dict of plain values whose "kind" names the operator:

  cross_entropy   softmax cross entropy of x @ weight.T + bias against one class a row, the logits never kept, and the gradients of x,
                  weight and bias
  newton_schulz   five steps X <- a X + (b A + c A A) X, A = X X^T, from X = G / |G|: an update's nearest matrix with equal singular values
  group_norm      group norm over channels-last activations followed by an activation function: forward, or forward and the gradients
                  of x, gamma and beta ("train")

`run` is one pass of a case: in elementary torch operations held in 32 bits and rounded once at the end, or, where `own` is set, through
the calls of this repository.
"""
import functools
import math

import torch

own = False

DEV = "cuda"
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
STEPS = 5
NORM_EPS = 1e-7         # added to |G|
GROUP_EPS = 1e-5        # added to a group's variance


def listed():
    return [
        # the head of a digit recogniser at the mini-batch of 64: latency only
        dict(name="ce_train_digits_f32_b64", kind="cross_entropy", dtype="float32", rows=64, width=128, classes=10, bias=True),
        # a head over some thousand symbols, sizes that are nobody's round numbers
        dict(name="ce_train_f32_1000x300x5003", kind="cross_entropy", dtype="float32", rows=1000, width=300, classes=5003, bias=True),
        # the nodes of a 32 x 32 grid as classes, at the batch of 4096
        dict(name="ce_train_bf16_4096x512x1024", kind="cross_entropy", dtype="bfloat16", rows=4096, width=512, classes=1024, bias=True),
        # as many classes as a Distribution may have symbols: the largest case
        dict(name="ce_train_bf16_8192x1024x65535", kind="cross_entropy", dtype="bfloat16", rows=8192, width=1024, classes=65535, bias=False),
        # the update of the digit recogniser's head: latency only
        dict(name="ns_f32_10x128", kind="newton_schulz", dtype="float32", batch=1, rows=10, cols=128),
        # a recogniser's middle layer, taller than wide, odd
        dict(name="ns_f32_1000x777", kind="newton_schulz", dtype="float32", batch=1, rows=1000, cols=777),
        # equal layers of a deep network, orthogonalised together
        dict(name="ns_bf16_8x512x1024", kind="newton_schulz", dtype="bfloat16", batch=8, rows=512, cols=1024),
        # a wide network's square layer
        dict(name="ns_bf16_4096x4096", kind="newton_schulz", dtype="bfloat16", batch=1, rows=4096, cols=4096),
        # first layer of the digit recogniser, 28 x 28 pixels, mini-batch of 64
        dict(name="gn_train_f32_64x784x32", kind="group_norm", dtype="float32", batch=64, points=784, channels=32, groups=8, act="silu", train=True),
        # a middle layer of a deep image network
        dict(name="gn_train_bf16_128x1024x256", kind="group_norm", dtype="bfloat16", batch=128, points=1024, channels=256, groups=32, act="silu", train=True),
        # odd images, groups of six channels, the other activation function
        dict(name="gn_train_bf16_100x399x84", kind="group_norm", dtype="bfloat16", batch=100, points=399, channels=84, groups=14, act="gelu", train=True),
        # inference over large images: few groups, each of many points
        dict(name="gn_eval_bf16_16x65536x128", kind="group_norm", dtype="bfloat16", batch=16, points=65536, channels=128, groups=32, act="silu", train=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["cross_entropy", "newton_schulz", "group_norm"])
    dtype = rng.choice(["float32", "bfloat16"])
    if kind == "cross_entropy":
        return dict(kind=kind, dtype=dtype, rows=_log_int(rng, 1, 8192), width=_log_int(rng, 16, 1024), classes=_log_int(rng, 2, 65535),
                    bias=rng.random() < 0.5)
    if kind == "newton_schulz":
        rows, cols = _log_int(rng, 8, 4096), _log_int(rng, 8, 4096)
        return dict(kind=kind, dtype=dtype, batch=_log_int(rng, 1, max(1, min(16, (1 << 22) // (rows * cols)))), rows=rows, cols=cols)
    groups, each = rng.choice([1, 2, 4, 8, 14, 32]), _log_int(rng, 1, 24)
    points = _log_int(rng, 4, 256) * _log_int(rng, 4, 256)
    return dict(kind=kind, dtype=dtype, batch=_log_int(rng, 1, max(1, min(512, (1 << 26) // (groups * each * points)))), points=points,
                channels=groups * each, groups=groups, act=rng.choice(["silu", "gelu", "none"]), train=rng.random() < 0.7)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    dtype = TYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=DEV)

    def uniform(lo, hi, *shape):
        return torch.rand(shape, generator=gen, device=DEV) * (hi - lo) + lo

    def empty(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device=DEV)

    s = dict(case)
    if case["kind"] == "cross_entropy":
        n, d, v = case["rows"], case["width"], case["classes"]
        target = torch.randint(0, v, (n,), generator=gen, device=DEV, dtype=torch.int32)
        s["x"] = normal(n, d).to(dtype)
        s["weight"] = (normal(v, d) * (2.0 / math.sqrt(d))).to(dtype)
        s["bias_v"] = normal(v) * 0.5 if case["bias"] else None
        s["target"] = torch.where(uniform(0, 1, n) < 0.05, -1, target)          # rows without a label are left out
        s["grad_loss"] = uniform(0.5, 1.5, n) / n                               # samples weighed in a mean
        s["loss"], s["lse"] = empty(n), empty(n)
        s["grad_x"], s["grad_weight"] = empty(n, d, dtype=dtype), empty(v, d, dtype=dtype)
        s["grad_bias"] = empty(v) if case["bias"] else None
    elif case["kind"] == "newton_schulz":
        b, m, n = case["batch"], case["rows"], case["cols"]
        k = max(1, min(m, n) // 4)
        g = normal(b, m, k) @ normal(b, k, n) / math.sqrt(k) + normal(b, m, n)  # some directions stronger than others, as in a gradient
        s["g"] = (g * 1e-3).to(dtype)
        s["out"] = empty(b, m, n, dtype=dtype)
    else:
        b, p, c, g = case["batch"], case["points"], case["channels"], case["groups"]
        s["x"] = (normal(b, p, c) * uniform(0.5, 2, c) + normal(c) * 0.5).to(dtype)
        s["gamma"], s["beta"] = uniform(0.5, 1.5, c), normal(c) * 0.2
        s["y"], s["mean"], s["rstd"] = empty(b, p, c, dtype=dtype), empty(b, g), empty(b, g)
        if case["train"]:
            s["grad_y"] = normal(b, p, c).to(dtype)
            s["grad_x"], s["grad_gamma"], s["grad_beta"] = empty(b, p, c, dtype=dtype), empty(c), empty(c)
    return s


# ---- the plain forms

def _plain_cross_entropy(s):
    x, w, t = s["x"].float(), s["weight"].float(), s["target"].long()
    logits = x @ w.t()
    if s["bias"]:
        logits = logits + s["bias_v"]
    kept = (t >= 0) & (t < s["classes"])
    at = t.clamp(0, s["classes"] - 1).unsqueeze(1)
    top = logits.max(dim=1, keepdim=True).values
    lse = top + torch.log(torch.exp(logits - top).sum(dim=1, keepdim=True))
    loss = torch.where(kept, (lse - logits.gather(1, at)).squeeze(1), 0.0)
    out = {"loss": loss, "lse": lse.squeeze(1)}
    grad = torch.exp(logits - lse)
    grad.scatter_add_(1, at, torch.full_like(lse, -1.0))
    grad = torch.where(kept.unsqueeze(1), grad * s["grad_loss"].unsqueeze(1), 0.0)
    out["grad_x"] = (grad @ w).to(s["x"].dtype)
    out["grad_weight"] = (grad.t() @ torch.where(kept.unsqueeze(1), x, 0.0)).to(s["x"].dtype)
    if s["bias"]:
        out["grad_bias"] = grad.sum(dim=0)
    return out


def _plain_step(x, _):
    a, b, c = COEFFICIENTS
    gram = x @ x.transpose(1, 2).contiguous()
    return a * x + (b * gram + c * (gram @ gram)) @ x


def _plain_newton_schulz(s):
    g = s["g"].float()
    tall = g.shape[1] > g.shape[2]
    x = g.transpose(1, 2).contiguous() if tall else g
    x = x / (torch.sqrt((x * x).sum(dim=(1, 2), keepdim=True)) + NORM_EPS)
    x = functools.reduce(_plain_step, range(STEPS), x)
    return {"out": (x.transpose(1, 2).contiguous() if tall else x).to(s["g"].dtype)}


def _act(z, act):
    """The activation function and its derivative at z."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "silu":
        sig = 1.0 / (1.0 + torch.exp(-z))
        return z * sig, sig * (1.0 + z * (1.0 - sig))
    cdf = 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z * cdf, cdf + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain_group_norm(s):
    b, p, c, g = s["batch"], s["points"], s["channels"], s["groups"]
    x = s["x"].float().view(b, p, g, c // g)
    gamma, beta = s["gamma"].view(g, c // g), s["beta"].view(g, c // g)
    mean = x.mean(dim=(1, 3), keepdim=True)
    dev = x - mean
    rstd = 1.0 / torch.sqrt((dev * dev).mean(dim=(1, 3), keepdim=True) + GROUP_EPS)
    xhat = dev * rstd
    y, slope = _act(xhat * gamma + beta, s["act"])
    out = {"y": y.reshape(b, p, c).to(s["x"].dtype), "mean": mean.view(b, g), "rstd": rstd.view(b, g)}
    if s["train"]:
        dz = s["grad_y"].float().view(b, p, g, c // g) * slope
        out["grad_gamma"], out["grad_beta"] = (dz * xhat).sum(dim=(0, 1)).view(c), dz.sum(dim=(0, 1)).view(c)
        dh = dz * gamma
        dx = rstd * (dh - dh.mean(dim=(1, 3), keepdim=True) - xhat * (dh * xhat).mean(dim=(1, 3), keepdim=True))
        out["grad_x"] = dx.reshape(b, p, c).to(s["x"].dtype)
    return out


# ---- this repository's calls

def _own_cross_entropy(s):
    from paper_2410_03348_amd import binding as dol
    dol.cross_entropy(s["x"], s["weight"], s["target"], s["loss"], s["lse"], bias=s["bias_v"])
    dol.cross_entropy_backward(s["x"], s["weight"], s["target"], s["lse"], s["grad_loss"], s["grad_x"], s["grad_weight"],
                               bias=s["bias_v"], grad_bias=s["grad_bias"])
    out = {"loss": s["loss"], "lse": s["lse"], "grad_x": s["grad_x"], "grad_weight": s["grad_weight"]}
    if s["bias"]:
        out["grad_bias"] = s["grad_bias"]
    return out


def _own_newton_schulz(s):
    from paper_2410_03348_amd import binding as dol
    dol.newton_schulz(s["g"], s["out"], steps=STEPS, coefficients=COEFFICIENTS, eps=NORM_EPS)
    return {"out": s["out"]}


def _own_group_norm(s):
    from paper_2410_03348_amd import binding as dol
    dol.group_norm(s["x"], s["gamma"], s["beta"], s["groups"], s["y"], s["mean"], s["rstd"], eps=GROUP_EPS, act=s["act"])
    out = {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    if s["train"]:
        dol.group_norm_backward(s["x"], s["gamma"], s["beta"], s["groups"], s["mean"], s["rstd"], s["grad_y"], s["grad_x"],
                                s["grad_gamma"], s["grad_beta"], act=s["act"])
        out["grad_gamma"], out["grad_beta"], out["grad_x"] = s["grad_gamma"], s["grad_beta"], s["grad_x"]
    return out


_PLAIN = {"cross_entropy": _plain_cross_entropy, "newton_schulz": _plain_newton_schulz, "group_norm": _plain_group_norm}
_OWN = {"cross_entropy": _own_cross_entropy, "newton_schulz": _own_newton_schulz, "group_norm": _own_group_norm}


def run(state):
    return (_OWN if own else _PLAIN)[state["kind"]](state)


def work(case):
    """Inputs read once and outputs written once.  Cross entropy: one product forward, two backward (the second pass over the logits that
    not keeping them costs is left out).  Newton-Schulz: both products of a step that are symmetric counted at half."""
    e = 4 if case["dtype"] == "float32" else 2
    if case["kind"] == "cross_entropy":
        n, d, v = case["rows"], case["width"], case["classes"]
        size = (n * d + v * d) * e + 4 * v * case["bias"]
        return {"bytes": 2 * size + 16 * n, "flops": 6 * n * d * v}
    if case["kind"] == "newton_schulz":
        m, n = sorted((case["rows"], case["cols"]))
        return {"bytes": 2 * case["batch"] * m * n * e, "flops": STEPS * case["batch"] * (3 * m * m * n + m ** 3)}
    n = case["batch"] * case["points"] * case["channels"]
    small = 8 * case["batch"] * case["groups"] + 8 * case["channels"] * (2 if case["train"] else 1)
    return {"bytes": n * e * (4 if case["train"] else 2) + small, "flops": n * (30 if case["train"] else 12)}


# ---- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "cross_entropy":
        x, w, t = s["x"].double(), s["weight"].double(), s["target"].long()
        logits = torch.mm(x, w.t().contiguous())
        if case["bias"]:
            logits += s["bias_v"].double()
        lse = torch.logsumexp(logits, dim=1)
        rows = torch.nonzero((t >= 0) & (t < case["classes"])).squeeze(1)
        loss = torch.zeros_like(lse)
        loss[rows] = lse[rows] - logits[rows, t[rows]]
        grad = torch.softmax(logits[rows], dim=1)
        grad[torch.arange(rows.numel(), device=DEV), t[rows]] -= 1.0
        grad *= s["grad_loss"].double()[rows, None]
        out = {"loss": loss, "lse": lse, "grad_x": torch.zeros_like(x).index_copy_(0, rows, torch.mm(grad, w)),
               "grad_weight": torch.mm(grad.t().contiguous(), x[rows])}
        if case["bias"]:
            out["grad_bias"] = grad.sum(dim=0)
        return out
    if case["kind"] == "newton_schulz":
        a, b, c = COEFFICIENTS
        x = s["g"].double()
        tall = case["rows"] > case["cols"]
        x = x / (torch.linalg.vector_norm(x, dim=(1, 2), keepdim=True) + NORM_EPS)
        xt = x.transpose(1, 2).contiguous()
        x, xt = (xt, x) if tall else (x, xt)                    # x wide, xt its transpose
        for _ in range(STEPS):
            gram = torch.bmm(x, xt)
            eye = torch.eye(gram.shape[1], dtype=gram.dtype, device=DEV)
            poly = a * eye + torch.bmm(gram, b * eye + c * gram)
            x = torch.bmm(poly, x)
            xt = x.transpose(1, 2).contiguous()
        return {"out": xt if tall else x}
    b, p, c, g = case["batch"], case["points"], case["channels"], case["groups"]
    x = s["x"].double().view(b, p, g, -1).permute(0, 2, 1, 3).reshape(b, g, -1)                # a group to a row
    var, mean = torch.var_mean(x, dim=2, unbiased=False)
    rstd = (var + GROUP_EPS) ** -0.5

    def rows(v):
        return v.double().view(1, g, 1, -1).expand(b, g, p, -1).reshape(b, g, -1)

    def back(v):
        return v.view(b, g, p, -1).permute(0, 2, 1, 3).reshape(b, p, c)

    gamma = rows(s["gamma"])
    xhat = (x - mean[:, :, None]) * rstd[:, :, None]
    z = gamma * xhat + rows(s["beta"])
    if case["act"] == "silu":
        y, slope = z * torch.sigmoid(z), torch.sigmoid(z) * (1 + z * torch.sigmoid(-z))
    elif case["act"] == "gelu":
        cdf = torch.special.ndtr(z)
        y, slope = z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    else:
        y, slope = z, torch.ones_like(z)
    out = {"y": back(y), "mean": mean, "rstd": rstd}
    if case["train"]:
        dz = s["grad_y"].double().view(b, p, g, -1).permute(0, 2, 1, 3).reshape(b, g, -1) * slope
        out["grad_gamma"], out["grad_beta"] = back(dz * xhat).sum(dim=(0, 1)), back(dz).sum(dim=(0, 1))
        dh = dz * gamma
        out["grad_x"] = back(rstd[:, :, None] * (dh - dh.mean(dim=2, keepdim=True) - xhat * (dh * xhat).mean(dim=2, keepdim=True)))
    return out
