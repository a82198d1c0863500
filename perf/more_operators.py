"""The work between the layers of a network whose outputs become a program's Distributions and between its gradients and their update, as sized
cases beside those of operators.py.

A case is a dict of plain values whose "kind" names the operator:

  linear          z = x @ weight.T + bias, y = act(z) + residual: forward, or forward and the gradients of x, weight and bias ("train")
  residual_norm   where one block of a network ends and the next begins: h = x + scale * gate * norm(u), y = norm(h), norm(v) = gamma * v /
                  sqrt(mean(v^2) + eps): forward, or forward and all gradients ("train")
  clip            the norm over all gradients of a network together, and the gradients times min(1, max_norm / (norm + eps))

`run` is one pass of a case: in elementary torch operations held in 32 bits and rounded once at the end, or, where `own` is set, through
the calls of this repository.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16}
NORM_EPS = 1e-6         # added to a row's mean square
CLIP_EPS = 1e-6         # added to the gradients' norm


def listed():
    return [
        # one sample answered through a wide layer: every weight is read for it, latency and bytes
        dict(name="lin_eval_bf16_1x4096x16384", kind="linear", dtype="bfloat16", rows=1, width=4096, out=16384, act="silu", residual=False, train=False),
        # the digit recogniser's features into a hidden layer at the mini-batch of 64: latency only
        dict(name="lin_train_f32_64x1568x128", kind="linear", dtype="float32", rows=64, width=1568, out=128, act="silu", residual=False, train=True),
        # odd sizes in float, a layer whose input stream is added behind it
        dict(name="lin_train_f32_1000x777x1501", kind="linear", dtype="float32", rows=1000, width=777, out=1501, act="gelu", residual=True, train=True),
        # the widening layer of a block
        dict(name="lin_train_bf16_4096x1024x4096", kind="linear", dtype="bfloat16", rows=4096, width=1024, out=4096, act="gelu", residual=False, train=True),
        # a wide network's square layer with its stream added: the largest case
        dict(name="lin_train_bf16_8192x4096x4096", kind="linear", dtype="bfloat16", rows=8192, width=4096, out=4096, act="none", residual=True, train=True),
        # one sample between two blocks of a wide network: latency only
        dict(name="rn_eval_bf16_1x4096", kind="residual_norm", dtype="bfloat16", samples=1, points=1, cols=4096, post=True, gate="one", train=False),
        # the recogniser's 49 patches of 64 digits at 32 channels, one gate for all
        dict(name="rn_train_f32_64x49x32", kind="residual_norm", dtype="float32", samples=64, points=49, cols=32, post=True, gate="one", train=True),
        # a wide network's mini-batch, a gate for each sample
        dict(name="rn_train_bf16_8x1024x4096", kind="residual_norm", dtype="bfloat16", samples=8, points=1024, cols=4096, post=True, gate="sample", train=True),
        # odd sizes, a gate for every point, no norm behind the block
        dict(name="rn_train_bf16_37x131x1111", kind="residual_norm", dtype="bfloat16", samples=37, points=131, cols=1111, post=False, gate="point", train=True),
        # the gradients of a network lie behind each other in a buffer for each type, as the exchange between GPUs wants them
        # the digit recogniser's: latency only
        dict(name="clip_digits", kind="clip", shapes="32x16,32,32,10x1568,10", floats="all", repeat=1, factor=0.6),
        # many layers of odd sizes, matrices in bf16 beside vectors in float
        dict(name="clip_40_odd_layers", kind="clip", shapes="777x1000,1000,1000x333,333,1501", floats="vectors", repeat=40, factor=0.3),
        # a large network: twelve blocks of two wide matrices, some 0.8 GB
        dict(name="clip_12_wide_blocks", kind="clip", shapes="4096x4096,4096,4096x4096,4096", floats="vectors", repeat=12, factor=0.7),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["linear", "residual_norm", "clip"])
    if kind == "linear":
        dtype, train = rng.choice(["float32", "bfloat16"]), rng.random() < 0.6
        width, out = _log_int(rng, 16, 4096), _log_int(rng, 10, 16384)
        most = (1 << 37 if dtype == "bfloat16" else 1 << 34) // (width * out)       # of 8192 x 4096 x 4096, float an eighth of it
        return dict(kind=kind, dtype=dtype, rows=_log_int(rng, 1, max(1, min(8192, most))), width=width, out=out,
                    act=rng.choice(["none", "silu", "gelu"]), residual=rng.random() < 0.5, train=train)
    if kind == "residual_norm":
        cols = _log_int(rng, 8, 8192)
        points = _log_int(rng, 1, max(1, min(2048, (1 << 25) // cols)))
        samples = _log_int(rng, 1, max(1, min(1024, (1 << 25) // (cols * points))))
        return dict(kind=kind, dtype=rng.choice(["float32", "bfloat16"]), samples=samples, points=points, cols=cols, post=rng.random() < 0.6,
                    gate=rng.choice(["none", "one", "sample", "point"]), train=rng.random() < 0.7)
    rows, cols, layers = _log_int(rng, 1, 4096), _log_int(rng, 1, 4096), _log_int(rng, 1, 64)
    repeat = max(1, min(layers, (1 << 26) // (rows * cols)))
    return dict(kind=kind, shapes="%dx%d,%d,%dx%d,%d" % (rows, cols, cols, cols, _log_int(rng, 1, rows), rows),
                floats=rng.choice(["all", "vectors", "none"]), repeat=repeat, factor=rng.choice([0.1, 0.3, 0.9, 2.0]))


def _shapes(case):
    """[(sizes, dtype)] of a clip case's gradients."""
    one = [tuple(int(n) for n in s.split("x")) for s in case["shapes"].split(",")]
    floats = case["floats"]
    return [(s, torch.float32 if floats == "all" or (floats == "vectors" and len(s) == 1) else torch.bfloat16) for s in one] * case["repeat"]


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=DEV)

    def uniform(lo, hi, *shape):
        return torch.rand(shape, generator=gen, device=DEV) * (hi - lo) + lo

    def empty(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device=DEV)

    s = dict(case)
    if case["kind"] == "linear":
        dtype = TYPES[case["dtype"]]
        n, d, m = case["rows"], case["width"], case["out"]
        s["x"], s["weight"] = normal(n, d).to(dtype), (normal(m, d) * (1.0 / math.sqrt(d))).to(dtype)
        s["bias"] = normal(m) * 0.2
        s["stream"] = normal(n, m).to(dtype) if case["residual"] else None
        s["y"] = empty(n, m, dtype=dtype)
        if case["train"]:
            s["z"] = empty(n, m, dtype=dtype) if case["act"] != "none" else None
            s["grad_y"] = normal(n, m).to(dtype)
            s["grad_x"], s["grad_weight"], s["grad_bias"] = empty(n, d, dtype=dtype), empty(m, d, dtype=dtype), empty(m)
    elif case["kind"] == "residual_norm":
        dtype = TYPES[case["dtype"]]
        n, c = case["samples"] * case["points"], case["cols"]
        gates = {"none": 0, "one": 1, "sample": case["samples"], "point": n}[case["gate"]]
        s["scale"] = 0.5
        # rows of different lengths, as a stream has them
        s["x"], s["u"] = (normal(n, c) * uniform(0.5, 2, n, 1)).to(dtype), (normal(n, c) * uniform(0.5, 2, n, 1)).to(dtype)
        s["gamma_u"] = uniform(0.5, 1.5, c) if case["post"] else None
        s["gates"] = (uniform(0, 1, gates, c)).to(dtype) if gates else None
        s["gamma_y"] = uniform(0.5, 1.5, c)
        s["h"], s["y"] = empty(n, c, dtype=dtype), empty(n, c, dtype=dtype)
        s["rstd_u"], s["rstd_h"] = empty(n) if case["post"] else None, empty(n)
        if case["train"]:
            s["grad_h"], s["grad_y"] = normal(n, c).to(dtype), normal(n, c).to(dtype)
            s["grad_x"], s["grad_u"] = empty(n, c, dtype=dtype), empty(n, c, dtype=dtype)
            s["grad_gamma_u"] = empty(c) if case["post"] else None
            s["grad_gates"] = empty(gates, c, dtype=dtype) if gates else None
            s["grad_gamma_y"] = empty(c)
    else:
        # layers' gradients differ in size; the norm that is allowed is some factor of what theirs will be
        shapes, total = _shapes(case), 0.0
        s["grads"], s["clipped"], s["flat"] = [None] * len(shapes), [None] * len(shapes), {}
        for name, dtype in TYPES.items():
            mine = [k for k, (_, t) in enumerate(shapes) if t == dtype]
            flat = [torch.empty(sum(math.prod(shapes[k][0]) for k in mine), dtype=dtype, device=DEV) for _ in range(2)]
            if mine:
                s["flat"][name] = flat[1]
            at = 0
            for k in mine:
                n = math.prod(shapes[k][0])
                s["grads"][k], s["clipped"][k] = (f[at:at + n].view(shapes[k][0]) for f in flat)
                size = 1e-3 * (1 + k % 5)
                s["grads"][k].copy_(normal(*shapes[k][0]) * size)
                total += size * size * n
                at += n
        s["max_norm"] = case["factor"] * math.sqrt(total)
        s["norm"], s["coef"] = empty(1), empty(1)
        if own:
            _plan(s)
    return s


# ---- the plain forms

def _act(z, act):
    """The activation function and its derivative at z."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return torch.where(z > 0, z, 0.0), (z > 0).float()
    if act == "silu":
        sig = 1.0 / (1.0 + torch.exp(-z))
        return z * sig, sig * (1.0 + z * (1.0 - sig))
    cdf = 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z * cdf, cdf + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain_linear(s):
    dtype, x, w = s["x"].dtype, s["x"].float(), s["weight"].float()
    z = x @ w.t() + s["bias"]
    y, slope = _act(z, s["act"])
    if s["residual"]:
        y = y + s["stream"].float()
    out = {"y": y.to(dtype)}
    if s["train"]:
        if s["act"] != "none":
            out["z"] = z.to(dtype)
        dz = s["grad_y"].float() * slope
        out["grad_x"], out["grad_weight"], out["grad_bias"] = (dz @ w).to(dtype), (dz.t() @ x).to(dtype), dz.sum(dim=0)
    return out


def _plain_residual_norm(s):
    dtype, n, c = s["x"].dtype, s["samples"] * s["points"], s["cols"]
    x, u, gamma_y = s["x"].float(), s["u"].float(), s["gamma_y"]
    out = {}
    rstd_u, uhat, v = None, None, u
    if s["post"]:
        rstd_u = 1.0 / torch.sqrt((u * u).mean(dim=1, keepdim=True) + NORM_EPS)
        uhat = u * rstd_u
        v = uhat * s["gamma_u"]
        out["rstd_u"] = rstd_u.view(n)
    each = None
    if s["gates"] is not None:
        gates = s["gates"].shape[0]
        each = s["gates"].float().unsqueeze(1).expand(gates, n // gates, c).reshape(n, c)
    h = x + s["scale"] * (v if each is None else each * v)
    rstd_h = 1.0 / torch.sqrt((h * h).mean(dim=1, keepdim=True) + NORM_EPS)
    hhat = h * rstd_h
    out.update(h=h.to(dtype), y=(hhat * gamma_y).to(dtype), rstd_h=rstd_h.view(n))
    if s["train"]:
        grad_y = s["grad_y"].float()
        a = grad_y * gamma_y
        dh = s["grad_h"].float() + rstd_h * (a - hhat * (a * hhat).mean(dim=1, keepdim=True))
        dv = s["scale"] * (dh if each is None else each * dh)
        du = dv
        if s["post"]:
            b = dv * s["gamma_u"]
            du = rstd_u * (b - uhat * (b * uhat).mean(dim=1, keepdim=True))
            out["grad_gamma_u"] = (dv * uhat).sum(dim=0)
        if each is not None:
            out["grad_gates"] = (s["scale"] * dh * v).view(gates, n // gates, c).sum(dim=1).to(dtype)
        out.update(grad_x=dh.to(dtype), grad_u=du.to(dtype), grad_gamma_y=(grad_y * hhat).sum(dim=0))
    return out


def _plain_clip(s):
    squares = torch.stack([(g.float() * g.float()).sum() for g in s["grads"]])
    norm = torch.sqrt(squares.sum())
    ratio = s["max_norm"] / (norm + CLIP_EPS)
    coef = torch.where(ratio < 1.0, ratio, torch.ones_like(ratio))
    for g, to in zip(s["grads"], s["clipped"]):
        to.copy_(g.float() * coef)
    return dict(s["flat"], norm=norm.view(1), coef=coef.view(1))


# ---- this repository's calls

def _own_linear(s):
    from paper_2410_03348_amd import binding as dol
    z = s["z"] if s["train"] else None
    dol.linear(s["x"], s["weight"], s["y"], bias=s["bias"], act=s["act"], residual=s["stream"], z=z)
    out = {"y": s["y"]}
    if s["train"]:
        if z is not None:
            out["z"] = z
        dol.linear_backward(s["x"], s["weight"], s["grad_y"], s["grad_x"], s["grad_weight"], grad_bias=s["grad_bias"], act=s["act"], z=z)
        out["grad_x"], out["grad_weight"], out["grad_bias"] = s["grad_x"], s["grad_weight"], s["grad_bias"]
    return out


def _own_residual_norm(s):
    from paper_2410_03348_amd import binding as dol
    dol.residual_norm(s["x"], s["u"], s["gamma_u"], s["gates"], s["gamma_y"], s["h"], s["y"], s["rstd_u"], s["rstd_h"], norm_u=s["post"],
                      scale=s["scale"], eps=NORM_EPS)
    keys = ["h", "y", "rstd_h"] + (["rstd_u"] if s["post"] else [])
    if s["train"]:
        dol.residual_norm_backward(s["u"], s["gamma_u"], s["gates"], s["gamma_y"], s["h"], s["rstd_u"], s["rstd_h"], s["grad_h"], s["grad_y"],
                                   s["grad_x"], s["grad_u"], s["grad_gamma_u"], s["grad_gates"], s["grad_gamma_y"], norm_u=s["post"],
                                   scale=s["scale"])
        keys += ["grad_x", "grad_u", "grad_gamma_y"] + (["grad_gamma_u"] if s["post"] else []) + (["grad_gates"] if s["gates"] is not None else [])
    return {k: s[k] for k in keys}


def _plan(s):
    """The lists of buffers that a training program makes once, beside the buffers themselves."""
    from paper_2410_03348_amd import binding as dol
    s["grad_list"], s["clipped_list"] = dol.TensorList(s["grads"]), dol.TensorList(s["clipped"])


def _own_clip(s):
    from paper_2410_03348_amd import binding as dol
    if "grad_list" not in s:
        _plan(s)
    dol.clip_grads(s["grad_list"], s["max_norm"], s["norm"], s["coef"], out=s["clipped_list"], eps=CLIP_EPS)
    return dict(s["flat"], norm=s["norm"], coef=s["coef"])


_PLAIN = {"linear": _plain_linear, "residual_norm": _plain_residual_norm, "clip": _plain_clip}
_OWN = {"linear": _own_linear, "residual_norm": _own_residual_norm, "clip": _own_clip}


# Those calls hand bf16's backward passes z and h as they were rounded, of which nothing can make a 32-bit gradient as exact as it should be: up to 2^-8
# of each number is gone.  Training in bf16 keeps what rounding z has left beside z, and x, which it has in hand, instead of h.

def _own_linear_with_rest(s):
    from paper_2410_03348_amd import binding as dol
    if not s["train"] or s["act"] == "none" or s["x"].dtype != torch.bfloat16:
        return _own_linear(s)
    if "rest" not in s:
        s["rest"] = torch.empty(s["z"].shape, dtype=torch.int16, device=DEV)
    dol.linear(s["x"], s["weight"], s["y"], bias=s["bias"], act=s["act"], residual=s["stream"], z=s["z"], z_rest=s["rest"])
    dol.linear_backward(s["x"], s["weight"], s["grad_y"], s["grad_x"], s["grad_weight"], grad_bias=s["grad_bias"], act=s["act"], z=s["z"],
                        z_rest=s["rest"])
    return {k: s[k] for k in ("y", "z", "grad_x", "grad_weight", "grad_bias")}


def _own_residual_norm_from_x(s):
    from paper_2410_03348_amd import binding as dol
    if not s["train"] or s["x"].dtype != torch.bfloat16:
        return _own_residual_norm(s)
    dol.residual_norm(s["x"], s["u"], s["gamma_u"], s["gates"], s["gamma_y"], s["h"], s["y"], s["rstd_u"], s["rstd_h"], norm_u=s["post"],
                      scale=s["scale"], eps=NORM_EPS)
    dol.residual_norm_backward(s["x"], s["u"], s["gamma_u"], s["gates"], s["gamma_y"], s["rstd_u"], s["rstd_h"], s["grad_h"], s["grad_y"],
                               s["grad_x"], s["grad_u"], s["grad_gamma_u"], s["grad_gates"], s["grad_gamma_y"], norm_u=s["post"], scale=s["scale"])
    keys = ["h", "y", "rstd_h", "grad_x", "grad_u", "grad_gamma_y"]
    keys += (["rstd_u", "grad_gamma_u"] if s["post"] else []) + (["grad_gates"] if s["gates"] is not None else [])
    return {k: s[k] for k in keys}


def _calls():
    return dict(_OWN, linear=_own_linear_with_rest, residual_norm=_own_residual_norm_from_x)


def run(state):
    return (_calls() if own else _PLAIN)[state["kind"]](state)


def work(case):
    """Inputs read once and outputs written once.  A linear layer: one product forward, two backward."""
    if case["kind"] == "clip":
        sizes = [(math.prod(s), 4 if t == torch.float32 else 2) for s, t in _shapes(case)]
        return {"bytes": 2 * sum(n * e for n, e in sizes) + 8, "flops": 3 * sum(n for n, _ in sizes)}
    e = 4 if case["dtype"] == "float32" else 2
    if case["kind"] == "linear":
        n, d, m = case["rows"], case["width"], case["out"]
        elements = n * d + m * d + n * m * (2 if case["residual"] else 1)
        if case["train"]:
            elements += n * m * (1 if case["act"] == "none" else 2) + n * d + m * d
        return {"bytes": elements * e + 4 * m * (2 if case["train"] else 1), "flops": 2 * n * d * m * (3 if case["train"] else 1)}
    n, c = case["samples"] * case["points"], case["cols"]
    gates = {"none": 0, "one": 1, "sample": case["samples"], "point": n}[case["gate"]]
    gammas, rstds = (2, 2) if case["post"] else (1, 1)
    passes = 2 if case["train"] else 1
    return {"bytes": n * c * e * (8 if case["train"] else 4) + passes * (gates * e + gammas * 4) * c + rstds * 4 * n,
            "flops": n * c * (30 if case["train"] else 10)}


# ---- the definitions in 64 bits

def _exact_act(z, act):
    return {"none": lambda v: v, "relu": lambda v: v.clamp(min=0), "silu": lambda v: v * torch.sigmoid(v),
            "gelu": lambda v: v * torch.special.ndtr(v)}[act](z)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "clip":
        norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(g.reshape(-1), dtype=torch.float64) for g in s["grads"]]))
        coef = (s["max_norm"] / (norm + CLIP_EPS)).clamp(max=1.0)
        out = {"norm": norm.view(1), "coef": coef.view(1)}
        for name in s["flat"]:
            out[name] = torch.cat([g.reshape(-1).double() * coef for g in s["grads"] if g.dtype == TYPES[name]])
        return out
    back = case["train"]
    if case["kind"] == "linear":
        x, w, b = (s[k].double().requires_grad_(back) for k in ("x", "weight", "bias"))
        z = torch.addmm(b, x, w.t())
        y = _exact_act(z, case["act"])
        if case["residual"]:
            y = y + s["stream"].double()
        out = {"y": y.detach()}
        if back:
            if case["act"] != "none":
                out["z"] = z.detach()
            out["grad_x"], out["grad_weight"], out["grad_bias"] = torch.autograd.grad(y, (x, w, b), s["grad_y"].double())
        return out
    names = ["x", "u", "gamma_y"] + (["gamma_u"] if case["post"] else []) + (["gates"] if s["gates"] is not None else [])
    t = {k: s[k].double().requires_grad_(back) for k in names}
    n = t["x"].shape[0]
    out = {}
    v = t["u"]
    if case["post"]:
        r = torch.rsqrt(v.pow(2).mean(1) + NORM_EPS)
        out["rstd_u"] = r.detach()
        v = v * (r[:, None] * t["gamma_u"])
    if s["gates"] is not None:
        v = v * t["gates"].repeat_interleave(n // t["gates"].shape[0], dim=0)
    h = torch.add(t["x"], v, alpha=s["scale"])
    r = torch.rsqrt(h.pow(2).mean(1) + NORM_EPS)
    y = h * r[:, None] * t["gamma_y"]
    out.update(h=h.detach(), y=y.detach(), rstd_h=r.detach())
    if back:
        grads = torch.autograd.grad([h, y], [t[k] for k in names], [s["grad_h"].double(), s["grad_y"].double()])
        out.update({"grad_" + k: g for k, g in zip(names, grads)})
    return out
