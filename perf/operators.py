"""The operators of a gated block's training step and of its serving, as measurable cases.

``run`` computes each of them in its plain form (elementary torch operations in 32 bits,
rounded once at the end) or, where ``own`` is true, through the package's classes:

  ff      GatedFeedForward.forward: (act(x Wg + bg) * (x Wu + bu)) Wd + bd, the weights
          loaded beforehand, as a serving program keeps them
  step    GatedFeedForward.load, forward and backward: a training step, whose weights
          are new in every step
  norm    ResidualNorm.forward: y = x + residual and the LayerNorm of y
  dnorm   ResidualNorm.backward: the gradients of both for the sum, gamma and beta
  clip    GradClip: the global norm of a list of gradients, and the list scaled to it

Points have the features of the model's input embedding; weights are Xavier-uniform with
small random biases.  ``exact`` gives the same outputs from the definitions in float64.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
LN_EPS = 1e-5


def listed():
    return [
        # serving one query point: the weights of a layer against a single row
        dict(name="ff_1_bf16", op="ff", N=1, C=256, F=1024, act="silu", dtype="bf16", bias=True),
        # a serving request of a few thousand query points at the 8-block model's width
        dict(name="ff_4k_bf16", op="ff", N=4096, C=256, F=1024, act="gelu", dtype="bf16", bias=True),
        # a surface mesh in float32; two thirds of the usual hidden width, as gated layers
        # of equal weight count have it (4C * 2/3, not a multiple of anything)
        dict(name="ff_100k_fp32", op="ff", N=100_003, C=128, F=341, act="silu", dtype="fp32", bias=False),
        # a surface mesh of a million points through the 8-block model's feed-forward
        dict(name="ff_1m_bf16", op="ff", N=1_000_000, C=256, F=1024, act="silu", dtype="bf16", bias=True),
        # training on a small ragged subset, float32
        dict(name="step_60k_fp32", op="step", N=60_001, C=128, F=512, act="silu", dtype="fp32", bias=True),
        # training at the 8-block model's width in bf16, ragged
        dict(name="step_250k_bf16", op="step", N=250_001, C=256, F=1024, act="gelu", dtype="bf16", bias=True),
        # the training subset of the benchmark
        dict(name="step_2m_fp32", op="step", N=2_000_000, C=128, F=512, act="silu", dtype="fp32", bias=True),
        # a serving request: the sum and norm of a few thousand rows
        dict(name="norm_5k_bf16", op="norm", N=5003, C=128, dtype="bf16", residual=True),
        # the gradient of the training subset's norms
        dict(name="dnorm_2m_fp32", op="dnorm", N=2_000_000, C=128, dtype="fp32", residual=True),
        # a mesh of a million points, the wide model's norm in bf16
        dict(name="dnorm_1m_bf16", op="dnorm", N=1_000_003, C=256, dtype="bf16", residual=True),
        # gradients of one block of the narrow model: some twenty tensors, the smallest call
        dict(name="clip_block_fp32", op="clip", L=1, C=128, F=512, H=8, M=64, ff="fp32", scale=0.05),
        # gradients of the 24-layer model, the feed-forward's in bf16: hundreds of tensors
        dict(name="clip_model_mixed", op="clip", L=24, C=256, F=1024, H=8, M=64, ff="bf16", scale=0.05),
    ]


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["ff", "ff", "step", "step", "norm", "dnorm", "clip"])
    dtype = rng.choice(["bf16", "fp32"])
    if op in ("ff", "step"):
        C = 16 * rng.randint(1, 16)
        F = size(24, 1600)
        # no more work, and no larger a hidden layer, than the largest listed step
        n = min(2_000_000, int(2_000_000 * 128 * 512 / (C * F)), int(1e9 / F), int(2.5e8 / C))
        return dict(op=op, N=size(1 if op == "ff" else 50, n), C=C, F=F, act=rng.choice(["silu", "gelu"]), dtype=dtype,
                    bias=rng.random() < 0.7)
    if op == "clip":
        return dict(op="clip", L=rng.randint(1, 24), C=16 * rng.randint(3, 16), F=size(100, 1024), H=rng.choice([1, 2, 4, 8]),
                    M=16 * rng.randint(1, 4), ff=dtype, scale=size(1, 1000) * 1e-4)
    C = 16 * rng.randint(1, 32)
    return dict(op=op, N=size(1, int(2.5e8 / C) if dtype == "fp32" else int(2.5e8 / C) // 2), C=C, dtype=dtype,
                residual=rng.random() < 0.7)


# ------------------------------------------------------------------ inputs

def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 64 + stream)
    return g


def _uniform(shape, bound, g):
    return (torch.rand(shape, generator=g, device="cuda") * 2.0 - 1.0) * bound


def _features(n, C, dtype, seed, stream=0):
    """Rows of the model's input embedding for n points: Fourier features of the
    coordinates under a Gaussian map, normalised per point."""
    g = _gen(seed, stream)
    R = torch.randn((96, C), generator=_gen(seed, 63), device="cuda") / math.sqrt(96.0)
    f = math.pi * 2.0 ** (torch.arange(16, device="cuda") / 3.0)
    x = torch.empty((n, C), device="cuda", dtype=dtype)
    for a in range(0, n, 1 << 20):
        b = min(n, a + (1 << 20))
        q = torch.rand((b - a, 3), generator=g, device="cuda") * 2.0 - 1.0
        arg = q[:, :, None] * f
        z = torch.cat([arg.sin(), arg.cos()], dim=2).reshape(b - a, 96) @ R
        z = z - z.mean(1, keepdim=True)
        x[a:b] = (z / (z.square().mean(1, keepdim=True) + LN_EPS).sqrt()).to(dtype)
    return x


def _noise(n, C, dtype, seed, stream):
    return torch.randn((n, C), generator=_gen(seed, stream), device="cuda").to(dtype)


def _ff_weights(case, seed):
    C, F, dtype = case["C"], case["F"], DTYPES[case["dtype"]]
    g = _gen(seed, 8)
    bound = math.sqrt(6.0 / (C + F))
    w = dict(Wg=_uniform((C, F), bound, g), Wu=_uniform((C, F), bound, g), Wd=_uniform((F, C), bound, g))
    if case["bias"]:
        w.update(bg=_uniform((F,), 0.1, g), bu=_uniform((F,), 0.1, g), bd=_uniform((C,), 0.1, g))
    return {k: v.to(dtype) for k, v in w.items()}


def _gradient_shapes(case):
    """(shape, dtype) of every gradient of L blocks: Physics-Attention, two norms and
    the gated feed-forward, which may be held in bf16."""
    C, F, H, M = case["C"], case["F"], case["H"], case["M"]
    dh = max(1, C // H)
    attention = [(C, H * M), (H * M,), (C, C), (C,), (H, dh, dh), (H, dh, dh), (H, dh, dh), (C, C), (C,)]
    ff = [(C, F), (F,), (C, F), (F,), (F, C), (C,)]
    block = [(s, torch.float32) for s in attention + [(C,)] * 4] + [(s, DTYPES[case["ff"]]) for s in ff]
    return block * case["L"]


def prepare(case, seed):
    s = {"case": case}
    op = case["op"]
    if op == "clip":
        g = _gen(seed, 1)
        rng = random.Random(seed)
        shapes = _gradient_shapes(case)
        # The program keeps the gradients of a type in one buffer, each a view of it;
        # those of a real step differ in size from tensor to tensor.
        s["flat"], s["flat_out"] = [], []
        views, views_out = {}, {}
        for dt in dict.fromkeys(dt for _, dt in shapes):
            mine = [(i, shape) for i, (shape, d) in enumerate(shapes) if d == dt]
            buf = torch.randn(sum(math.prod(shape) for _, shape in mine), generator=g, device="cuda")
            out, at = torch.empty_like(buf, dtype=dt), 0
            for i, shape in mine:
                buf[at:at + math.prod(shape)] *= case["scale"] * 10.0 ** rng.uniform(-2, 0)
                at += math.prod(shape)
            buf, at = buf.to(dt), 0
            for i, shape in mine:
                n = math.prod(shape)
                views[i], views_out[i] = buf[at:at + n].view(shape), out[at:at + n].view(shape)
                at += n
            s["flat"].append(buf)
            s["flat_out"].append(out)
        s["grads"], s["out"] = ([v[i] for i in range(len(shapes))] for v in (views, views_out))
        if own:
            from paper_2602_04940_amd import GradClip
            s["clip"] = GradClip()
        return s
    N, C, dtype = case["N"], case["C"], DTYPES[case["dtype"]]
    s["x"] = _features(N, C, dtype, seed)
    if op in ("ff", "step"):
        s["w"] = _ff_weights(case, seed)
        if op == "step":
            s["g"] = _noise(N, C, dtype, seed, 2)
        if own:
            from paper_2602_04940_amd import GatedFeedForward, GatedWeights
            s["w"] = GatedWeights(s["w"], case["dtype"])
            s["ff"] = GatedFeedForward(C, case["F"], activation=case["act"], dtype=case["dtype"])
            if op == "ff":
                s["ff"].load(s["w"])
        return s
    g = _gen(seed, 8)
    s["gamma"] = 1.0 + _uniform((C,), 0.1, g)
    s["beta"] = _uniform((C,), 0.1, g)
    if op == "norm":
        s["r"] = _noise(N, C, dtype, seed, 2) if case["residual"] else None
    else:
        s["g"] = _noise(N, C, dtype, seed, 2)
        s["r"] = _noise(N, C, dtype, seed, 3) if case["residual"] else None
    if own:
        from paper_2602_04940_amd import ResidualNorm
        s["norm"] = ResidualNorm(C, dtype=case["dtype"], eps=LN_EPS)
    return s


# ------------------------------------------------------------------ the call

def run(state):
    op = state["case"]["op"]
    if not own:
        return {"ff": _plain_ff, "step": _plain_step, "norm": _plain_norm, "dnorm": _plain_dnorm,
                "clip": _plain_clip}[op](state)
    if op == "ff":
        return state["ff"].forward(state["x"])
    if op == "step":
        ff = state["ff"]
        ff.load(state["w"])
        out = ff.forward(state["x"])
        dx, grads = ff.backward(state["x"], state["g"])
        res = {"out": out, "dx": dx, "dWg": grads["dWg"], "dWu": grads["dWu"], "dWd": grads["dWd"]}
        if state["case"]["bias"]:
            res.update(dbg=grads["dbg"], dbu=grads["dbu"], dbd=grads["dbd"])
        return res
    if op == "norm":
        y, n = state["norm"].forward(state["x"], state["gamma"], state["beta"], residual=state["r"])
        return {"y": y, "n": n}
    if op == "dnorm":
        dx, dgamma, dbeta = state["norm"].backward(state["x"], state["g"], state["gamma"], residual_grad=state["r"])
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    norm = state["clip"](state["grads"], 1.0, out=state["out"])
    return [norm] + state["flat_out"]


# ------------------------------------------------------------------ plain forms

def _act(a, kind):
    """The activation and its derivative."""
    if kind == "silu":
        s = 1.0 / (1.0 + torch.exp(-a))
        return a * s, s * (1.0 + a * (1.0 - s))
    phi = 0.5 * (1.0 + torch.erf(a * math.sqrt(0.5)))
    return a * phi, phi + a * torch.exp(-0.5 * a * a) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain_hidden(state):
    w = {k: v.float() for k, v in state["w"].items()}
    x = state["x"].float()
    a, u = x @ w["Wg"], x @ w["Wu"]
    if "bg" in w:
        a, u = a + w["bg"], u + w["bu"]
    return w, x, a, u


def _plain_ff(state):
    w, x, a, u = _plain_hidden(state)
    out = (_act(a, state["case"]["act"])[0] * u) @ w["Wd"]
    if "bd" in w:
        out = out + w["bd"]
    return out.to(state["x"].dtype)


def _plain_step(state):
    dtype = state["x"].dtype
    w, x, a, u = _plain_hidden(state)
    g = state["g"].float()
    act, slope = _act(a, state["case"]["act"])
    h = act * u
    out = h @ w["Wd"]
    dh = g @ w["Wd"].T
    du = dh * act
    da = dh * u * slope
    res = {"out": out if "bd" not in w else out + w["bd"], "dx": da @ w["Wg"].T + du @ w["Wu"].T, "dWg": x.T @ da,
           "dWu": x.T @ du, "dWd": h.T @ g}
    if "bd" in w:
        res.update(dbg=da.sum(0), dbu=du.sum(0), dbd=g.sum(0))
    return {k: v.to(dtype) for k, v in res.items()}


def _plain_stats(y):
    c = y - y.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt((c * c).mean(1, keepdim=True) + LN_EPS)
    return c * rstd, rstd


def _plain_norm(state):
    dtype = state["x"].dtype
    y = state["x"].float()
    if state["r"] is not None:
        y = y + state["r"].float()
    h, _ = _plain_stats(y)
    return {"y": y.to(dtype), "n": (h * state["gamma"] + state["beta"]).to(dtype)}


def _plain_dnorm(state):
    h, rstd = _plain_stats(state["x"].float())
    g = state["g"].float()
    dh = g * state["gamma"]
    dx = rstd * (dh - dh.mean(1, keepdim=True) - h * (dh * h).mean(1, keepdim=True))
    if state["r"] is not None:
        dx = dx + state["r"].float()
    return {"dx": dx.to(state["x"].dtype), "dgamma": (g * h).sum(0), "dbeta": g.sum(0)}


def _plain_clip(state):
    norm = torch.stack([t.float().square().sum() for t in state["grads"]]).sum().sqrt()
    scale = torch.where(norm > 1.0, 1.0 / norm, torch.ones_like(norm))
    for t, out in zip(state["grads"], state["out"]):
        out.copy_(t.float() * scale)
    return [norm] + state["flat_out"]


# ------------------------------------------------------------------ what it takes

def work(case):
    """Bytes: inputs once, outputs once.  Flops: the products of the definition, without
    what is computed again."""
    op = case["op"]
    if op == "clip":
        count = [(math.prod(s), 2 if dt == torch.bfloat16 else 4) for s, dt in _gradient_shapes(case)]
        return {"bytes": float(sum(2 * n * e for n, e in count)), "flops": float(sum(3 * n for n, _ in count))}
    N, C, e = case["N"], case["C"], 2 if case["dtype"] == "bf16" else 4
    if op in ("norm", "dnorm"):
        # x, residual, y, out; without the residual y is x.  y, g, dx and the residual's gradient.
        rows = 4 if case["residual"] else 2 if op == "norm" else 3
        return {"bytes": float(rows * N * C * e + 4 * C * (2 if op == "norm" else 3)), "flops": 10.0 * N * C}
    F = case["F"]
    weights = 3 * C * F + (2 * F + C if case["bias"] else 0)
    if op == "ff":
        return {"bytes": float(e * (2 * N * C + weights)), "flops": 6.0 * N * C * F}
    return {"bytes": float(e * (4 * N * C + 2 * weights)), "flops": 18.0 * N * C * F}


# ------------------------------------------------------------------ float64

STEP = 1 << 16


def exact(case, seed):
    """The outputs from the definitions in float64, the gradients by differentiation."""
    st = {**_plain_inputs(case, seed)}
    op = case["op"]
    if op == "clip":
        g = [t.double() for t in st["flat"]]
        norm = torch.linalg.vector_norm(torch.cat(g))
        return [norm] + [t / norm.clamp(min=1.0) for t in g]
    if op in ("norm", "dnorm"):
        gamma, beta = st["gamma"].double().requires_grad_(), st["beta"].double().requires_grad_()
        res = {"dx": [], "y": [], "n": []}
        for a in range(0, case["N"], STEP):
            y = st["x"][a:a + STEP].double()
            r = st["r"][a:a + STEP].double() if st["r"] is not None else 0.0
            if op == "norm":
                y = y + r
                with torch.no_grad():
                    res["n"].append(torch.nn.functional.layer_norm(y, (case["C"],), gamma, beta, LN_EPS))
                res["y"].append(y)
                continue
            y.requires_grad_()
            n = torch.nn.functional.layer_norm(y, (case["C"],), gamma, beta, LN_EPS)
            n.backward(st["g"][a:a + STEP].double())
            res["dx"].append(y.grad + r)
        if op == "norm":
            return {"y": torch.cat(res["y"]), "n": torch.cat(res["n"])}
        return {"dx": torch.cat(res["dx"]), "dgamma": gamma.grad, "dbeta": beta.grad}
    w = {k: v.double().requires_grad_(op == "step") for k, v in st["w"].items()}
    act = torch.nn.functional.silu if case["act"] == "silu" else torch.nn.functional.gelu
    out, dx = [], []
    for a in range(0, case["N"], STEP):
        x = st["x"][a:a + STEP].double().requires_grad_(op == "step")
        h = act(torch.addmm(w["bg"], x, w["Wg"]) if "bg" in w else x @ w["Wg"]) * (
            torch.addmm(w["bu"], x, w["Wu"]) if "bu" in w else x @ w["Wu"])
        o = torch.addmm(w["bd"], h, w["Wd"]) if "bd" in w else h @ w["Wd"]
        out.append(o.detach())
        if op == "step":
            o.backward(st["g"][a:a + STEP].double())
            dx.append(x.grad)
    if op == "ff":
        return torch.cat(out)
    res = {"out": torch.cat(out), "dx": torch.cat(dx)}
    res.update({"d" + k: w[k].grad for k in ("Wg", "Wu", "Wd", "bg", "bu", "bd") if k in w})
    return res


def _plain_inputs(case, seed):
    """The inputs of a case without the package's objects."""
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was
