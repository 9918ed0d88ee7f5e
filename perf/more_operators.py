"""The operators of a conditioned block, as measurable cases: cross attention from mesh points
to an encoder's states, the norms around a block with its gate and residual scale, and the
orthogonalised update of its weights.

``run`` computes each of them in its plain form (elementary torch operations in 32 bits,
rounded once at the end) or, where ``own`` is true, through the package's classes:

  attend    CrossAttention.forward: softmax(scale q k^T) v of each point and head over the
            states of its sample, of which some may be absent (a length, a mask)
  dattend   CrossAttention.forward and backward: a training step's share
  join      SandwichNorm.forward: y = x + scale * sigmoid(gate) * LN(f) and LN(y)
  djoin     SandwichNorm.backward: the gradients of f, x, the gate and the parameters
  orth      Orthogonalizer: a list of matrices G, each replaced by five Newton-Schulz steps
            X <- a X + (b X X^T + c (X X^T)^2) X from X = G / (|G| + eps)

``exact`` gives the same outputs from the definitions in float64.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
LN_EPS = 1e-5
NS_EPS = 1e-7
NS = (3.4445, -4.7750, 2.0315)  # Orthogonalizer's own
NS_STEPS = 5


def listed():
    return [
        # serving one query point against the states of a coarse mesh's encoder
        dict(name="attend_1_bf16", op="attend", B=1, N=1, S=4096, H=8, G=1, D=32, ragged=False, masked=False, dtype="bf16"),
        # a probe per sample of a batch, long ragged states that heads share four by four
        dict(name="attend_probe_bf16", op="attend", B=4, N=1, S=100_003, H=8, G=4, D=64, ragged=True, masked=False,
             dtype="bf16"),
        # a surface mesh in float32 against masked states, the narrow model's heads
        dict(name="attend_50k_fp32", op="attend", B=1, N=50_003, S=1000, H=8, G=1, D=16, ragged=False, masked=True,
             dtype="fp32"),
        # a mesh of a million points at the 8-block model's width against 512 states
        dict(name="attend_1m_bf16", op="attend", B=1, N=1_000_000, S=512, H=8, G=1, D=32, ragged=False, masked=False,
             dtype="bf16"),
        # training on two samples with states of different lengths, float32, shared heads
        dict(name="dattend_20k_fp32", op="dattend", B=2, N=10_007, S=333, H=8, G=2, D=16, ragged=True, masked=False,
             dtype="fp32"),
        # training at the 8-block model's width in bf16, ragged
        dict(name="dattend_250k_bf16", op="dattend", B=1, N=250_001, S=512, H=8, G=1, D=32, ragged=False, masked=False,
             dtype="bf16"),
        # a serving request of a few thousand query points
        dict(name="join_5k_bf16", op="join", N=5003, C=128, gate=True, pre=True, dtype="bf16"),
        # the gradient on the training subset of the benchmark
        dict(name="djoin_2m_fp32", op="djoin", N=2_000_000, C=128, gate=False, pre=True, dtype="fp32"),
        # a mesh of a million points at the wide model's width in bf16, gated
        dict(name="djoin_1m_bf16", op="djoin", N=1_000_003, C=256, gate=True, pre=True, dtype="bf16"),
        # the gradients of one block of the narrow model, the smallest update
        dict(name="orth_block_fp32", op="orth", L=1, C=128, F=512, H=8, M=64, dtype="fp32"),
        # the gradients of the 24-layer model in bf16: a few hundred matrices
        dict(name="orth_model_bf16", op="orth", L=24, C=256, F=1024, H=8, M=64, dtype="bf16"),
        # a few large maps of ragged sides, one way and the other
        dict(name="orth_large_fp32", op="orth", count=4, rows=1003, cols=4095, dtype="fp32"),
    ]


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["attend", "attend", "dattend", "dattend", "join", "djoin", "orth", "orth"])
    dtype = rng.choice(["bf16", "fp32"])
    if op in ("attend", "dattend"):
        H, D = rng.choice([1, 2, 4, 8, 16]), 16 * rng.choice([1, 1, 2, 2, 3, 4, 4, 5, 6, 8])
        G = rng.choice([g for g in (1, 1, 2, 4, 8) if g <= H])
        B = rng.choice([1, 1, 2, 3, 5])
        S = size(1, 100_003 if op == "attend" else 8192)
        # no more products, rows or states than the largest listed ones
        n = min(1_000_000, int((1.3e11 if op == "attend" else 3.3e10) / (B * S * H * D)), int(2.5e8 / (B * H * D)))
        if dtype == "fp32":
            n = n // 6
        return dict(op=op, B=B, N=size(1, max(n, 1)), S=S, H=H, G=G, D=D, ragged=rng.random() < 0.5,
                    masked=rng.random() < 0.3, dtype=dtype)
    if op in ("join", "djoin"):
        C = 16 * rng.randint(1, 32)
        return dict(op=op, N=size(1, int(1.2e8 / C)), C=C, gate=rng.random() < 0.6, pre=rng.random() < 0.8, dtype=dtype)
    if rng.random() < 0.5:
        H = rng.choice([1, 2, 4, 8])
        return dict(op="orth", L=rng.randint(1, 24), C=16 * H * rng.randint(1, 16 // H), F=size(100, 1024), H=H,
                    M=16 * rng.randint(1, 4), dtype=dtype)
    rows, cols = size(1, 2048), size(1, 4096)
    lo, hi = min(rows, cols), max(rows, cols)
    most = int(4e10 / (lo * lo * (4 * hi + 2 * lo)))
    return dict(op="orth", count=size(1, max(1, min(64, most))), rows=rows, cols=cols, dtype=dtype)


# ------------------------------------------------------------------ inputs

def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 64 + stream)
    return g


def _randn(shape, dtype, seed, stream, scale=1.0):
    return (torch.randn(shape, generator=_gen(seed, stream), device="cuda") * scale).to(dtype)


def _uniform(shape, bound, g):
    return (torch.rand(shape, generator=g, device="cuda") * 2.0 - 1.0) * bound


def _lengths(case):
    """States of each sample: the first has them all, the others some part."""
    if not case["ragged"]:
        return [case["S"]] * case["B"]
    return [case["S"]] + [case["S"] * ((37 * b) % 64) // 64 for b in range(1, case["B"])]


def _shapes(case):
    """The matrices of L blocks (Physics-Attention and the gated feed-forward), or a list of large
    ones, every second of them turned."""
    if "L" not in case:
        r, c = case["rows"], case["cols"]
        return [(r, c) if i % 2 == 0 else (c, r) for i in range(case["count"])]
    C, F, H, M = case["C"], case["F"], case["H"], case["M"]
    dh = C // H
    return [(C, H * M), (C, C), (H, dh, dh), (H, dh, dh), (H, dh, dh), (C, C), (C, F), (C, F), (F, C)] * case["L"]


def prepare(case, seed):
    s = {"case": case}
    op, dtype = case["op"], DTYPES[case["dtype"]]
    if op in ("attend", "dattend"):
        B, N, S, H, D = case["B"], case["N"], case["S"], case["H"], case["D"]
        s["q"] = _randn((B, N, H, D), dtype, seed, 1, 1.5)
        # one projection gives the states' keys and values, side by side
        kv = _randn((B, S, 2, H // case["G"], D), dtype, seed, 2)
        s["k"], s["v"] = kv[:, :, 0], kv[:, :, 1]
        s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda") if case["ragged"] else None
        s["mask"] = torch.rand((B, S), generator=_gen(seed, 3), device="cuda") < 0.8 if case["masked"] else None
        if op == "dattend":
            s["g"] = _randn((B, N, H, D), dtype, seed, 4)
        if own:
            from paper_2602_04940_amd import CrossAttention
            s["attention"] = CrossAttention(H, D, kv_heads=H // case["G"], dtype=case["dtype"])
        return s
    if op in ("join", "djoin"):
        N, C = case["N"], case["C"]
        g = _gen(seed, 8)
        s["f"], s["x"] = _randn((N, C), dtype, seed, 1, 0.5), _randn((N, C), dtype, seed, 2)
        s["gate"] = _randn((N, C), dtype, seed, 3) if case["gate"] else None
        s["gamma_post"], s["beta_post"] = 1.0 + _uniform((C,), 0.1, g), _uniform((C,), 0.1, g)
        s["scale"] = 0.3 + _uniform((C,), 0.1, g)
        s["gamma_pre"], s["beta_pre"] = (1.0 + _uniform((C,), 0.1, g), _uniform((C,), 0.1, g)) if case["pre"] else (None, None)
        if op == "djoin":
            # the backward reads the forward's sum y, not x
            s["y"] = s.pop("x")
            s["gy"] = _randn((N, C), dtype, seed, 4)
            s["gn"] = _randn((N, C), dtype, seed, 5) if case["pre"] else None
        if own:
            from paper_2602_04940_amd import SandwichNorm
            s["norm"] = SandwichNorm(C, dtype=case["dtype"], eps=LN_EPS)
        return s
    # Gradients: sums of outer products whose sizes fall off, and noise, of tensors of different sizes.
    # The program keeps them in one buffer, each a view of it, and the updates in another.
    rng, shapes = random.Random(seed), _shapes(case)
    g, at = _gen(seed, 9), 0
    s["flat"] = torch.empty(sum(math.prod(shape) for shape in shapes), dtype=dtype, device="cuda")
    s["flat_out"], s["grads"], s["out"] = torch.empty_like(s["flat"]), [], []
    for shape in shapes:
        r, c = shape[-2:]
        k = min(r, c, 64)
        left = torch.randn((*shape[:-1], k), generator=g, device="cuda") / torch.arange(1, k + 1, device="cuda")
        t = left @ torch.randn((*shape[:-2], k, c), generator=g, device="cuda")
        t = t + 0.3 * torch.randn(shape, generator=g, device="cuda")
        for name, flat in (("grads", s["flat"]), ("out", s["flat_out"])):
            s[name].append(flat[at:at + t.numel()].view(shape))
        s["grads"][-1].copy_(t * 10.0 ** rng.uniform(-5, -2))
        at += t.numel()
    if own:
        from paper_2602_04940_amd import Orthogonalizer
        s["orth"] = Orthogonalizer(steps=NS_STEPS, eps=NS_EPS)
    return s


# ------------------------------------------------------------------ the call

def run(state):
    op = state["case"]["op"]
    if not own:
        return {"attend": _plain_attend, "dattend": _plain_dattend, "join": _plain_join, "djoin": _plain_djoin,
                "orth": _plain_orth}[op](state)
    if op == "attend":
        out, _ = state["attention"].forward(state["q"], state["k"], state["v"], lengths=state["lengths"], mask=state["mask"])
        return out
    if op == "dattend":
        a, q, k, v = state["attention"], state["q"], state["k"], state["v"]
        out, lse = a.forward(q, k, v, lengths=state["lengths"], mask=state["mask"])
        dq, dk, dv = a.backward(q, k, v, out, lse, state["g"], lengths=state["lengths"], mask=state["mask"])
        return {"out": out, "dq": dq, "dk": dk, "dv": dv}
    if op == "join":
        y, n = state["norm"].forward(state["f"], state["x"], state["gamma_post"], state["beta_post"], state["scale"],
                                     gate=state["gate"], gamma_pre=state["gamma_pre"], beta_pre=state["beta_pre"])
        return {"y": y} if n is None else {"y": y, "n": n}
    if op == "djoin":
        df, dx, dgate, d = state["norm"].backward(state["f"], state["y"], state["gy"], state["gamma_post"],
                                                  state["beta_post"], state["scale"], gate=state["gate"],
                                                  gn=state["gn"], gamma_pre=state["gamma_pre"])
        res = {"df": df, "dx": dx, "dgamma_post": d["gamma_post"], "dbeta_post": d["beta_post"], "dscale": d["scale"]}
        if state["gate"] is not None:
            res["dgate"] = dgate
        if state["gn"] is not None:
            res.update(dgamma_pre=d["gamma_pre"], dbeta_pre=d["beta_pre"])
        return res
    state["orth"](state["grads"], out=state["out"])
    return state["flat_out"]


# ------------------------------------------------------------------ plain forms

def _plain_states(state, b):
    """Keys and values of sample b by query head [H, S, D] (absent ones zero), and which are there."""
    case = state["case"]
    there = torch.ones(case["S"], dtype=torch.bool, device="cuda")
    if state["lengths"] is not None:
        there &= torch.arange(case["S"], device="cuda") < state["lengths"][b]
    if state["mask"] is not None:
        there &= state["mask"][b]
    k, v = (torch.where(there[:, None, None], t[b], torch.zeros_like(t[b])).float().repeat_interleave(case["G"], dim=1)
            .transpose(0, 1).contiguous() for t in (state["k"], state["v"]))
    return k, v, there


def _plain_weights(q, k, there):
    """softmax of the scaled scores [H, n, S]; rows of no state are zero."""
    s = (q @ k.transpose(1, 2)) * (1.0 / math.sqrt(q.shape[2]))
    s = torch.where(there, s, torch.full_like(s, -math.inf))
    m = s.amax(2, keepdim=True)
    p = torch.exp(s - torch.where(m == -math.inf, torch.zeros_like(m), m))
    z = p.sum(2, keepdim=True)
    return p / torch.where(z > 0, z, torch.ones_like(z))


def _step(case):
    return max(1, (1 << 28) // (case["H"] * case["S"]))


def _plain_attend(state):
    case, out = state["case"], torch.empty_like(state["q"])
    for b in range(case["B"]):
        k, v, there = _plain_states(state, b)
        for a in range(0, case["N"], _step(case)):
            q = state["q"][b, a:a + _step(case)].float().transpose(0, 1)
            out[b, a:a + _step(case)] = (_plain_weights(q, k, there) @ v).transpose(0, 1).to(out.dtype)
    return out


def _plain_dattend(state):
    case, dtype = state["case"], state["q"].dtype
    B, S, H, G, D = (case[n] for n in ("B", "S", "H", "G", "D"))
    out, dq = torch.empty_like(state["q"]), torch.empty_like(state["q"])
    dks, dvs = [], []
    for b in range(B):
        k, v, there = _plain_states(state, b)
        dk, dv = torch.zeros((2, H, S, D), dtype=torch.float64, device="cuda")
        for a in range(0, case["N"], _step(case)):
            e = a + _step(case)
            q, g = (state[n][b, a:e].float().transpose(0, 1).contiguous() for n in ("q", "g"))
            p = _plain_weights(q, k, there)
            o = p @ v
            dp = g @ v.transpose(1, 2)
            ds = p * (dp - (g * o).sum(2, keepdim=True)) * (1.0 / math.sqrt(D))
            dv += p.transpose(1, 2) @ g
            dk += ds.transpose(1, 2) @ q
            out[b, a:e] = o.transpose(0, 1).to(dtype)
            dq[b, a:e] = (ds @ k).transpose(0, 1).to(dtype)
        for total, parts in ((dk, dks), (dv, dvs)):
            parts.append(total.view(H // G, G, S, D).sum(1).transpose(0, 1).to(dtype))
    return {"out": out, "dq": dq, "dk": torch.stack(dks), "dv": torch.stack(dvs)}


def _plain_stats(y):
    c = y - y.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt((c * c).mean(1, keepdim=True) + LN_EPS)
    return c * rstd, rstd


def _plain_gate(state):
    if state["gate"] is None:
        return 1.0
    return 1.0 / (1.0 + torch.exp(-state["gate"].float()))


def _plain_join(state):
    dtype = state["x"].dtype
    h, _ = _plain_stats(state["f"].float())
    y = state["x"].float() + state["scale"] * _plain_gate(state) * (h * state["gamma_post"] + state["beta_post"])
    if state["gamma_pre"] is None:
        return {"y": y.to(dtype)}
    n, _ = _plain_stats(y)
    return {"y": y.to(dtype), "n": (n * state["gamma_pre"] + state["beta_pre"]).to(dtype)}


def _plain_djoin(state):
    dtype, res = state["y"].dtype, {}
    dy = state["gy"].float()
    if state["gn"] is not None:
        gn = state["gn"].float()
        h, rstd = _plain_stats(state["y"].float())
        e = gn * state["gamma_pre"]
        dy = dy + rstd * (e - e.mean(1, keepdim=True) - h * (e * h).mean(1, keepdim=True))
        res.update(dgamma_pre=(gn * h).sum(0, dtype=torch.float64).float(), dbeta_pre=gn.sum(0, dtype=torch.float64).float())
    res["dx"] = dy.to(dtype)
    h, rstd = _plain_stats(state["f"].float())
    m, gate = h * state["gamma_post"] + state["beta_post"], _plain_gate(state)
    res["dscale"] = (dy * gate * m).sum(0, dtype=torch.float64).float()
    if state["gate"] is not None:
        res["dgate"] = (dy * state["scale"] * m * gate * (1.0 - gate)).to(dtype)
    dm = dy * state["scale"] * gate
    res.update(dgamma_post=(dm * h).sum(0, dtype=torch.float64).float(), dbeta_post=dm.sum(0, dtype=torch.float64).float())
    e = dm * state["gamma_post"]
    res["df"] = (rstd * (e - e.mean(1, keepdim=True) - h * (e * h).mean(1, keepdim=True))).to(dtype)
    return res


def _plain_orth(state):
    a, b, c = NS
    for t, out in zip(state["grads"], state["out"]):
        x = t.float()
        turned = x.shape[-2] > x.shape[-1]
        if turned:
            x = x.transpose(-2, -1).contiguous()
        norm = x.double().square().sum((-2, -1), keepdim=True).sqrt()
        x = (x.double() / (norm + NS_EPS)).float()
        for _ in range(NS_STEPS):
            gram = x @ x.transpose(-2, -1)
            x = a * x + (b * gram + c * (gram @ gram)) @ x
        out.copy_(x.transpose(-2, -1) if turned else x)
    return state["flat_out"]


# ------------------------------------------------------------------ what it takes

def work(case):
    """Bytes: inputs once, outputs once.  Flops: the products of the definition, without
    what is computed again."""
    op, e = case["op"], 2 if case["dtype"] == "bf16" else 4
    if op in ("attend", "dattend"):
        states = sum(_lengths(case))
        rows, kv = case["B"] * case["N"] * case["H"] * case["D"], 2 * states * (case["H"] // case["G"]) * case["D"]
        pairs = 2.0 * case["N"] * states * case["H"] * case["D"]
        if op == "attend":
            return {"bytes": float(e * (2 * rows + kv)), "flops": 2 * pairs}
        # q, g in, out, dq out; scores, weights times values, and five products back, scores among them
        return {"bytes": float(e * (4 * rows + 2 * kv)), "flops": 6 * pairs}
    if op in ("join", "djoin"):
        N, C, gate, pre = case["N"], case["C"], case["gate"], case["pre"]
        rows = 3 + gate + pre if op == "join" else 4 + pre + 2 * gate + 1 * pre
        return {"bytes": float(rows * N * C * e + 4 * C * (5 if op == "join" else 9)), "flops": 20.0 * N * C}
    size = flops = 0.0
    for shape in _shapes(case):
        n, lo, hi = math.prod(shape), min(shape[-2:]), max(shape[-2:])
        size += 2 * n * e
        # X X^T and its square are symmetric: half their products
        flops += NS_STEPS * (n // (lo * hi)) * (lo * lo * hi + float(lo) ** 3 + 2 * lo * lo * hi)
    return {"bytes": size, "flops": flops}


# ------------------------------------------------------------------ float64

def exact(case, seed):
    """The outputs from the definitions in float64, the gradients by differentiation."""
    st = _plain_inputs(case, seed)
    op = case["op"]
    if op == "orth":
        return torch.cat([_exact_orth(t.double()).reshape(-1) for t in st["grads"]])
    if op in ("join", "djoin"):
        return _exact_join(case, st)
    out, dq = [], []
    dk, dv = (torch.zeros(st[n].shape, dtype=torch.float64, device="cuda") for n in ("k", "v"))
    train = op == "dattend"
    for b in range(case["B"]):
        there = torch.arange(case["S"], device="cuda") < _lengths(case)[b]
        if st["mask"] is not None:
            there = there & st["mask"][b]
        at = there.nonzero()[:, 0]
        k, v = (st[n][b][at].double().requires_grad_(train) for n in ("k", "v"))
        step = max(1, (1 << 26) // (case["H"] * max(1, len(at))))
        for a in range(0, case["N"], step):
            q = st["q"][b, a:a + step].double().requires_grad_(train)
            heads = []
            for h in range(case["H"]):
                if len(at) == 0:
                    heads.append(q[:, h] * 0.0 + 0.0 * v.sum() + 0.0 * k.sum())
                    continue
                s = q[:, h] @ k[:, h // case["G"]].T / math.sqrt(case["D"])
                heads.append(torch.softmax(s, dim=1) @ v[:, h // case["G"]])
            o = torch.stack(heads, dim=1)
            out.append(o.detach())
            if train:
                o.backward(st["g"][b, a:a + step].double())
                dq.append(q.grad)
        if train:
            dk[b, at], dv[b, at] = k.grad, v.grad
    shape = st["q"].shape
    out = torch.cat(out).view(shape)
    return {"out": out, "dq": torch.cat(dq).view(shape), "dk": dk, "dv": dv} if train else out


def _exact_join(case, st):
    names = [n for n in ("gamma_post", "beta_post", "scale", "gamma_pre", "beta_pre") if st[n] is not None]
    p = {n: st[n].double().requires_grad_() for n in names}
    norm, C = torch.nn.functional.layer_norm, (case["C"],)
    res = {}

    def add(**values):
        for n, t in values.items():
            res.setdefault(n, []).append(t.detach())

    for a in range(0, case["N"], 1 << 16):
        f = st["f"][a:a + (1 << 16)].double().requires_grad_()
        gate = None if st["gate"] is None else st["gate"][a:a + (1 << 16)].double().requires_grad_()
        m = p["scale"] * norm(f, C, p["gamma_post"], p["beta_post"], LN_EPS)
        if gate is not None:
            m = m * torch.sigmoid(gate)
        if case["op"] == "join":
            y = st["x"][a:a + (1 << 16)].double() + m
            add(y=y)
            if case["pre"]:
                add(n=norm(y, C, p["gamma_pre"], p["beta_pre"], LN_EPS))
            continue
        y = st["y"][a:a + (1 << 16)].double().requires_grad_()
        gy = st["gy"][a:a + (1 << 16)].double()
        if case["pre"]:
            norm(y, C, p["gamma_pre"], p["beta_pre"], LN_EPS).backward(st["gn"][a:a + (1 << 16)].double())
            gy = gy + y.grad
        m.backward(gy)
        add(df=f.grad, dx=gy)
        if gate is not None:
            add(dgate=gate.grad)
    res = {n: torch.cat(t) for n, t in res.items()}
    if case["op"] == "djoin":
        res.update({"d" + n: t.grad for n, t in p.items()})
    return res


def _exact_orth(t):
    """X p(X^T X) on the side with fewer columns, p of a step as one polynomial of the Gram matrix."""
    turned = t.shape[-1] > t.shape[-2]
    x = t.transpose(-2, -1) if turned else t
    x = x / (torch.linalg.matrix_norm(x, keepdim=True) + NS_EPS)
    one = torch.eye(x.shape[-1], dtype=torch.float64, device=x.device)
    for _ in range(NS_STEPS):
        gram = x.transpose(-2, -1) @ x
        x = x @ (NS[0] * one + gram @ (NS[1] * one + NS[2] * gram))
    return x.transpose(-2, -1) if turned else x


def _plain_inputs(case, seed):
    """The inputs of a case without the package's objects."""
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was
