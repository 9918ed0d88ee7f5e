"""The operators of a conditioned block on the GPU against the float64 reference: every type and
padded width, lengths around the tiles, shared heads, masks that leave rows empty, what absent
states hold, views, streams, captured graphs.

Bars, fixed before the first run; u is 2^-24.

Attention.  A score is a sum of D products of operands carried to u: it is off by (4 + sqrt D) u of
X = scale |q| |k| at its largest, and so is its weight, relative to itself.  Sums over S states and N
points walk their square roots.  In float32 every output is then within four times
(8 + sqrt S + sqrt N + (4 + sqrt D) X) u of the size of its terms (the sum of their absolute values).
In bfloat16 the output is rounded once (2^-8 of itself), and so are its weights (2^-8 of the size of its
terms); so is dv, and so are dq and dk with the slopes in the weights' place: g.out is taken from the rounded output
first, but put right by float32 sums.  What rounded operands do to that mend is of second order: 2 2^-8 of 2^-8.

Norms.  As the other training operators': four walks over C, and over N for sums over rows, of the
largest value in float32; in bfloat16 2^-8 in the mean square.

Orthogonalised matrices.  A product's operands are within 2^-22 of themselves and its sum walks
sqrt(r + c) u: d = 2^-22 + sqrt(r + c) u of the Frobenius norm a step.  Where all singular values start near one
another, the polynomial's slope is at most three times its value, in five steps 16 d; with singular
values near zero a step grows errors as it grows those, 3.45 times, and the bar is 6 3.45^5 d |X| / |result| with
|X| = 1 at the start.  bfloat16 results add 2^-8."""
import math

import numpy as np
import pytest

from gpu_helpers import banner, normwise, rel_l2, to_device, to_host

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _round(a, dtype):
    """float64 values that the storage type holds exactly"""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32))
    return (t.bfloat16() if dtype == "bf16" else t).double().numpy()


# ------------------------------------------------------------------ cross attention

def _case(B, N, S, H, HK, D, dtype, seed=0, scale=1.0):
    rng = np.random.default_rng([seed, B, N, S, H, D])
    q, g = (_round(rng.standard_normal((B, N, H, D)) * s, dtype) for s in (scale, 1.0))
    k, v = (_round(rng.standard_normal((B, S, HK, D)), dtype) for _ in range(2))
    return q, k, v, g


def _check(name, got, ref, size, dtype, walk):
    got = to_host(got)
    assert got.shape == ref.shape, name
    if ref.size == 0:
        return
    assert np.isfinite(got).all(), name
    err = np.abs(got - ref)
    bar = 4 * walk * U * size.max()
    if dtype == "bf16":
        bar = bar + 2.0 ** -8 * (np.abs(ref) + 1.02 * size)
    else:
        bar = np.full_like(err, bar)
    print(f"{name}: normwise {normwise(got, ref):.2e}, of the bar {float((err / np.maximum(bar, 1e-300)).max()):.3f}", flush=True)
    assert (err <= bar).all(), name


def _run(q, k, v, g, dtype, HK, lengths=None, mask=None, scale=None):
    import torch
    from paper_2602_04940_amd import CrossAttention
    with CrossAttention(q.shape[2], q.shape[3], kv_heads=HK, dtype=dtype, scale=scale) as a:
        t = [to_device(x, dtype) for x in (q, k, v, g)]
        more = dict(lengths=None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda"),
                    mask=None if mask is None else torch.tensor(mask, device="cuda"))
        out, lse = a.forward(*t[:3], **more)
        grads = a.backward(*t[:3], out, lse, t[3], **more)
        torch.cuda.synchronize()
    return out, lse, dict(zip(("dq", "dk", "dv"), grads))


def _compare(q, k, v, g, dtype, there, scale, out, lse, grads):
    from oracle import conditioned as R
    B, N, H, D = q.shape
    S, G = k.shape[1], H // k.shape[2]
    k, v = (np.where(there[..., None, None], t, 0.0) for t in (k, v))
    ref, ref_lse = R.cross_forward(q, k, v, there, scale)
    refs, sizes = R.cross_backward(q, k, v, there, scale, g)
    X = scale * np.sqrt((q * q).sum(3).max(initial=0.0) * (k * k).sum(3).max(initial=0.0))
    walk = 8 + math.sqrt(S) + math.sqrt(N * G) + (4 + math.sqrt(D)) * X
    _check("out", out, ref, sizes["out"], dtype, walk)
    empty = np.isinf(ref_lse)
    got = to_host(lse)
    assert (got[empty] == -np.inf).all()
    assert np.abs(got[~empty] - ref_lse[~empty]).max(initial=0.0) <= 4 * walk * U * (1 + X)
    for name in ("dq", "dk", "dv"):
        _check(name, grads[name], refs[name], sizes[name], dtype, walk)
        if name != "dq":
            assert (to_host(grads[name])[~there] == 0).all(), name


# (B, N, S, H, Hkv, D): every padded width, exactly and not; one state, lengths around a tile of 32 and
# of 64 and a block of 128; rows of one query, of a few (a wave of its own, the states split over
# workgroups), around a wave's 32 and a workgroup's 128; enough for the blocks of 64 rows per wave; sums over
# points that are split.
CROSS = [(1, 1, 1, 1, 1, 16), (1, 1, 700, 8, 8, 32), (2, 1, 3001, 8, 2, 64), (3, 1, 129, 16, 2, 128), (1, 2, 33, 4, 4, 48),
         (2, 4, 1000, 8, 1, 16), (1, 31, 64, 2, 1, 80), (2, 33, 65, 3, 3, 32), (1, 127, 32, 4, 2, 64), (1, 130, 63, 2, 2, 112),
         (2, 129, 31, 6, 2, 96), (1, 300, 500, 2, 2, 128), (1, 257, 127, 8, 8, 16), (1, 1003, 129, 4, 1, 32),
         (1, 70, 2500, 1, 1, 64), (2, 2049, 40, 2, 2, 16), (1, 17_000, 70, 8, 8, 32), (1, 8500, 45, 16, 4, 64),
         (1, 33_000, 33, 4, 4, 16), (2, 17_000, 97, 16, 16, 32), (1, 70_000, 40, 8, 4, 48),
         (2, 50, 90, 16, 1, 128), (1, 9, 70, 64, 1, 32), (1, 3, 150, 1024, 1, 16), (2, 700, 3000, 32, 2, 32)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,N,S,H,HK,D", CROSS)
def test_cross_forward_and_backward(B, N, S, H, HK, D, dtype):
    from oracle import conditioned as R
    banner(f"cross B={B} N={N} S={S} H={H}/{HK} D={D} {dtype}")
    q, k, v, g = _case(B, N, S, H, HK, D, dtype)
    _compare(q, k, v, g, dtype, R.present(B, S), 1 / math.sqrt(D), *_run(q, k, v, g, dtype, HK))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("what", ["lengths", "mask", "both"])
@pytest.mark.parametrize("B,N,S,H,HK,D", [(4, 3, 700, 4, 2, 32), (4, 200, 130, 2, 2, 16), (4, 150, 97, 4, 1, 64), (4, 40, 300, 2, 2, 128),
                                          (4, 9000, 66, 4, 4, 32), (4, 9000, 67, 16, 16, 16)])
def test_cross_states_that_are_absent(B, N, S, H, HK, D, what, dtype):
    """Lengths of all, one, none and beyond the ends, masks with long runs and a sample of none; absent
    states hold infinities and not-a-numbers."""
    from oracle import conditioned as R
    banner(f"cross absent {what} B={B} N={N} S={S} H={H}/{HK} D={D} {dtype}")
    q, k, v, g = _case(B, N, S, H, HK, D, dtype, seed=1)
    rng = np.random.default_rng(2)
    lengths = [S + 7, 1, -3, S // 2] if what != "mask" else None
    mask = None
    if what != "lengths":
        mask = rng.random((B, S)) < 0.5
        mask[0, 20:min(S - 3, 160)] = False
        mask[3] = what == "both"
        if what == "both":
            mask[0] = np.arange(S) == S - 1
    there = R.present(B, S, None if lengths is None else np.clip(lengths, 0, S), mask)
    bad = rng.choice([np.nan, np.inf, -np.inf], (B, S))
    k, v = (np.where(there[..., None, None], t, bad[..., None, None]) for t in (k, v))
    _compare(q, k, v, g, dtype, there, 1 / math.sqrt(D), *_run(q, k, v, g, dtype, HK, lengths, mask))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("factor", [30.0, -30.0])
def test_cross_scores_far_from_zero(dtype, factor):
    """Scores of hundreds, growing from tile to tile or falling, whose exponentials leave float32
    without the maximum."""
    from oracle import conditioned as R
    B, N, S, H, D = 1, 200, 300, 2, 32
    q, k, v, g = _case(B, N, S, H, H, D, dtype, seed=3)
    q[..., 0] = _round(np.abs(q[..., 0]) + 1, dtype)
    k[..., 0] = _round(factor * np.arange(S)[None, :, None] / S * np.ones((B, S, H)), dtype)
    _compare(q, k, v, g, dtype, R.present(B, S), 1.0, *_run(q, k, v, g, dtype, H, scale=1.0))


def test_cross_gradient_against_differences():
    """d/dt of sum(g * out) along random directions, from the float64 reference's forward (good to about
    1e-7 of the terms), against float32 gradients."""
    from oracle import conditioned as R
    B, N, S, H, HK, D, t = 2, 40, 50, 4, 2, 16, 1e-4
    q, k, v, g = _case(B, N, S, H, HK, D, "fp32", seed=4)
    lengths = [50, 20]
    there = R.present(B, S, lengths)
    _, _, grads = _run(q, k, v, g, "fp32", HK, lengths)
    rng = np.random.default_rng(5)
    dirs = [rng.standard_normal(a.shape) for a in (q, k, v)]

    def loss(s):
        return (g * R.cross_forward(*(a + s * d for a, d in zip((q, k, v), dirs)), there, 0.25)[0]).sum()
    fd = (loss(t) - loss(-t)) / (2 * t)
    terms = [(to_host(grads[n]) * d).sum() for n, d in zip(("dq", "dk", "dv"), dirs)]
    size = math.sqrt(sum((to_host(grads[n]) ** 2).sum() for n in grads))
    print(f"differences {fd:.6e}, gradients {sum(terms):.6e}", flush=True)
    assert abs(sum(terms) - fd) / size <= 1e-5


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_cross_views_and_destinations(dtype):
    """Keys and values of one projection, queries out of wider rows, a gradient broadcast over samples,
    in any order of the dimensions: bitwise as contiguous copies; nothing is written beside the results."""
    import torch
    from paper_2602_04940_amd import CrossAttention
    B, N, S, H, HK, D = 3, 70, 90, 4, 2, 32
    tt = torch.float32 if dtype == "fp32" else torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(6)
    kv = torch.randn((B, S, 2, HK, D), generator=gen, device="cuda").to(tt)
    wide = torch.randn((N, B, H + 3, D + 16), generator=gen, device="cuda").to(tt)
    q, k, v = wide.transpose(0, 1)[:, :, 1:H + 1, 16:], kv[:, :, 0], kv[:, :, 1]
    g = torch.randn((1, N, H, D), generator=gen, device="cuda").to(tt).expand(B, N, H, D)
    with CrossAttention(H, D, kv_heads=HK, dtype=dtype) as a:
        guard = torch.full((B * N * H * D + 64,), 7.0, device="cuda", dtype=tt)
        lg = torch.full((B * N * H + 64,), 7.0, device="cuda")
        out, lse = a.forward(q, k, v, out=guard[32:-32].view(B, N, H, D), lse=lg[32:-32].view(B, H, N))
        dq = torch.full_like(guard, 7.0)
        grads = a.backward(q, k, v, out, lse, g, dq=dq[32:-32].view(B, N, H, D))
        c = [t.contiguous() for t in (q, k, v, g)]
        out2, lse2 = a.forward(*c[:3])
        grads2 = a.backward(*c[:3], out2, lse2, c[3])
        torch.cuda.synchronize()
    assert torch.equal(out, out2) and torch.equal(lse, lse2) and all(torch.equal(x, y) for x, y in zip(grads, grads2))
    for t in (guard, lg, dq):
        assert (t[:32] == 7).all() and (t[-32:] == 7).all()


def test_cross_offsets_past_32_bits():
    """States and queries whose rows lie 2^31 elements and more from the first."""
    import torch
    from paper_2602_04940_amd import CrossAttention
    N, S, H, D = 3, 3, 2, 32
    big = torch.empty(3 * ((1 << 30) + (1 << 29)), dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(7)
    q, k, v, g = (torch.as_strided(big, (1, N, H, D), (0, (1 << 30) + (1 << 29), D, 1), off * 4096) for off in range(4))
    for t in (q, k, v, g):
        t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
    with CrossAttention(H, D) as a:
        out, lse = a.forward(q, k, v)
        grads = a.backward(q, k, v, out, lse, g)
        c = [t.contiguous() for t in (q, k, v, g)]
        out2, lse2 = a.forward(*c[:3])
        grads2 = a.backward(*c[:3], out2, lse2, c[3])
        torch.cuda.synchronize()
    assert torch.equal(out, out2) and torch.equal(lse, lse2) and all(torch.equal(x, y) for x, y in zip(grads, grads2))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_cross_of_nothing(dtype):
    import torch
    from paper_2602_04940_amd import CrossAttention
    tt = torch.float32 if dtype == "fp32" else torch.bfloat16

    def some(*shape):
        return torch.ones(shape, device="cuda", dtype=tt)
    with CrossAttention(2, 16, dtype=dtype) as a:
        for B, N, S in ((0, 3, 4), (2, 0, 4), (2, 3, 0), (0, 0, 0), (2, 0, 0)):
            q, k = some(B, N, 2, 16), some(B, S, 2, 16)
            out, lse = a.forward(q, k, k.clone())
            dq, dk, dv = a.backward(q, k, k.clone(), out, lse, q.clone())
            torch.cuda.synchronize()
            for t in (out, dq, dk, dv):
                assert (t == 0).all()
            assert (lse == -math.inf).all() and out.shape == q.shape and dk.shape == k.shape


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_cross_repeats_bitwise(dtype):
    B, N, S, H, HK, D = 2, 3000, 200, 4, 2, 32
    q, k, v, g = _case(B, N, S, H, HK, D, dtype, seed=8)
    import torch
    first, second = (_run(q, k, v, g, dtype, HK) for _ in range(2))
    assert torch.equal(first[0], second[0]) and torch.equal(first[1], second[1])
    assert all(torch.equal(first[2][n], second[2][n]) for n in first[2])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_cross_first_call_captured(dtype):
    """Enough rows for the kernels that hold all states in LDS, which need no workspace forward: a handle's
    first call may be captured."""
    import torch
    from paper_2602_04940_amd import CrossAttention
    q, k, v, _ = (to_device(t, dtype) for t in _case(1, 131_072, 64, 4, 1, 16, dtype, seed=10))
    with CrossAttention(4, 16, 1, dtype=dtype) as a, CrossAttention(4, 16, 1, dtype=dtype) as b:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out, lse = a.forward(q, k, v)
        for scale in (1.0, -0.5, 2.0):
            q.mul_(scale)
            graph.replay()
            torch.cuda.synchronize()
            ref, ref_lse = b.forward(q, k, v)
            assert a.bytes() == 0 and torch.equal(out, ref) and torch.equal(lse, ref_lse), scale


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_cross_rows_are_independent(dtype):
    """A query of not-a-numbers, or a gradient of one, reaches its own row of out and dq alone."""
    import torch
    from paper_2602_04940_amd import CrossAttention
    q, k, v, g = (to_device(t, dtype) for t in _case(1, 300, 70, 2, 2, 32, dtype, seed=9))
    with CrossAttention(2, 32, dtype=dtype) as a:
        out, lse = a.forward(q, k, v)
        dq, _, _ = a.backward(q, k, v, out, lse, g)
        q2, g2 = q.clone(), g.clone()
        q2[0, 17, 1], g2[0, 18, 0] = math.nan, math.nan
        out2, lse2 = a.forward(q2, k, v)
        dq2, _, _ = a.backward(q2, k, v, out2, lse2, g2)
        torch.cuda.synchronize()
    hit = torch.zeros((300, 2), dtype=torch.bool, device="cuda")
    hit[17, 1] = True
    assert out2[0][hit].isnan().all() and torch.equal(out2[0][~hit], out[0][~hit])
    hit[18, 0] = True
    assert dq2[0][hit].isnan().all() and torch.equal(dq2[0][~hit], dq[0][~hit])


# ------------------------------------------------------------------ the norms around a block

def _close(name, got, ref, dtype, K):
    if ref.size == 0:
        return
    got = to_host(got)
    assert got.shape == ref.shape and np.isfinite(got).all(), name
    if dtype == "fp32":
        err, bar = normwise(got, ref), 4 * U * (8 + sum(math.sqrt(k) for k in K))
    else:
        err, bar = rel_l2(got, ref), 2.0 ** -8
    print(f"{name}: {err:.2e} (bar {bar:.2e})", flush=True)
    assert err <= bar, name


def _sandwich(N, C, gate, pre, dtype, seed=0, scale=1.0):
    rng = np.random.default_rng([seed, N, C])
    names = ("gamma_post", "beta_post", "scale") + (("gamma_pre", "beta_pre") if pre else ())
    w = {n: np.float32(rng.uniform(0.5, 1.5, C) if n[0] in "gs" else rng.uniform(-0.5, 0.5, C)).astype(np.float64) for n in names}
    x = {n: _round(rng.standard_normal((N, C)) * scale, dtype) for n in ("f", "x", "gate", "gy", "gn")}
    if not gate:
        x["gate"] = None
    if not pre:
        x["gn"] = None
    return x, w


SANDWICH = [(1, 16), (3, 48), (64, 80), (257, 128), (1001, 256), (500, 272), (333, 512), (9001, 64), (40_003, 32)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("pre", [True, False])
@pytest.mark.parametrize("N,C", SANDWICH)
def test_sandwich_forward_and_backward(N, C, pre, gate, dtype):
    import torch
    from oracle import conditioned as R
    from paper_2602_04940_amd import SandwichNorm
    banner(f"sandwich N={N} C={C} pre={pre} gate={gate} {dtype}")
    x, w = _sandwich(N, C, gate, pre, dtype)
    d = {n: None if t is None else to_device(t, dtype) for n, t in x.items()}
    p = {n: to_device(t, "fp32") for n, t in w.items()}
    with SandwichNorm(C, dtype=dtype) as s:
        y, out = s.forward(d["f"], d["x"], gate=d["gate"], **p)
        y2 = _round(R.sandwich_forward(x["f"], x["x"], x["gate"], w, 1e-5)[0], dtype)
        back = {n: t for n, t in p.items() if n != "beta_pre"}
        df, dx, dgate, grads = s.backward(d["f"], to_device(y2, dtype), d["gy"], gate=d["gate"], gn=d["gn"], **back)
        torch.cuda.synchronize()
    ry, rn = R.sandwich_forward(x["f"], x["x"], x["gate"], w, 1e-5)
    _close("y", y, ry, dtype, (C,))
    assert (out is None) == (not pre) and (dgate is None) == (not gate)
    if pre:
        _close("out", out, rn, dtype, (C, C))
    ref = R.sandwich_backward(x["f"], y2, x["gate"], x["gy"], x["gn"], w, 1e-5)
    _close("df", df, ref["df"], dtype, (C, C))
    _close("dx", dx, ref["dx"], dtype, (C,))
    if gate:
        _close("dgate", dgate, ref["dgate"], dtype, (C,))
    for n in ("gamma_post", "beta_post", "scale", "gamma_pre", "beta_pre"):
        if n in w:
            _close(n, grads[n], ref[n], "fp32", (C, C, N))
        else:
            assert grads[n] is None


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_sandwich_gates_far_from_zero(dtype):
    """Gates of hundreds and infinite ones: open or closed, no not-a-number; a closed gate leaves x."""
    import torch
    from oracle import conditioned as R
    from paper_2602_04940_amd import SandwichNorm
    N, C = 200, 64
    x, w = _sandwich(N, C, True, True, dtype, seed=1)
    x["gate"] = _round(x["gate"] * 60.0, dtype)
    x["gate"][0], x["gate"][1], x["gate"][2] = -np.inf, np.inf, -500.0
    d = {n: to_device(t, dtype) for n, t in x.items()}
    p = {n: to_device(t, "fp32") for n, t in w.items()}
    with SandwichNorm(C, dtype=dtype) as s:
        y, out = s.forward(d["f"], d["x"], gate=d["gate"], **p)
        p.pop("beta_pre")
        df, dx, dgate, grads = s.backward(d["f"], y, d["gy"], gate=d["gate"], gn=d["gn"], **p)
        torch.cuda.synchronize()
    ry, rn = R.sandwich_forward(x["f"], x["x"], x["gate"], w, 1e-5)
    _close("y", y, ry, dtype, (C,))
    _close("out", out, rn, dtype, (C, C))
    assert torch.equal(y[0], d["x"][0]) and torch.equal(y[2], d["x"][2]) and (df[0] == 0).all()
    ref = R.sandwich_backward(x["f"], to_host(y), x["gate"], x["gy"], x["gn"], w, 1e-5)
    for n, t in (("df", df), ("dx", dx), ("dgate", dgate)):
        _close(n, t, ref[n], dtype, (C, C))
    for n in w:
        _close(n, grads[n], ref[n], "fp32", (C, C, N))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_sandwich_in_place_without_gy_of_no_rows_and_independent_rows(dtype):
    import torch
    from oracle import conditioned as R
    from paper_2602_04940_amd import SandwichNorm
    from paper_2602_04940_amd._lib import TS3Error
    N, C = 301, 96
    x, w = _sandwich(N, C, True, True, dtype, seed=2)
    d = {n: to_device(t, dtype) for n, t in x.items()}
    p = {n: to_device(t, "fp32") for n, t in w.items()}
    back = {n: t for n, t in p.items() if n != "beta_pre"}
    with SandwichNorm(C, dtype=dtype) as s:
        y, out = s.forward(d["f"], d["x"], gate=d["gate"], **p)
        there = d["x"].clone()
        y2, out2 = s.forward(d["f"], there, gate=d["gate"], y=there, **p)
        assert y2 is there and torch.equal(y, y2) and torch.equal(out, out2)
        first = s.backward(d["f"], y, d["gy"], gate=d["gate"], gn=d["gn"], **back)
        gy = d["gy"].clone()
        second = s.backward(d["f"], y, gy, gate=d["gate"], gn=d["gn"], dx=gy, **back)
        assert second[1] is gy and all(torch.equal(a, b) for a, b in zip(first[:3], second[:3]))
        assert all(torch.equal(first[3][n], second[3][n]) for n in first[3])
        df, dx, dgate, grads = s.backward(d["f"], y, None, gate=d["gate"], gn=d["gn"], **back)
        ref = R.sandwich_backward(x["f"], to_host(y), x["gate"], None, x["gn"], w, 1e-5)
        _close("df", df, ref["df"], dtype, (C, C))
        _close("dx", dx, ref["dx"], dtype, (C,))
        f = d["f"].clone()
        f[7] = math.nan
        y3, out3 = s.forward(f, d["x"], gate=d["gate"], **p)
        keep = torch.arange(N, device="cuda") != 7
        assert torch.equal(y3[keep], y[keep]) and torch.equal(out3[keep], out[keep]) and out3[7].isnan().all()
        none = torch.empty((0, C), device="cuda", dtype=f.dtype)
        assert s.forward(none, none, gate=none, **p)[0].shape == (0, C)
        grads = s.backward(none, none, none, gate=none, gn=none, **back)[3]
        assert all((t == 0).all() for t in grads.values())
        flat = torch.zeros(3 * N * C, device="cuda", dtype=f.dtype)
        part = flat[C:C + N * C].view(N, C)
        whole = flat[:N * C].view(N, C)
        for call in (lambda: s.forward(d["f"], whole, gate=d["gate"], y=part, **p),
                     lambda: s.forward(whole, d["x"], gate=d["gate"], y=whole, **p),
                     lambda: s.forward(d["f"], d["x"], gate=d["gate"], out=d["x"], **p),
                     lambda: s.forward(d["f"], d["x"], gate=whole, out=part, **p),
                     lambda: s.backward(d["f"], y, whole, gate=d["gate"], gn=d["gn"], dx=part, **back),
                     lambda: s.backward(d["f"], y, d["gy"], gate=d["gate"], gn=d["gn"], dx=y, **back)):
            with pytest.raises(TS3Error, match="overlap"):
                call()


# ------------------------------------------------------------------ orthogonalised updates

def _flat(shapes, dtype, seed, rank=None, scale=1.0):
    """Matrices one after another in one array."""
    rng = np.random.default_rng(seed)
    parts = []
    for s in shapes:
        if rank:
            t = rng.standard_normal((*s[:-1], rank)) @ rng.standard_normal((*s[:-2], rank, s[-1])) * 0.3
        else:
            t = rng.standard_normal(s)
        parts.append(_round(t * scale, dtype))
    flat = to_device(np.concatenate([p.reshape(-1) for p in parts]), dtype)
    at, views = 0, []
    for p in parts:
        views.append(flat[at:at + p.size].view(p.shape))
        at += p.size
    return parts, views, flat


def _frobenius(got, ref):
    return float(np.linalg.norm(got - ref) / max(np.linalg.norm(ref), 1e-300))


# Sides of one, around the padding of 64 and the tiles of 128, wide and tall, batches; products of
# several tiles of each size.
ORTH = [[(1, 1)], [(1, 300)], [(300, 1)], [(16, 16)], [(63, 65)], [(64, 128), (130, 64)], [(8, 32, 32), (3, 5, 7, 40)],
        [(129, 257), (257, 129), (65, 64)], [(200, 1000)], [(31, 31)] * 70, [(256, 1024)] * 40 + [(1024, 256), (100, 90)],
        [(640, 700), (12, 200, 130)]]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shapes", ORTH)
def test_orth_of_matrices_of_low_condition(shapes, dtype):
    """Random matrices twice as wide as tall or more keep their singular values together; squarer ones
    have small ones."""
    import torch
    from oracle import conditioned as R
    from paper_2602_04940_amd import Orthogonalizer
    banner(f"orth {len(shapes)} tensors, first {shapes[0]} {dtype}")
    parts, views, _ = _flat(shapes, dtype, 1, scale=1e-3)
    with Orthogonalizer() as orth:
        out = orth(views)
        torch.cuda.synchronize()
    worst = 0.0
    for p, t in zip(parts, out):
        assert t.shape == p.shape
        ref, got = R.orthogonalise(p), to_host(t)
        r, c = min(p.shape[-2:]), max(p.shape[-2:])
        delta = 2.0 ** -22 + math.sqrt(r + c) * U
        for g, e in zip(got.reshape(-1, *p.shape[-2:]), ref.reshape(-1, *p.shape[-2:])):
            bar = 16 * delta if c >= 2 * r else 6 * 3.4445 ** 5 * delta / np.linalg.norm(e)
            bar += 2.0 ** -8 if dtype == "bf16" else 0.0
            err = _frobenius(g, e)
            worst = max(worst, err / bar)
            assert err <= bar, (p.shape, err, bar)
    print(f"worst of the bars {worst:.3f}", flush=True)


@pytest.mark.parametrize("rank", [1, 3, 20])
@pytest.mark.parametrize("shape", [(100, 300), (300, 100), (64, 64)])
def test_orth_of_low_rank(shape, rank):
    """Directions that are not there stay out: errors there grow 3.45 times a step."""
    import torch
    from oracle import conditioned as R
    from paper_2602_04940_amd import Orthogonalizer
    parts, views, _ = _flat([shape], "fp32", 2, rank=rank)
    with Orthogonalizer() as orth:
        got = to_host(orth(views)[0])
    ref = R.orthogonalise(parts[0])
    bar = 6 * 3.4445 ** 5 * (2.0 ** -22 + math.sqrt(sum(shape)) * U) / np.linalg.norm(ref)
    err = _frobenius(got, ref)
    print(f"{err:.2e} (bar {bar:.2e})", flush=True)
    assert err <= bar


def test_orth_of_extreme_sizes_zeros_and_bad_values():
    """Elements whose squares leave float32, elements far smaller than the largest, zero matrices; an
    infinity or not-a-number stays in its matrix."""
    import torch
    from oracle import conditioned as R
    from paper_2602_04940_amd import Orthogonalizer
    rng = np.random.default_rng(3)
    base = rng.standard_normal((20, 90))
    spread = base.copy()
    spread[10:] *= 1e-6
    cases = [base * 1e30, base * 1e-25, spread, np.zeros((7, 9)), base, base]
    cases = [_round(c, "fp32") for c in cases]
    dev = [to_device(c, "fp32") for c in cases]
    dev[4][3, 5], dev[5][2, 2] = math.nan, math.inf
    with Orthogonalizer(eps=0.0) as orth:
        got = [to_host(t) for t in orth(dev)]
    delta = 2.0 ** -22 + math.sqrt(110) * U
    for i in (0, 1):
        assert _frobenius(got[i], R.orthogonalise(cases[i], eps=0.0)) <= 16 * delta
    ref = R.orthogonalise(spread, eps=0.0)
    assert np.linalg.norm(got[2] - ref) <= 6 * 3.4445 ** 5 * delta
    assert np.isnan(got[3]).all() and np.isnan(got[4]).any() and np.isnan(got[5]).any()
    with Orthogonalizer(steps=2, eps=1e-3) as orth:
        got = [to_host(t) for t in orth(dev[:4])]
    assert (got[3] == 0).all() and np.isfinite(got[0]).all()
    assert np.abs(got[1] - R.orthogonalise(cases[1], 2, 1e-3)).max() <= 16 * delta * np.abs(got[1]).max() + 2.0 ** -36 * 12
    for t in (got[0],):
        assert _frobenius(t, R.orthogonalise(cases[0], 2, 1e-3)) <= 16 * delta


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_orth_in_place_unaligned_and_beside_its_results(dtype):
    import torch
    from paper_2602_04940_amd import Orthogonalizer
    from paper_2602_04940_amd._lib import TS3Error
    shapes = [(33, 45), (2, 17, 9), (70, 31), (1, 1)]
    parts, views, flat = _flat(shapes, dtype, 4)
    guard = torch.full((flat.numel() + 2,), 7.0, device="cuda", dtype=flat.dtype)
    inner, at = [], 1
    for v in views:
        inner.append(guard[at:at + v.numel()].view(v.shape))
        at += v.numel()
    with Orthogonalizer() as orth:
        fresh = orth(views)
        assert orth(views, out=inner) is inner
        assert all(torch.equal(a, b) for a, b in zip(fresh, inner)) and guard[0] == 7 and guard[-1] == 7
        orth(views, out=views)
        assert all(torch.equal(a, b) for a, b in zip(fresh, views))
        assert orth([]) == [] and orth([torch.empty((0, 4), device="cuda")])[0].shape == (0, 4)
        with pytest.raises(TS3Error, match="overlap"):
            orth([views[0], views[0]], out=[views[0], views[0]])
        for bad in ([views[0].t()], [views[0][0]], [views[0].double()], [views[0].cpu()]):
            with pytest.raises(ValueError):
                orth(bad, out=bad)
        with pytest.raises(ValueError):
            orth([views[0]], out=[views[2]])


# ------------------------------------------------------------------ together

@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_on_another_stream_and_in_a_graph(dtype):
    """A step of all three, on a stream of its own and captured: replays with new inputs, with eager work of
    the same handles between them, give the eager results bit for bit."""
    import torch
    from paper_2602_04940_amd import CrossAttention, Orthogonalizer, SandwichNorm
    from paper_2602_04940_amd._lib import TS3Error
    tt = torch.float32 if dtype == "fp32" else torch.bfloat16
    N, S, H, HK, D = 3000, 150, 4, 2, 16
    C = H * D
    gen = torch.Generator(device="cuda").manual_seed(10)

    def fresh(*shape):
        return torch.randn(shape, generator=gen, device="cuda").to(tt)
    held = dict(q=fresh(1, N, H, D), kv=fresh(1, S, 2, HK, D), q1=fresh(1, 1, H, D), x=fresh(N, C), gate=fresh(N, C),
                g=fresh(N, C), w=fresh(C, 3 * C), u=fresh(3, D, D))
    p = {n: torch.rand(C, generator=gen, device="cuda") for n in ("gamma_post", "beta_post", "scale", "gamma_pre", "beta_pre")}
    lengths = torch.tensor([140], dtype=torch.int32, device="cuda")
    a, s, orth = CrossAttention(H, D, HK, dtype), SandwichNorm(C, dtype), Orthogonalizer()

    def step(h):
        k, v = h["kv"][:, :, 0], h["kv"][:, :, 1]
        out, lse = a.forward(h["q"], k, v, lengths=lengths)
        one, _ = a.forward(h["q1"], k, v, lengths=lengths)
        f = out.view(N, C)
        y, n = s.forward(f, h["x"], gate=h["gate"], **p)
        df, dx, dgate, grads = s.backward(f, y, h["g"], p["gamma_post"], p["beta_post"], p["scale"], gate=h["gate"], gn=n,
                                          gamma_pre=p["gamma_pre"])
        dq, dk, dv = a.backward(h["q"], k, v, out, lse, df.view(1, N, H, D), lengths=lengths)
        return [out, lse, one, y, n, df, dx, dgate, dq, dk, dv, *grads.values(), *orth([h["w"], h["u"]])]
    ref = step(held)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step(held)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(ref, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(held)
        with pytest.raises(TS3Error, match="make the call once before"):
            orth([torch.zeros((2000, 2000), device="cuda")])
    big = fresh(1, 1, H, D), fresh(1, 40_000, HK, D)
    for i in range(4):
        for t in held.values():
            t.copy_(fresh(*t.shape))
        # larger eager calls of the same handles between the replays: the graph's workspaces stay
        a.forward(big[0], big[1], big[1])
        orth([fresh(500 + 100 * i, 700)])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(step(held), captured)), i
    for h in (a, s, orth):
        h.close()
