"""The training operators on the GPU against the float64 reference: every type, ragged
lengths and widths, what a row of NaN reaches, empty calls, repeats, refusals, streams
and captured graphs.

Bars, fixed before the first run.  Float32: each output is a sum of K products of operands
carried to 2^-24; roundings of such a sum walk about sqrt(K) 2^-24 of the largest value, and
the bar is four such walks over every sum on the way (C, F, and N for what is summed over
points), plus 8 for the elementwise steps; relative to the output's largest value.
BFloat16: an output is rounded once (2^-9 at most, 2^-9/sqrt 3 in the mean square), and so is
each hidden value that it is a sum of; the bar is 2^-8 in the mean square over the array, and
2e-2 per row, the bar of the other bf16 tests."""
import math

import numpy as np
import pytest

from gated_shapes import LONG, MIDDLE
from gpu_helpers import banner, normwise, rel_l2, row_rel, to_device, to_host

pytestmark = pytest.mark.gpu

NAMES = ("dWg", "dWu", "dWd", "dbg", "dbu", "dbd")


def _round(a, dtype):
    """float64 values that the storage type holds exactly"""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32))
    return (t.bfloat16() if dtype == "bf16" else t).double().numpy()


def _check(name, got, ref, dtype, K):
    if ref.size == 0:
        return
    got = to_host(got)
    assert got.shape == ref.shape, name
    assert np.isfinite(got).all(), name
    if dtype == "fp32":
        err, bar = normwise(got, ref), 4 * 2.0 ** -24 * (8 + sum(math.sqrt(k) for k in K))
        print(f"{name}: normwise {err:.2e} (bar {bar:.2e})", flush=True)
        assert err <= bar, name
    else:
        err, row = rel_l2(got, ref), row_rel(got.reshape(len(got), -1), ref.reshape(len(ref), -1)) if ref.ndim == 2 else 0.0
        print(f"{name}: rel L2 {err:.2e}, worst row {row:.2e}", flush=True)
        assert err <= 2.0 ** -8 and row <= 2e-2, name


def _gated(n, C, F, dtype, bias, seed=0, scale=1.0):
    rng = np.random.default_rng([seed, n, C, F])
    bound = math.sqrt(6.0 / (C + F))
    w = {"Wg": rng.uniform(-bound, bound, (C, F)), "Wu": rng.uniform(-bound, bound, (C, F)),
         "Wd": rng.uniform(-bound, bound, (F, C))}
    if bias:
        w.update(bg=rng.uniform(-0.5, 0.5, F), bu=rng.uniform(-0.5, 0.5, F), bd=rng.uniform(-0.5, 0.5, C))
    w = {k: _round(v, dtype) for k, v in w.items()}
    return (_round(rng.standard_normal((n, C)) * scale, dtype), w, _round(rng.standard_normal((n, C)), dtype))


def _operator(C, F, kind, dtype, w):
    from paper_2602_04940_amd import GatedFeedForward, GatedWeights
    ff = GatedFeedForward(C, F, activation=kind, dtype=dtype)
    ff.load(GatedWeights({k: to_device(v, dtype) for k, v in w.items()}, dtype))
    return ff


# (N, C, F, tile): one point to a few rounds of workgroups; every padded width, exactly and
# not; hidden widths of one unit, around a chunk of 32 and of several blocks; tiles of the
# backward that end inside a workgroup.
SHAPES = [(1, 256, 1024, 1000), (1, 16, 1, 1), (2, 48, 33, 1000), (31, 64, 32, 1000), (33, 80, 100, 16), (127, 128, 341, 1000),
          (128, 128, 512, 128), (129, 144, 31, 100), (1000, 192, 257, 384), (1003, 208, 65, 1000), (2500, 256, 96, 1024),
          (4097, 112, 700, 5000), (40_001, 128, 64, 16_384), (40_001, 256, 40, 1 << 18)]


@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("N,C,F,tile", SHAPES)
def test_gated_forward_and_backward(N, C, F, tile, dtype, kind):
    import torch
    from oracle import train as T
    bias = (N + F) % 2 == 0
    banner(f"gated N={N} C={C} F={F} {dtype} {kind} tile={tile} bias={bias}")
    x, w, g = _gated(N, C, F, dtype, bias)
    with _operator(C, F, kind, dtype, w) as ff:
        xt, gt = to_device(x, dtype), to_device(g, dtype)
        out = ff.forward(xt)
        dx, grads = ff.backward(xt, gt, tile=tile)
        torch.cuda.synchronize()
    _check("out", out, T.gated_forward(x, w, kind), dtype, (C, F))
    ref = T.gated_backward(x, w, kind, g)
    _check("dx", dx, ref["dx"], dtype, (C, F))
    for n in NAMES:
        _check(n, grads[n], ref[n], dtype, (C, F, N))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_gated_gradient_against_differences(dtype):
    """d/dt of sum(g * out(x + t v, W + t V)) against the gradients' products with v and V.
    The forward is float64 from the reference: its central difference of step 1e-4 is good to
    about 1e-7 of the derivative's terms, the operator's gradients to its own bars."""
    import torch
    from oracle import train as T
    N, C, F, t = 700, 96, 130, 1e-4
    x, w, g = _gated(N, C, F, dtype, True, seed=5)
    rng = np.random.default_rng(9)
    v, V = rng.standard_normal(x.shape), {k: rng.standard_normal(a.shape) * 0.1 for k, a in w.items()}
    with _operator(C, F, "gelu", dtype, w) as ff:
        dx, grads = ff.backward(to_device(x, dtype), to_device(g, dtype), tile=256)
        torch.cuda.synchronize()

    def loss(s):
        return (g * T.gated_forward(x + s * v, {k: a + s * V[k] for k, a in w.items()}, "gelu")).sum()
    fd = (loss(t) - loss(-t)) / (2 * t)
    terms = [(to_host(dx) * v).sum()] + [(to_host(grads["d" + k]) * V[k]).sum() for k in w]
    size = math.sqrt((to_host(dx) ** 2).sum() + sum((to_host(grads["d" + k]) ** 2).sum() * 0.01 for k in w))
    err = abs(sum(terms) - fd) / size
    print(f"differences {fd:.6e}, gradients {sum(terms):.6e}, of the gradients' norm {err:.1e}", flush=True)
    assert err <= (1e-5 if dtype == "fp32" else 2.0 ** -7)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_gated_gates_far_from_zero(kind, dtype):
    """Gates of hundreds: the exponentials overflow and vanish, the outputs do not."""
    import torch
    from oracle import train as T
    N, C, F = 300, 64, 96
    x, w, g = _gated(N, C, F, dtype, True, seed=2, scale=300.0)
    with _operator(C, F, kind, dtype, w) as ff:
        xt, gt = to_device(x, dtype), to_device(g, dtype)
        out = ff.forward(xt)
        dx, grads = ff.backward(xt, gt)
        torch.cuda.synchronize()
    _check("out", out, T.gated_forward(x, w, kind), dtype, (C, F))
    ref = T.gated_backward(x, w, kind, g)
    _check("dx", dx, ref["dx"], dtype, (C, F))
    for n in NAMES:
        _check(n, grads[n], ref[n], dtype, (C, F, N))


# Padded widths of every kernel, one point to several tiles, hidden widths around a chunk.
@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("N,C,F,tile", [(1, 64, 32, 1000), (70, 48, 33, 64), (3001, 128, 300, 1024), (300, 192, 31, 1000),
                                        (5003, 256, 100, 2048)])
def test_gated_bf16_bias_gradients_round_once(N, C, F, tile, kind):
    """dbg, dbu and dbd are sums of float32 values, rounded to bfloat16 once: within 2^-8 of each
    value, plus what float32 sums and exponentials good to some 2^-21 leave of the largest."""
    import torch
    from oracle import train as T
    x, w, g = _gated(N, C, F, "bf16", True, seed=6)
    with _operator(C, F, kind, "bf16", w) as ff:
        _, grads = ff.backward(to_device(x, "bf16"), to_device(g, "bf16"), tile=tile)
        torch.cuda.synchronize()
    ref = T.gated_backward(x, w, kind, g)
    for n in ("dbg", "dbu", "dbd"):
        err = np.abs(to_host(grads[n]) - ref[n])
        assert (err <= 2.0 ** -8 * np.abs(ref[n]) + 2.0 ** -16 * np.abs(ref[n]).max()).all(), n


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("gate", [-3.0, -4.0, -5.0])
def test_gated_gates_that_are_nearly_closed(gate, kind, dtype):
    """Every gate far down its tail: the outputs are small, and as exact relative to themselves."""
    import torch
    from oracle import train as T
    N, C, F = 200, 96, 70
    x, w, _ = _gated(N, C, F, dtype, True, seed=7, scale=0.05)
    w["bg"], w["bd"] = np.full(F, gate), np.zeros(C)
    with _operator(C, F, kind, dtype, w) as ff:
        out = ff.forward(to_device(x, dtype))
        torch.cuda.synchronize()
    _check("out", out, T.gated_forward(x, w, kind), dtype, (C, F))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("gate", [-5.5, -6.0, -7.0, -8.0, -10.0])
def test_gated_gates_far_down_the_tail(gate, kind, dtype):
    """As above, further down, and every gradient.  A relative change of a by d changes GELU and its
    slope by about a^2 d of themselves, so float32's walk of the sums over C counts a^2 times; in
    bfloat16 that is still far below a rounding."""
    import torch
    from oracle import train as T
    N, C, F = 200, 96, 70
    x, w, g = _gated(N, C, F, dtype, True, seed=7, scale=0.05)
    w["bg"], w["bd"] = np.full(F, gate), np.zeros(C)
    with _operator(C, F, kind, dtype, w) as ff:
        xt = to_device(x, dtype)
        out = ff.forward(xt)
        dx, grads = ff.backward(xt, to_device(g, dtype))
        torch.cuda.synchronize()
    _check("out", out, T.gated_forward(x, w, kind), dtype, (C * gate ** 4, F))
    ref = T.gated_backward(x, w, kind, g)
    _check("dx", dx, ref["dx"], dtype, (C * gate ** 4, F))
    for n in NAMES:
        _check(n, grads[n], ref[n], dtype, (C * gate ** 4, F, N))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("N", [5, 300, 50_000])
def test_gated_rows_are_independent(N, dtype):
    """A row of NaN and one of infinities stay where they are, also at the end of the call."""
    import torch
    C, F = 112, 200
    x, w, _ = _gated(N, C, F, dtype, False, seed=3)
    bad = sorted({0, N // 2, N - 1})
    with _operator(C, F, "silu", dtype, w) as ff:
        xt = to_device(x, dtype)
        clean = ff.forward(xt)
        xt[bad[0]], xt[bad[1]], xt[bad[2], 3] = float("nan"), float("inf"), float("nan")
        out = ff.forward(xt)
        torch.cuda.synchronize()
    keep = torch.ones(N, dtype=torch.bool, device="cuda")
    keep[bad] = False
    assert torch.equal(out[keep], clean[keep])
    assert out[bad].isnan().any(1).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_gated_repeats_bitwise_in_place_and_reloaded(dtype):
    import torch
    C, F, N = 176, 300, 5000
    x, w, g = _gated(N, C, F, dtype, True, seed=4)
    _, w2, _ = _gated(N, C, F, dtype, False, seed=44)
    with _operator(C, F, "silu", dtype, w) as ff:
        from paper_2602_04940_amd import GatedWeights
        xt, gt = to_device(x, dtype), to_device(g, dtype)
        out = ff.forward(xt)
        dx, grads = ff.backward(xt, gt, tile=2048)
        ff.load(GatedWeights({k: to_device(v, dtype) for k, v in w2.items()}, dtype))
        other = ff.forward(xt)
        ff.load(GatedWeights({k: to_device(v, dtype) for k, v in w.items()}, dtype))
        again = ff.forward(xt)
        dx2, grads2 = ff.backward(xt, gt, tile=2048)
        place = xt.clone()
        ff.forward(place, out=place)
        torch.cuda.synchronize()
    assert torch.equal(out, again) and torch.equal(out, place) and not torch.equal(out, other)
    assert torch.equal(dx, dx2) and all(torch.equal(grads[n], grads2[n]) for n in NAMES)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_gated_of_no_points(dtype):
    import torch
    C, F = 64, 70
    _, w, _ = _gated(1, C, F, dtype, True)
    with _operator(C, F, "gelu", dtype, w) as ff:
        x = torch.empty((0, C), device="cuda", dtype=ff.torch_dtype)
        assert ff.forward(x).shape == (0, C)
        dx, grads = ff.backward(x, x)
        torch.cuda.synchronize()
        assert dx.shape == (0, C) and all((grads[n] == 0).all() for n in NAMES)


def test_gated_refusals():
    import torch
    from paper_2602_04940_amd import GatedFeedForward, GatedWeights
    from paper_2602_04940_amd import _lib as L
    C, F = 64, 48
    x, w, g = _gated(10, C, F, "bf16", True)
    xt, gt = to_device(x, "bf16"), to_device(g, "bf16")
    with GatedFeedForward(C, F) as ff:
        with pytest.raises(L.TS3Error) as e:
            ff.forward(xt)
        assert e.value.status == L.TS3_ERR_BAD_STATE
        with pytest.raises(L.TS3Error) as e:
            ff.backward(xt, gt)
        assert e.value.status == L.TS3_ERR_BAD_STATE
        weights = {k: to_device(v, "bf16") for k, v in w.items()}
        with pytest.raises(ValueError, match="weights of"):
            ff.load(GatedWeights(weights, "fp32"))
        ff.load(GatedWeights(weights, "bf16"))
        for bad in (xt.float(), xt[:, :32], xt.t().contiguous().t(), xt.cpu(), xt[0]):
            with pytest.raises(ValueError, match="contiguous cuda"):
                ff.forward(bad)
        with pytest.raises(ValueError, match="g must be"):
            ff.backward(xt, gt[:9])
        for kw in (dict(tile=0), dict(dx=xt), dict(dx=gt)):
            with pytest.raises(L.TS3Error) as e:
                ff.backward(xt, gt, **kw)
            assert e.value.status == L.TS3_ERR_INVALID_ARG
        lib = L.lib()
        odd = xt.data_ptr() + 2
        assert lib.ts3_gated_forward(ff.h, odd, 4, gt.data_ptr(), None) == L.TS3_ERR_INVALID_ARG
        assert lib.ts3_gated_forward(ff.h, xt.data_ptr(), -1, gt.data_ptr(), None) == L.TS3_ERR_INVALID_ARG
        assert lib.ts3_gated_forward(ff.h, xt.data_ptr(), 4, None, None) == L.TS3_ERR_INVALID_ARG
        torch.cuda.synchronize()


NORM_CASES = [(1, 16), (2, 512), (3, 48), (63, 32), (65, 80), (1000, 64), (1003, 128), (257, 240), (300, 256), (129, 272),
              (5003, 496), (70_001, 96)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("N,C", NORM_CASES)
def test_norm_forward_and_backward(N, C, residual, dtype):
    import torch
    from oracle import train as T
    from paper_2602_04940_amd import ResidualNorm
    banner(f"norm N={N} C={C} {dtype} residual={residual}")
    rng = np.random.default_rng([N, C])
    x, r, g, gr = (_round(a, dtype) for a in rng.standard_normal((4, N, C)))
    r, gr = (r, gr) if residual else (None, None)
    gamma, beta = _round(1 + rng.uniform(-0.5, 0.5, C), "fp32"), _round(rng.uniform(-1, 1, C), "fp32")
    y, out = T.norm_forward(x, r, gamma, beta, 1e-5)
    dev = {k: None if a is None else to_device(a, dtype) for k, a in dict(x=x, r=r, g=g, gr=gr, y=_round(y, dtype)).items()}
    gm, bt = to_device(gamma, "fp32"), to_device(beta, "fp32")
    with ResidualNorm(C, dtype) as norm:
        yt, ot = norm.forward(dev["x"], gm, bt, residual=dev["r"])
        dx, dgamma, dbeta = norm.backward(dev["y"], dev["g"], gm, residual_grad=dev["gr"])
        dx2, dgamma2, dbeta2 = norm.backward(dev["y"], dev["g"], gm, residual_grad=dev["gr"], dx=dev["g"].clone())
        place = dev["x"].clone()
        norm.forward(place, gm, bt, residual=dev["r"], y=place)
        torch.cuda.synchronize()
    _check("y", yt, y, dtype, (1,))
    _check("out", ot, out, dtype, (C, C))
    rx, rg, rb = T.norm_backward(_round(y, dtype), g, gr, gamma, 1e-5)
    _check("dx", dx, rx, dtype, (C, C))
    _check("dgamma", dgamma, rg, "fp32", (C, N))
    _check("dbeta", dbeta, rb, "fp32", (N,))
    assert torch.equal(dx, dx2) and torch.equal(dgamma, dgamma2) and torch.equal(dbeta, dbeta2)
    assert torch.equal(place, yt)


def test_norm_of_rows_far_from_zero_and_of_equal_values():
    """A mean of 4,096 beside a spread of one costs 12 bits of each value, no more (the variance
    is taken about the mean); a constant row gives beta; the gradient's rows are finite."""
    import torch
    from oracle import train as T
    from paper_2602_04940_amd import ResidualNorm
    N, C = 100, 160
    rng = np.random.default_rng(0)
    x = _round(rng.standard_normal((N, C)) + 4096.0, "fp32")
    x[50] = 3.0
    g = _round(rng.standard_normal((N, C)), "fp32")
    gamma, beta = np.ones(C), _round(rng.standard_normal(C), "fp32")
    with ResidualNorm(C, "fp32") as norm:
        y, out = norm.forward(to_device(x, "fp32"), to_device(gamma, "fp32"), to_device(beta, "fp32"))
        dx, _, _ = norm.backward(y, to_device(g, "fp32"), to_device(gamma, "fp32"))
        torch.cuda.synchronize()
    _, ref = T.norm_forward(x, None, gamma, beta, 1e-5)
    # the mean's rounding: 2^-24 of 4,096 times a few lane sums, sqrt(C) walks of it
    assert np.abs(to_host(out) - ref).max() <= 4096 * 2.0 ** -24 * (8 + math.sqrt(C))
    assert np.array_equal(to_host(out)[50], beta)
    assert np.isfinite(to_host(dx)).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_norm_of_no_rows_and_refusals(dtype):
    import torch
    from paper_2602_04940_amd import ResidualNorm
    from paper_2602_04940_amd import _lib as L
    C = 48
    gm = torch.ones(C, device="cuda")
    with ResidualNorm(C, dtype) as norm:
        e = torch.empty((0, C), device="cuda", dtype=norm.torch_dtype)
        y, out = norm.forward(e, gm, gm)
        dx, dgamma, dbeta = norm.backward(e, e, gm)
        torch.cuda.synchronize()
        assert out.shape == dx.shape == (0, C) and (dgamma == 0).all() and (dbeta == 0).all()
        x = torch.ones((4, C), device="cuda", dtype=norm.torch_dtype)
        for bad in (x[:, :32], x.double(), x.cpu()):
            with pytest.raises(ValueError, match="contiguous cuda"):
                norm.forward(bad, gm, gm)
        with pytest.raises(ValueError, match="gamma must be"):
            norm.forward(x, gm.bfloat16(), gm)
        with pytest.raises(ValueError, match="residual must be"):
            norm.forward(x, gm, gm, residual=x[:3])
        for call in (lambda: norm.forward(x, gm, gm, out=x), lambda: norm.backward(x, x.clone(), gm, dx=x)):
            with pytest.raises(L.TS3Error) as err:
                call()
            assert err.value.status == L.TS3_ERR_INVALID_ARG


def _clip_case(sizes, seed, scale=1.0, gap=0):
    """Tensors of alternating type in one buffer each, `gap` elements apart (an odd gap leaves
    them off the 16-byte boundaries)."""
    import torch
    rng = np.random.default_rng(seed)
    grads = []
    for dtype in (torch.float32, torch.bfloat16):
        mine = [s for i, s in enumerate(sizes) if i % 2 == (dtype == torch.bfloat16)]
        buf = torch.zeros(sum(mine) + gap * (len(mine) + 1), device="cuda", dtype=dtype)
        at = gap
        for s in mine:
            buf[at:at + s] = torch.from_numpy((rng.standard_normal(s) * scale).astype(np.float32)).to(buf)
            grads.append(buf[at:at + s])
            at += s + gap
    return grads


CLIP_SIZES = [[1], [0, 0, 5], [7, 8, 9, 0, 15, 16, 17], [8191, 8192, 8193, 100_003], [3] * 301, [2_000_001, 64]]


@pytest.mark.parametrize("gap", [0, 1, 8])
@pytest.mark.parametrize("sizes", CLIP_SIZES)
@pytest.mark.parametrize("place", [True, False])
def test_clip(sizes, gap, place):
    import torch
    from oracle import train as T
    from paper_2602_04940_amd import GradClip
    grads = _clip_case(sizes, len(sizes), gap=gap)
    ref_in = [to_host(g) for g in grads]
    ref_norm = T.clip(ref_in, 1.0)[0]
    for max_norm in (0.25 * ref_norm, 4.0 * ref_norm, float("inf")):
        work = [g.clone() for g in grads] if place else grads
        if place and gap == 0 and max_norm < ref_norm:
            work = _clip_case(sizes, len(sizes))  # still one after another in memory
        out = work if place else [torch.full_like(g, 7.0) for g in grads]
        with GradClip() as clip:
            norm = clip(work, max_norm, out=None if place else out)
            torch.cuda.synchronize()
        _, ref = T.clip(ref_in, max_norm)
        # float64 sums, one rounding; the scale and the product round once each
        assert abs(float(norm) - ref_norm) <= 2.0 ** -23 * ref_norm
        for g, o, r in zip(grads, out, ref):
            tol = 2.0 ** -22 if g.dtype == torch.float32 else 2.0 ** -8
            assert np.abs(to_host(o) - r).max(initial=0.0) <= tol * np.abs(r).max(initial=0.0)
            if max_norm > ref_norm:
                assert torch.equal(o, g)


def test_clip_touches_nothing_between_the_tensors():
    import torch
    from paper_2602_04940_amd import GradClip
    buf = torch.full((1000,), 2.0, device="cuda")
    with GradClip() as clip:
        clip([buf[1:18], buf[100:133], buf[501:502]], 1.0)
        torch.cuda.synchronize()
    scaled = torch.zeros(1000, dtype=torch.bool)
    scaled[1:18] = scaled[100:133] = scaled[501:502] = True
    assert (buf.cpu()[~scaled] == 2.0).all() and (buf.cpu()[scaled] < 1.0).all()


def test_clip_values_whose_squares_leave_float32_and_bad_norms():
    import torch
    from paper_2602_04940_amd import GradClip
    from paper_2602_04940_amd import _lib as L
    with GradClip() as clip:
        for v in (1e30, 1e-30):
            g = torch.full((1000,), v, device="cuda")
            norm = float(clip([g], v))
            assert abs(norm / (v * math.sqrt(1000)) - 1) < 1e-6
            assert abs(float(g.double().norm()) / v - 1) < 1e-6
        assert float(clip([], 1.0)) == 0.0
        g = torch.ones(10, device="cuda")
        g[3] = float("inf")
        assert float(clip([g], 1.0)) == float("inf")
        assert g[3].isnan() and (g[[0, 9]] == 0).all()
        g = torch.ones(10, device="cuda")
        g[3] = float("nan")
        assert math.isnan(float(clip([g], 0.5)))
        assert (g[[0, 9]] == 1).all()
        g = torch.ones((4, 6), device="cuda")
        for bad in (0.0, -1.0, float("nan")):
            with pytest.raises(L.TS3Error) as e:
                clip([g], bad)
            assert e.value.status == L.TS3_ERR_INVALID_ARG
        for bad, out in (([g.t()], None), ([g.double()], None), ([g.cpu()], None), ([g], []), ([g], [g.bfloat16()]),
                         ([g], [g[:2]])):
            with pytest.raises(ValueError):
                clip(bad, 1.0, out=out)
        torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_on_another_stream_and_in_a_graph(dtype):
    """All three operators on a side stream, then captured and replayed with the program's own
    work and other inputs between the replays: each equals the eager result bitwise."""
    import torch
    from paper_2602_04940_amd import GradClip, ResidualNorm
    C, F = 96, 130
    _, w, _ = _gated(1, C, F, dtype, True)
    with _operator(C, F, "silu", dtype, w) as ff, ResidualNorm(C, dtype) as norm, GradClip() as clip:
        gm, bt = torch.linspace(0.5, 1.5, C, device="cuda"), torch.linspace(-1, 1, C, device="cuda")
        for n in (3, 2100):
            x = torch.zeros((n, C), device="cuda", dtype=ff.torch_dtype)
            g = torch.zeros_like(x)

            def step():
                y, h = norm.forward(x, gm, bt, residual=g)
                out = ff.forward(h)
                dh, grads = ff.backward(h, g, tile=1000)
                dx, dgamma, dbeta = norm.backward(y, dh, gm, residual_grad=g)
                total = clip(list(grads.values()) + [dgamma, dbeta], 0.01)
                return [y, out, dx, dgamma, dbeta, total] + list(grads.values())

            def fill(seed):
                gen = torch.Generator(device="cuda").manual_seed(seed)
                x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
                g.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
            fill(0)
            eager = [t.clone() for t in step()]
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                on_side = step()
            torch.cuda.current_stream().wait_stream(side)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(eager, on_side))
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                captured = step()
            for seed in (1, 2, 3):
                fill(seed)
                eager = [t.clone() for t in step()]
                torch.cuda.synchronize()
                graph.replay()
                torch.cuda.synchronize()
                for i, (a, b) in enumerate(zip(eager, captured)):
                    assert torch.equal(a, b), (n, seed, i)


@pytest.mark.parametrize("dtype,C", [("fp32", 96), ("bf16", 96), ("bf16", 256)])
def test_graphs_outlive_a_larger_call(dtype, C):
    """The store that a captured backward uses is kept when a later call grows past it: the first
    graph's replays, after two larger calls, still give the eager result."""
    import torch
    F = 130
    _, w, _ = _gated(1, C, F, dtype, True)
    with _operator(C, F, "silu", dtype, w) as ff:
        def inputs(n):
            return [torch.zeros((n, C), device="cuda", dtype=ff.torch_dtype) for _ in range(2)]

        def fill(tensors, seed):
            gen = torch.Generator(device="cuda").manual_seed(seed)
            for t in tensors:
                t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
        small, middle, large = inputs(300), inputs(3000), inputs(9000)
        for t in (small, middle, large):
            fill(t, 0)
        ff.backward(*small)
        first = ff.bytes()
        ff.backward(*middle)
        grown = ff.bytes()
        element = 2 if dtype == "bf16" else 4
        assert grown - first >= 2000 * 3 * F * element
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            dx, grads = ff.backward(*middle)
        ff.backward(*large)
        # the captured store and the larger one beside it
        assert ff.bytes() - grown >= 9000 * 3 * F * element
        for seed in (1, 2, 3):
            fill(middle, seed)
            fill(large, seed)
            edx, egrads = ff.backward(*middle)
            ff.backward(*large)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(dx, edx) and all(torch.equal(grads[n], egrads[n]) for n in NAMES), seed


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_capture_that_would_allocate_is_refused(dtype):
    import torch
    from paper_2602_04940_amd import _lib as L
    C, F, N = 64, 70, 500
    x, w, g = _gated(N, C, F, dtype, True)
    with _operator(C, F, "gelu", dtype, w) as ff:
        xt, gt = to_device(x, dtype), to_device(g, dtype)
        for ready in (0, 100):  # no call before, and one of fewer points
            if ready:
                ff.backward(xt[:ready], gt[:ready])
            held = ff.bytes()
            out = torch.empty_like(xt)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                with pytest.raises(L.TS3Error) as e:
                    ff.backward(xt, gt)
                ff.forward(xt, out=out)  # the capture goes on
            assert e.value.status == L.TS3_ERR_BAD_STATE and ff.bytes() == held
            graph.replay()
            assert torch.equal(out, ff.forward(xt))
        dx, grads = ff.backward(xt, gt)
        dx2, grads2 = ff.backward(xt, gt)
        torch.cuda.synchronize()
        assert torch.equal(dx, dx2) and all(torch.equal(grads[n], grads2[n]) for n in NAMES)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_arrays_that_overlap_in_part_are_refused(dtype):
    """Rows that one workgroup writes while another still reads them: out and dx shifted by a row
    against their inputs either way, and by their last row alone; gradients on top of each other."""
    import torch
    from paper_2602_04940_amd import ResidualNorm
    from paper_2602_04940_amd import _lib as L
    C, F, N = 64, 48, 300
    _, w, _ = _gated(1, C, F, dtype, True)
    with _operator(C, F, "silu", dtype, w) as ff, ResidualNorm(C, dtype) as norm:
        buf = torch.zeros((3 * N, C), device="cuda", dtype=ff.torch_dtype)
        x, far = buf[100:100 + N], torch.zeros((N, C), device="cuda", dtype=ff.torch_dtype)
        gm = torch.ones(C, device="cuda")

        def refused(call):
            with pytest.raises(L.TS3Error) as e:
                call()
            assert e.value.status == L.TS3_ERR_INVALID_ARG
        for at in (99, 101, 100 + N - 1):
            other = buf[at:at + N]
            for call in (lambda: ff.forward(x, out=other), lambda: ff.backward(x, far, dx=other),
                         lambda: ff.backward(far, x, dx=other), lambda: norm.forward(x, gm, gm, y=other),
                         lambda: norm.forward(far, gm, gm, residual=x, y=other), lambda: norm.forward(x, gm, gm, out=other),
                         lambda: norm.forward(far, gm, gm, residual=x, out=other),
                         lambda: norm.forward(far, gm, gm, y=x, out=other), lambda: norm.backward(x, far, gm, dx=other),
                         lambda: norm.backward(far, x, gm, dx=other),
                         lambda: norm.backward(far, far.clone(), gm, residual_grad=x, dx=other)):
                refused(call)
        # next to each other is not on top of each other
        ff.forward(buf[:N], out=buf[N:2 * N])
        norm.forward(buf[:N], gm, gm, out=buf[N:2 * N])
        norm.backward(buf[:N], far, gm, dx=buf[N:2 * N])
        # C calls: gradients that share their last and first bytes, parameters below the rows
        lib, stream = L.lib(), None
        flat = torch.zeros(8 * C * F, device="cuda", dtype=ff.torch_dtype)
        e = flat.element_size()
        sizes = dict(dWg=C * F, dWu=C * F, dWd=C * F, dbg=F, dbu=F, dbd=C)
        names, at, ptrs = list(sizes), flat.data_ptr(), {}
        for k in names:
            ptrs[k] = at
            at += sizes[k] * e
        dx = torch.empty_like(far)
        held = dx.nbytes
        for a, b in [(i, j) for i in names for j in names if i < j]:
            grads = L.GatedGrads(**{**ptrs, b: ptrs[a] + (sizes[a] - 1) * e})
            assert lib.ts3_gated_backward(ff.h, x.data_ptr(), far.data_ptr(), N, N, dx.data_ptr(), L.ct.byref(grads),
                                          stream) == L.TS3_ERR_INVALID_ARG, (a, b)
        for k in names:
            grads = L.GatedGrads(**{**ptrs, k: dx.data_ptr() + held - e})
            assert lib.ts3_gated_backward(ff.h, x.data_ptr(), far.data_ptr(), N, N, dx.data_ptr(), L.ct.byref(grads),
                                          stream) == L.TS3_ERR_INVALID_ARG, k
        params = torch.zeros((3, C), device="cuda")
        p = params.data_ptr()
        row = 4 * C
        for dgamma, dbeta in ((p, p + row - 4), (dx.data_ptr(), p), (p, dx.data_ptr() + held - 4)):
            assert lib.ts3_norm_backward(norm.h, x.data_ptr(), far.data_ptr(), None, gm.data_ptr(), N, dx.data_ptr(), dgamma,
                                         dbeta, stream) == L.TS3_ERR_INVALID_ARG
        for gamma, beta in ((dx.data_ptr(), p), (p, dx.data_ptr() + held - 4)):
            assert lib.ts3_norm_forward(norm.h, x.data_ptr(), None, gamma, beta, N, None, dx.data_ptr(),
                                        stream) == L.TS3_ERR_INVALID_ARG
        torch.cuda.synchronize()


def test_clip_refuses_tensors_that_overlap():
    """What is written may be no other tensor's: the same one twice, views of one buffer, a
    destination on another's source or a few elements off its own, in whatever order they come."""
    import torch
    from paper_2602_04940_amd import GradClip
    from paper_2602_04940_amd import _lib as L
    buf, other = torch.ones(1000, device="cuda"), torch.ones(1000, device="cuda")
    halves = buf.view(torch.bfloat16)
    with GradClip() as clip:
        for grads, out in (([buf, other, buf], None), ([buf[:500], other, buf[499:]], None), ([buf[499:], buf[:500]], None),
                           ([buf, buf[10:20]], None), ([buf[10:20], other, buf], None), ([buf[:100], halves[199:300]], None),
                           ([buf[:900]], [buf[100:]]), ([buf[100:]], [buf[:900]]), ([buf, other], [other, buf]),
                           ([buf[:500], buf[500:]], [other[:500], buf[:500]]), ([buf, other[:10]], [other, torch.zeros(10, device="cuda")]),
                           ([buf[:10], buf[20:30]], [other[:10], other[9:19]])):
            with pytest.raises(L.TS3Error) as e:
                clip(grads, 1.0, out=out)
            assert e.value.status == L.TS3_ERR_INVALID_ARG
        torch.cuda.synchronize()
        assert (buf == 1).all() and (other == 1).all()
        # not on top of each other; the same source read twice; measured only
        clip([buf[500:], other, buf[:500]], 1e9)
        outs = [torch.empty_like(buf) for _ in range(2)]
        assert abs(float(clip([buf, buf], 1.0, out=outs)) - math.sqrt(2000)) < 1e-4
        assert torch.equal(outs[0], outs[1]) and float(outs[0][0]) < 0.03
        assert abs(float(clip([buf, buf], float("inf"))) - math.sqrt(2000)) < 1e-4
        torch.cuda.synchronize()
        assert (buf == 1).all()


def test_clip_of_many_separate_tensors():
    """Separate allocations in an order that is not that of their addresses, in place: several
    launches' worth, as a program's own list of gradients is."""
    import torch
    from oracle import train as T
    from paper_2602_04940_amd import GradClip
    rng = np.random.default_rng(11)
    tensors = [torch.from_numpy(rng.standard_normal(int(n)).astype(np.float32)).to("cuda", torch.bfloat16 if i % 3 else torch.float32)
               for i, n in enumerate(rng.integers(1, 5000, 300))]
    grads = [tensors[i] for i in rng.permutation(len(tensors))]
    ref_norm, ref = T.clip([to_host(t) for t in grads], 2.0)
    with GradClip() as clip:
        norm = clip(grads, 2.0)
        torch.cuda.synchronize()
    assert abs(float(norm) - ref_norm) <= 2.0 ** -23 * ref_norm
    for t, r in zip(grads, ref):
        tol = 2.0 ** -22 if t.dtype == torch.float32 else 2.0 ** -8
        assert np.abs(to_host(t) - r).max() <= tol * np.abs(r).max()


@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("N,C,F,tile", LONG)
def test_gated_long_loops(N, C, F, tile, dtype, kind):
    test_gated_forward_and_backward(N, C, F, tile, dtype, kind)


@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("N,C,F", MIDDLE)
def test_gated_forward_of_a_workgroup_per_compute_unit(N, C, F, dtype, kind):
    import torch
    from oracle import train as T
    banner(f"gated forward N={N} C={C} F={F} {dtype} {kind}")
    x, w, _ = _gated(N, C, F, dtype, True)
    with _operator(C, F, kind, dtype, w) as ff:
        xt = to_device(x, dtype)
        out = ff.forward(xt)
        ff.forward(xt, out=xt)
        torch.cuda.synchronize()
    _check("out", out, T.gated_forward(x, w, kind), dtype, (C, F))
    assert torch.equal(xt, out)
