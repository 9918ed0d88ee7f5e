"""Attention to an encoder's states on the GPU, where the shapes of test_gpu_conditioned.py do not reach
or their bars do not see: every kernel at scores of hundreds, many samples, a
mesh of 100 million points.  Bars, fixed before the first
run; u is 2^-24."""
import math

import numpy as np
import pytest

from cross_shapes import FEW_PARTS, LDS_ROWS, LDS_STATES, MANY, WHOLE, some_lengths
from gpu_helpers import banner, to_device, to_host
from test_gpu_conditioned import _case, _check, _compare, _round, _run

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,N,S,H,HK,D", [(1, 128, 40, 1, 1, 16), (1, 20, 1500, 2, 2, 16), (1, 131_072, 40, 4, 2, 16), (2, 300, 70, 2, 1, 32),
                                          (1, 31, 900, 1, 1, 32), (1, 131_072, 70, 4, 4, 32), (1, 200, 70, 2, 2, 48), (1, 300, 40, 1, 1, 128)])
def test_lse_of_scores_in_the_hundreds(B, N, S, H, HK, D, dtype):
    """lse is float32 whatever the operands' type.  Every value of a query is the same, and of a state, so that errors
    of the operands do not average out over the products.

    A score is a sum of D products of bfloat16 values, exact (float32: six part products, of which those dropped and the
    rounding of the scaled query are 4 u), times scale log2(e): 3 u; then the base, the logarithm and the way back: 4 u, of
    the largest score X.  S weights walk S u at most, and the exponential and logarithm 4 u.

    The output of values of one is one, but for the weights' rounding and its own in bfloat16, and for the walks of
    two sums in float32, one of three part products a state, and 8 u."""
    import torch
    from paper_2602_04940_amd import CrossAttention
    banner(f"lse B={B} N={N} S={S} H={H}/{HK} D={D} {dtype}")
    scale = np.float64(np.float32(75.0 / D))
    rng = np.random.default_rng([1, N, S, D])
    x, y = 1 + np.arange(128) / 128, 1 + rng.integers(0, 128, (B, S, HK)) / 128
    tt = torch.float32 if dtype == "fp32" else torch.bfloat16
    q = to_device(x, dtype)[torch.arange(N, device="cuda") % 128][None, :, None, None].expand(B, N, H, D).contiguous()
    k = to_device(y, dtype)[..., None].expand(B, S, HK, D).contiguous()
    with CrossAttention(H, D, kv_heads=HK, dtype=dtype, scale=float(scale)) as a:
        out, lse = a.forward(q, k, torch.ones_like(k))
        torch.cuda.synchronize()
    assert out.dtype is tt and np.abs(to_host(out) - 1).max() <= (2 * 2.0 ** -8 if dtype == "bf16" else (4 * S + 8) * U)
    s = scale * D * x[:, None, None, None] * y[None]  # [128, B, S, HK]
    top = s.max(axis=2, keepdims=True)
    ref = (top + np.log(np.exp(s - top).sum(axis=2, keepdims=True)))[:, :, 0]
    ref = np.repeat(ref.transpose(1, 2, 0), H // HK, axis=1)  # [B, H, 128]
    X = s.max()
    bar = ((D if dtype == "bf16" else 6 * D + 4) + 8) * U * X + (S + 4) * U
    got = to_host(lse)
    err = max(np.abs(got[:, :, i:i + 128] - ref[:, :, :got[:, :, i:i + 128].shape[2]]).max() for i in range(0, N, 128))
    print(f"lse to {ref.max():.1f}: off by {err:.2e} (bar {bar:.2e})", flush=True)
    assert err <= bar


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("lengths", [False, True])
@pytest.mark.parametrize("B,N,S,H,HK,D", MANY)
def test_many_samples(B, N, S, H, HK, D, lengths, dtype):
    from oracle import conditioned as R
    banner(f"cross B={B} N={N} S={S} H={H}/{HK} D={D} lengths={lengths} {dtype}")
    q, k, v, g = _case(B, N, S, H, HK, D, dtype, seed=11)
    lens = np.random.default_rng(12).integers(0, S + 1, B).tolist() if lengths else None
    _compare(q, k, v, g, dtype, R.present(B, S, lens), 1 / math.sqrt(D), *_run(q, k, v, g, dtype, HK, lens))


def test_a_mesh_of_100_million_points():
    """Eight heads, whose queries (and gradients) overlap in memory: head h of point n starts 16 (n + h) elements from
    the first.  A row depends on itself alone: blocks of points, at the ends and around the 2^26th, are bitwise as in a
    call of their own.  dk and dv are the sums of those of five calls of 20 million points, each rounded once to
    bfloat16 (2^-8 of its norm at most); the sums' walks are of terms of either sign, 2^-10 of the result at most."""
    import torch
    from paper_2602_04940_amd import CrossAttention
    N, S, H, D = 100_000_000, 40, 8, 16
    gen = torch.Generator(device="cuda").manual_seed(13)

    def rows():
        flat = torch.empty(16 * (N + H - 1), dtype=torch.bfloat16, device="cuda")
        for part in flat.split(1 << 28):
            part.copy_(torch.randn(part.shape, generator=gen, device="cuda"))
        return flat.as_strided((1, N, H, D), (0, 16, 16, 1))
    q, g = rows(), rows()
    k, v = (torch.randn((1, S, H, D), generator=gen, device="cuda").bfloat16() for _ in range(2))
    with CrossAttention(H, D) as a, CrossAttention(H, D) as b:
        out, lse = a.forward(q, k, v)
        dq, dk, dv = a.backward(q, k, v, out, lse, g)
        torch.cuda.synchronize()
        parts = []
        for at in range(0, N, 20_000_000):
            s = slice(at, at + 20_000_000)
            parts.append(b.backward(q[:, s], k, v, out[:, s].contiguous(), lse[:, :, s].contiguous(), g[:, s])[1:])
        for at in (0, (1 << 26) - 150_000, N - 262_144):
            s = slice(at, at + 262_144)
            o, l = b.forward(q[:, s], k, v)
            assert torch.equal(out[:, s], o) and torch.equal(lse[:, :, s], l), at
            assert torch.equal(dq[:, s], b.backward(q[:, s], k, v, o, l, g[:, s])[0]), at
        torch.cuda.synchronize()
    del q, g, out, lse, dq, o, l
    torch.cuda.empty_cache()
    for got, each in ((dk, [p[0] for p in parts]), (dv, [p[1] for p in parts])):
        got, each = got.double(), [t.double() for t in each]
        err, size = float((got - sum(each)).norm()), float(got.norm())
        bar = 2.0 ** -8 * (size + sum(float(t.norm()) for t in each)) + 2.0 ** -10 * size
        print(f"off by {err:.3e} of {size:.3e} (bar {bar:.3e})", flush=True)
        assert err <= bar


def _close_in_norm(name, got, ref, walk):
    """In bfloat16 every output is within 2^-8 in the mean square: its own rounding and the weights' or slopes', whose
    terms have about its size, have at most 2^-8 / sqrt 3 each, independently (0.0033 together).  In blocks of 32 rows or
    states, whose terms may be three times as large as their sum, within twice that and `walk`, what the float32 sums
    may be off by: of a sample with one state dq and dk are zero, as differences of equal float32 sums.  A sum over
    many rows that lacks one in a thousand is off by 3 %."""
    ref = ref.reshape(-1, ref.shape[2] * ref.shape[3])
    err = to_host(got).reshape(ref.shape) - ref
    whole, worst = np.linalg.norm(err) / np.linalg.norm(ref), 0.0
    for i in range(0, len(ref), 32):
        bar = 2.0 ** -7 * np.linalg.norm(ref[i:i + 32]) + walk * math.sqrt(ref[i:i + 32].size)
        worst = max(worst, np.linalg.norm(err[i:i + 32]) / max(bar, 1e-300))
    print(f"{name}: {whole:.2e} in norm, worst block {worst:.3f} of its bar", flush=True)
    assert whole <= 2.0 ** -8 and worst <= 1, name


def _both(B, N, S, H, HK, D, dtype, lengths, seed):
    """The bars of test_gpu_conditioned.py, of the size of the terms, and those in norm."""
    from oracle import conditioned as R
    banner(f"cross B={B} N={N} S={S} H={H}/{HK} D={D} lengths={lengths} {dtype}")
    q, k, v, g = _case(B, N, S, H, HK, D, dtype, seed=seed)
    lens = some_lengths(B, S) if lengths else None
    there, scale = R.present(B, S, lens), 1 / math.sqrt(D)
    out, lse, grads = _run(q, k, v, g, dtype, HK, lens)
    refs, sizes = R.cross_backward(q, k, v, there, scale, g)
    refs["out"], ref_lse = R.cross_forward(q, k, v, there, scale)
    X = scale * np.sqrt((q * q).sum(3).max() * (k * k).sum(3).max())
    walk = 8 + math.sqrt(S) + math.sqrt(N * H // HK) + (4 + math.sqrt(D)) * X
    got, empty = to_host(lse), np.isinf(ref_lse)
    assert (got[empty] == -np.inf).all() and np.abs(got[~empty] - ref_lse[~empty]).max() <= 4 * walk * U
    for name, t in dict(grads, out=out).items():
        _check(name, t, refs[name], sizes[name], dtype, walk)
        if dtype == "bf16":
            _close_in_norm(name, t, refs[name], 4 * walk * U * sizes[name].max())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("lengths", [False, True])
@pytest.mark.parametrize("B,N,S,H,HK,D", FEW_PARTS)
def test_parts_joined_by_lanes(B, N, S, H, HK, D, lengths, dtype):
    _both(B, N, S, H, HK, D, dtype, lengths, 14)


@pytest.mark.parametrize("lengths", [False, True])
@pytest.mark.parametrize("B,N,S,H,HK,D,dtype", [(*c, t) for c in WHOLE for t in ("fp32", "bf16") if t == "bf16" or c[5] == 16])
def test_all_states_in_lds(B, N, S, H, HK, D, lengths, dtype):
    _both(B, N, S, H, HK, D, dtype, lengths, 15)


@pytest.mark.parametrize("more", [0, 1])
@pytest.mark.parametrize("dtype,D", LDS_STATES)
def test_as_many_states_as_lds_holds_and_one_more(dtype, D, more):
    """Some hundred rows of many, the last among them, against the reference of those rows alone."""
    from oracle import conditioned as R
    B, N, H, HK = LDS_ROWS
    S = LDS_STATES[dtype, D] + more
    banner(f"cross N={N} S={S} H={H}/{HK} D={D} {dtype}")
    q, k, v, g = _case(B, N, S, H, HK, D, dtype, seed=16)
    mask = np.random.default_rng(17).random((B, S)) < 0.9
    mask[0, -1] = True
    out, lse, grads = _run(q, k, v, g, dtype, HK, mask=mask)
    rows = np.r_[0:70, np.random.default_rng(18).integers(70, N - 40, 100), N - 40:N]
    for t in (out, grads["dq"]):
        assert t.isfinite().all()
    # dk and dv are sums over all rows: of these alone, in a call of their own
    ours = _run(q[:, rows], k, v, g[:, rows], dtype, HK, mask=mask)[2]
    _compare(q[:, rows], k, v, g[:, rows], dtype, mask, 1 / math.sqrt(D), out[:, rows], lse[:, :, rows],
             dict(ours, dq=grads["dq"][:, rows]))


@pytest.mark.parametrize("B,N,S,H,HK,D", [(1, 300, 40, 1, 1, 16), (2, 300, 600, 1, 1, 32), (1, 200, 700, 2, 1, 64), (1, 140_000, 40, 4, 4, 16),
                                          (1, 500, 60, 2, 2, 128)])
def test_bfloat16_slopes_do_not_hang_on_the_rounded_output(B, N, S, H, HK, D):
    """Values that lie around 16 with a spread of a half: out is rounded by up to 1/16 and g.out with it, a tenth of
    the slopes' spread.  What that would do to dq and dk is computed here and is beyond the bar; the kernels put it right
    with float32 sums.

    Bar, in norm: 2^-8 of the result, and of the root of the sum of the squares of its terms, whose roundings
    are independent: p (dp - delta) k, delta of the rounded output, and delta's error times p k, for dq; ds q for dk."""
    from oracle import conditioned as R
    banner(f"cross slopes N={N} S={S} H={H}/{HK} D={D}")
    q, k, v, g = _case(B, N, S, H, HK, D, "bf16", seed=19, scale=2.0)
    v = np.round(4 * v).clip(-8, 8) / 8 + 16.0   # steps of 1/8: exact
    k = k + 1.0
    k = _round(k, "bf16")
    there, scale = R.present(B, S), 1 / math.sqrt(D)
    refs = R.cross_backward(q, k, v, there, scale, g)[0]
    out, lse, grads = _run(q, k, v, g, "bf16", HK)
    G = H // HK
    p, _ = R.cross_weights(q, k, there, scale)
    o = p @ R._heads(v, there, G)
    gr, kr, vr, qr = R._rows(g), R._heads(k, there, G), R._heads(v, there, G), R._rows(q)
    dp = gr @ vr.swapaxes(2, 3)
    off = (gr * (_round(o, "bf16") - o)).sum(3, keepdims=True)          # of delta from the rounded output
    ds = p * (dp - (gr * o).sum(3, keepdims=True))

    def shared(t):
        return t.reshape(B, HK, G, S, D).sum(axis=2).transpose(0, 2, 1, 3)
    x = ds - p * off
    terms = {"dq": scale * R._rows(np.sqrt((x * x) @ (kr * kr)) + np.abs(off) * np.sqrt((p * p) @ (kr * kr))),
             "dk": scale * np.sqrt(shared((ds * ds).swapaxes(2, 3) @ (qr * qr)))}
    wrong = {"dq": scale * R._rows(x @ kr), "dk": scale * shared(x.swapaxes(2, 3) @ qr)}
    for name, t in terms.items():
        ref = refs[name]
        bar = 2.0 ** -8 * (np.linalg.norm(ref) + np.linalg.norm(t))
        err, without = np.linalg.norm(to_host(grads[name]) - ref), np.linalg.norm(wrong[name] - ref)
        print(f"{name}: off by {err / np.linalg.norm(ref):.2e} (bar {bar / np.linalg.norm(ref):.2e}, as it would be "
              f"{without / np.linalg.norm(ref):.2e})", flush=True)
        assert without > 1.5 * bar and err <= bar, name


@pytest.mark.parametrize("D", [48, 128])
def test_float32_weights_in_the_gradient(D):
    """dk and dv of few rows and 5,000 states with scores below one: their errors are the weights', e^(s - lse).

    lse lies in 8 to 16, and so do the logarithm before it, its multiple and the exponent: four roundings of at most
    2^-21, uniform, one of them in nats and three times log 2, 2^-21 sqrt((1 + 3 log^2 2) / 3) = 4.3e-7 in the mean
    square; sums of 64 rows, 24 part products of at most the result's size, 1.7e-7.  The bar is twice both.  Scores whose
    sums of six part products per 16 of D start from the logarithm would be off by sqrt(6 D / 16) 2^-21 log 2 / sqrt 3 more:
    1.4e-6 at 128."""
    from oracle import conditioned as R
    banner(f"cross float32 weights D={D}")
    B, N, S, H = 1, 64, 5000, 8
    q, k, v, g = _case(B, N, S, H, H, D, "fp32", seed=20, scale=0.3)
    _, lse, grads = _run(q, k, v, g, "fp32", H)
    assert 8 < lse.min() and lse.max() < 16 / math.log2(math.e)
    refs = R.cross_backward(q, k, v, R.present(B, S), 1 / math.sqrt(D), g)[0]
    for name in ("dk", "dv"):
        err = np.linalg.norm(to_host(grads[name]) - refs[name]) / np.linalg.norm(refs[name])
        print(f"{name}: {err:.2e} in norm", flush=True)
        assert err <= 2 * math.hypot(4.3e-7, 1.7e-7), name


@pytest.mark.parametrize("B,N,S,H,HK,D", [(1, 300, 40, 1, 1, 16), (2, 300, 600, 1, 1, 32), (1, 200, 700, 2, 1, 64), (1, 140_000, 40, 4, 4, 16),
                                          (1, 500, 60, 2, 2, 128)])
def test_bfloat16_slopes_do_not_carry_the_keys_mean(B, N, S, H, HK, D):
    """A row's slopes sum to zero, their roundings do not: keys around 4 with a spread of one would put dq off by four
    times as much as the keys' differences do.  The kernels take the roundings' sum times the mean key off again.

    Bar, in norm: 2^-8, of which dq's own rounding and those of the terms p (dp - delta) (k - mean k), whose squares'
    sum is about dq's, take 2^-8 / sqrt 3 each at most.  The rounded slopes' own sum is computed here, and is beyond it."""
    from oracle import conditioned as R
    banner(f"cross mean key N={N} S={S} H={H}/{HK} D={D}")
    q, k, v, g = _case(B, N, S, H, HK, D, "bf16", seed=21)
    k = _round(k + 4.0, "bf16")
    there, scale = R.present(B, S), 1 / math.sqrt(D)
    ref = R.cross_backward(q, k, v, there, scale, g)[0]["dq"]
    _, _, grads = _run(q, k, v, g, "bf16", HK)
    p, _ = R.cross_weights(q, k, there, scale)
    G, gr = H // HK, R._rows(g)
    kr, vr = R._heads(k, there, G), R._heads(v, there, G)
    ds = p * (gr @ vr.swapaxes(2, 3) - (gr * (p @ vr)).sum(3, keepdims=True))
    size = np.linalg.norm(ref)
    err = np.linalg.norm(to_host(grads["dq"]) - ref) / size
    without = np.linalg.norm(scale * R._rows(_round(ds, "bf16") @ kr) - ref) / size
    print(f"dq: off by {err:.2e} (as it would be {without:.2e})", flush=True)
    assert without > 1.2 * 2.0 ** -8 and err <= 2.0 ** -8
