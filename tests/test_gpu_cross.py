"""Attention to an encoder's states on the GPU, where the shapes of test_gpu_conditioned.py do not reach
or their bars do not see: every kernel at scores of hundreds, many samples, a
mesh of 100 million points.  Bars, fixed before the first
run; u is 2^-24."""
import math

import numpy as np
import pytest

from gpu_helpers import banner, to_device, to_host
from test_gpu_conditioned import _case, _compare, _run

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


# (B, N, S, H, Hkv, D): more samples and shared heads than compute units, of a few rows (in the four-wave kernels)
# and of enough that a workgroup's waves each have four blocks of them (all states in LDS).
MANY = [(1500, 70, 50, 4, 4, 32), (4500, 1, 20, 4, 4, 16), (40, 2100, 40, 8, 8, 32), (33, 1050, 33, 16, 8, 16)]


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
