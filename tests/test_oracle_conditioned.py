"""Pins of the float64 reference of a conditioned block's operators: loops, closed forms,
differences and torch's float64 functions."""
import math

import numpy as np
import pytest
import torch

from oracle import conditioned as R


def _inputs(seed, B=2, N=3, S=5, H=4, HK=2, D=3):
    rng = np.random.default_rng(seed)
    return rng.standard_normal((B, N, H, D)), rng.standard_normal((B, S, HK, D)), rng.standard_normal((B, S, HK, D)), rng


def test_attention_by_loops_and_rows_of_no_state():
    q, k, v, rng = _inputs(0)
    there = R.present(2, 5, [4, 0], rng.random((2, 5)) < 0.7)
    there[0, 1] = True
    out, lse = R.cross_forward(q, k, v, there, 0.7)
    for n in range(3):
        for h in range(4):
            s = [math.exp(0.7 * q[0, n, h] @ k[0, j, h // 2]) if there[0, j] else 0.0 for j in range(5)]
            ref = sum(w * v[0, j, h // 2] for j, w in enumerate(s)) / sum(s)
            np.testing.assert_allclose(out[0, n, h], ref, rtol=1e-13)
            assert abs(lse[0, h, n] - math.log(sum(s))) < 1e-13
    assert (out[1] == 0).all() and (lse[1] == -np.inf).all()


def test_attention_matches_torch_and_its_gradients():
    q, k, v, rng = _inputs(1)
    there = np.ones((2, 5), dtype=bool)
    there[1, 3:] = False
    g = rng.standard_normal(q.shape)
    qt, kt, vt = (torch.tensor(a, requires_grad=True) for a in (q, k, v))
    heads = [t.repeat_interleave(2, dim=2).transpose(1, 2) for t in (kt, vt)]
    ref = torch.nn.functional.scaled_dot_product_attention(qt.transpose(1, 2), *heads, scale=0.4,
                                                           attn_mask=torch.tensor(there)[:, None, None, :]).transpose(1, 2)
    ref.backward(torch.tensor(g))
    out, _ = R.cross_forward(q, k, v, there, 0.4)
    np.testing.assert_allclose(out, ref.detach().numpy(), atol=1e-13)
    grads, sizes = R.cross_backward(q, k, v, there, 0.4, g)
    for name, t in (("dq", qt), ("dk", kt), ("dv", vt)):
        np.testing.assert_allclose(grads[name], t.grad.numpy(), atol=1e-13)
        assert (np.abs(grads[name]) <= sizes[name] + 1e-13).all()
    assert (np.abs(out) <= sizes["out"] + 1e-13).all()
    assert (grads["dk"][1, 3:] == 0).all() and (grads["dv"][1, 3:] == 0).all()


@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("pre", [True, False])
def test_sandwich_against_differences(gate, pre):
    rng = np.random.default_rng(2)
    N, C, t = 4, 6, 1e-6
    w = {n: rng.standard_normal(C) for n in ("gamma_post", "beta_post", "scale") + (("gamma_pre", "beta_pre") if pre else ())}
    x = {"f": rng.standard_normal((N, C)), "x": rng.standard_normal((N, C)), "gate": rng.standard_normal((N, C)) if gate else None}
    gy, gn = rng.standard_normal((N, C)), rng.standard_normal((N, C)) if pre else None

    def loss(x, w):
        y, n = R.sandwich_forward(x["f"], x["x"], x["gate"], w, 1e-5)
        return (gy * y).sum() + (0.0 if n is None else (gn * n).sum())
    y, _ = R.sandwich_forward(x["f"], x["x"], x["gate"], w, 1e-5)
    grads = R.sandwich_backward(x["f"], y, x["gate"], gy, gn, w, 1e-5)
    for name in w:
        v = rng.standard_normal(C)
        fd = (loss(x, dict(w, **{name: w[name] + t * v})) - loss(x, dict(w, **{name: w[name] - t * v}))) / (2 * t)
        assert abs(fd - grads[name] @ v) < 1e-7 * (1 + abs(fd)), name
    for name in ("f", "x") + (("gate",) if gate else ()):
        v = rng.standard_normal((N, C))
        fd = (loss(dict(x, **{name: x[name] + t * v}), w) - loss(dict(x, **{name: x[name] - t * v}), w)) / (2 * t)
        assert abs(fd - (grads["d" + name] * v).sum()) < 1e-7 * (1 + abs(fd)), name


def test_orthogonalise_by_products_and_in_one_dimension():
    rng = np.random.default_rng(3)
    for shape in ((5, 9), (9, 5), (6, 6), (1, 4), (1, 1)):
        g = rng.standard_normal(shape) * 1e-3
        np.testing.assert_allclose(R.orthogonalise(g), R.newton_schulz(g), atol=1e-11)
    s = 1.0
    for _ in range(5):
        s = 3.4445 * s - 4.7750 * s ** 3 + 2.0315 * s ** 5
    np.testing.assert_allclose(R.orthogonalise(np.array([[-2.0]]), eps=0.0), [[-s]], atol=1e-14)
    assert (R.orthogonalise(np.zeros((3, 4))) == 0).all()
    values = np.linalg.svd(R.orthogonalise(rng.standard_normal((20, 300))), compute_uv=False)
    assert values.min() > 0.6 and values.max() < 1.25
