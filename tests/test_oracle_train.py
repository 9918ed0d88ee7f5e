"""The float64 reference of the training operators: gradients against finite differences,
values against torch in float64, and planted mistakes that these checks must catch."""
import numpy as np
import pytest
import torch

from oracle import train as T


def _gated(seed=0, n=5, C=6, F=7, bias=True):
    rng = np.random.default_rng(seed)
    w = {"Wg": rng.standard_normal((C, F)), "Wu": rng.standard_normal((C, F)), "Wd": rng.standard_normal((F, C))}
    if bias:
        w.update(bg=rng.standard_normal(F), bu=rng.standard_normal(F), bd=rng.standard_normal(C))
    return rng.standard_normal((n, C)), w, rng.standard_normal((n, C))


def _differences(f, a, step=1e-6):
    d = np.empty_like(a)
    for i in np.ndindex(a.shape):
        keep = a[i]
        a[i] = keep + step
        hi = f()
        a[i] = keep - step
        lo = f()
        a[i] = keep
        d[i] = (hi - lo) / (2 * step)
    return d


# A central difference of step 1e-6 on values of order 10: truncation 1e-12, rounding
# 10 * 2^-53 / 1e-6 = 1e-9, a hundred of them added.
BAR = 1e-6


@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("bias", [True, False])
def test_gated_gradients_match_differences(kind, bias):
    x, w, g = _gated(bias=bias)
    got = T.gated_backward(x, w, kind, g)

    def loss():
        return float((g * T.gated_forward(x, w, kind)).sum())
    assert np.abs(got["dx"] - _differences(loss, x)).max() < BAR
    for n in w:
        assert np.abs(got["d" + n] - _differences(loss, w[n])).max() < BAR, n


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_gated_matches_torch(kind):
    x, w, _ = _gated(3, 9, 5, 11)
    t = {k: torch.from_numpy(v) for k, v in w.items()}
    act = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[kind]
    xt = torch.from_numpy(x)
    ref = (act(xt @ t["Wg"] + t["bg"]) * (xt @ t["Wu"] + t["bu"])) @ t["Wd"] + t["bd"]
    assert np.abs(T.gated_forward(x, w, kind) - ref.numpy()).max() < 1e-12


def test_gated_gate_of_large_values():
    """SiLU and GELU are the identity far right and zero far left."""
    a = np.array([-1e3, -60.0, 60.0, 1e3])
    for kind in ("silu", "gelu"):
        y, slope = T.activation(kind, a)
        assert np.allclose(y, [0, 0, 60, 1e3], atol=1e-20) and np.allclose(slope, [0, 0, 1, 1], atol=1e-20)


@pytest.mark.parametrize("residual", [True, False])
def test_norm_gradients_match_differences(residual):
    rng = np.random.default_rng(1)
    n, C, eps = 4, 9, 1e-3
    x, r, g, gr = rng.standard_normal((4, n, C))
    gamma, beta = rng.standard_normal((2, C))
    r, gr = (r, gr) if residual else (None, np.zeros_like(gr))

    def loss():
        y, out = T.norm_forward(x, r, gamma, beta, eps)
        return float((g * out).sum() + (gr * y).sum())
    y, out = T.norm_forward(x, r, gamma, beta, eps)
    dx, dgamma, dbeta = T.norm_backward(y, g, gr if residual else None, gamma, eps)
    assert np.abs(dx - _differences(loss, x)).max() < BAR
    assert np.abs(dgamma - _differences(loss, gamma)).max() < BAR
    assert np.abs(dbeta - _differences(loss, beta)).max() < BAR
    ref = torch.nn.functional.layer_norm(torch.from_numpy(y), (C,), torch.from_numpy(gamma), torch.from_numpy(beta), eps)
    assert np.abs(out - ref.numpy()).max() < 1e-12


def test_clip_scales_to_the_bound_and_leaves_smaller_lists():
    rng = np.random.default_rng(2)
    g = [rng.standard_normal(s) for s in ((3, 4), (1,), (0,), (17,))]
    ref = np.linalg.norm(np.concatenate([a.ravel() for a in g]))
    norm, out = T.clip(g, 0.5)
    assert abs(norm - ref) < 1e-12
    assert abs(np.linalg.norm(np.concatenate([a.ravel() for a in out])) - 0.5) < 1e-12
    norm, out = T.clip(g, 2 * ref)
    assert all((a == b).all() for a, b in zip(g, out))


@pytest.mark.parametrize("mistake", ["swap gate and up", "no slope", "unbiased variance", "mean not removed"])
def test_planted_mistakes_are_caught(mistake, monkeypatch):
    if mistake in ("swap gate and up", "no slope"):
        x, w, g = _gated()
        true = T.gated_backward(x, w, "silu", g)
        if mistake == "no slope":
            act = T.activation
            monkeypatch.setattr(T, "activation", lambda k, a: (act(k, a)[0], act(k, a)[0] / a))
        else:
            w = dict(w, Wg=w["Wu"], Wu=w["Wg"])
        assert np.abs(T.gated_backward(x, w, "silu", g)["dx"] - true["dx"]).max() > 1e-2
        return
    rng = np.random.default_rng(1)
    y, g = rng.standard_normal((2, 4, 9))
    gamma = rng.standard_normal(9)
    dx, _, _ = T.norm_backward(y, g, None, gamma, 0.0)
    assert np.abs(dx.sum(1)).max() < 1e-12 and np.abs((dx * y).sum(1)).max() < 1e-12  # orthogonal to 1 and y
    e = g * gamma
    rstd = 1 / np.sqrt(y.var(1, keepdims=True, ddof=1 if mistake == "unbiased variance" else 0))
    h = (y - y.mean(1, keepdims=True)) * rstd
    bad = rstd * (e - (0.0 if mistake == "mean not removed" else e.mean(1, keepdims=True)) - h * (e * h).mean(1, keepdims=True))
    assert max(np.abs(bad.sum(1)).max(), np.abs((bad * y).sum(1)).max()) > 1e-3
