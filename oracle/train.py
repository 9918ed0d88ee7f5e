"""Float64 reference of the training operators: the gated feed-forward, the residual
LayerNorm and clipping by the global norm, each from its formula in plain numpy.  Test
infrastructure only."""
import math

import numpy as np
from scipy.special import ndtr


def activation(kind, a):
    """act(a) and act'(a)."""
    if kind == "silu":
        s = 0.5 * (1.0 + np.tanh(0.5 * a))
        return a * s, s + a * s * (1.0 - s)
    if kind == "gelu":
        phi = ndtr(a)
        return a * phi, phi + a * np.exp(-0.5 * a * a) / math.sqrt(2.0 * math.pi)
    raise ValueError(kind)


def _bias(w, name, size):
    b = w.get(name)
    return np.zeros(size) if b is None else b


def gated_hidden(x, w, kind):
    F = w["Wg"].shape[1]
    a = x @ w["Wg"] + _bias(w, "bg", F)
    u = x @ w["Wu"] + _bias(w, "bu", F)
    return (a, u) + activation(kind, a)


def gated_forward(x, w, kind):
    _, u, y, _ = gated_hidden(x, w, kind)
    return (y * u) @ w["Wd"] + _bias(w, "bd", x.shape[1])


def gated_backward(x, w, kind, g):
    """dx and the six gradients of sum(g * gated_forward(x))."""
    _, u, y, slope = gated_hidden(x, w, kind)
    dh = g @ w["Wd"].T
    da, du = dh * u * slope, dh * y
    return {"dx": da @ w["Wg"].T + du @ w["Wu"].T, "dWg": x.T @ da, "dbg": da.sum(0), "dWu": x.T @ du, "dbu": du.sum(0),
            "dWd": (y * u).T @ g, "dbd": g.sum(0)}


def norm_forward(x, r, gamma, beta, eps):
    y = x if r is None else x + r
    h = (y - y.mean(1, keepdims=True)) / np.sqrt(y.var(1, keepdims=True) + eps)
    return y, h * gamma + beta


def norm_backward(y, g, gr, gamma, eps):
    """dx, dgamma, dbeta of sum(g * out) + sum(gr * y)."""
    rstd = 1.0 / np.sqrt(y.var(1, keepdims=True) + eps)
    h = (y - y.mean(1, keepdims=True)) * rstd
    e = g * gamma
    dx = rstd * (e - e.mean(1, keepdims=True) - h * (e * h).mean(1, keepdims=True))
    return dx + (0.0 if gr is None else gr), (g * h).sum(0), g.sum(0)


def clip(grads, max_norm):
    """The global norm, and the gradients scaled to it."""
    norm = math.sqrt(sum(float((g * g).sum()) for g in grads))
    scale = max_norm / norm if norm > max_norm else 1.0
    return norm, [g * scale for g in grads]
