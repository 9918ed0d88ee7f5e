"""Float64 reference of the operators of a conditioned block: attention to an encoder's states,
the norms around a block and orthogonalised updates, each from its formula in plain numpy.
Test infrastructure only."""
import math

import numpy as np

from .train import norm_backward, norm_forward


def present(B, S, lengths=None, mask=None):
    """Which states are there [B, S]."""
    there = np.ones((B, S), dtype=bool)
    if lengths is not None:
        there &= np.arange(S) < np.asarray(lengths)[:, None]
    return there if mask is None else there & mask


def _heads(t, there, G):
    """[B, S, Hkv, D] as [B, H, S, D] by query head, zero where absent."""
    return np.repeat(np.where(there[..., None, None], t, 0.0), G, axis=2).transpose(0, 2, 1, 3)


def _rows(t):
    return t.transpose(0, 2, 1, 3)


def cross_weights(q, k, there, scale):
    """p [B, H, N, S] and lse [B, H, N]; rows of no state are zero and minus infinity."""
    s = scale * (_rows(q) @ _heads(k, there, q.shape[2] // k.shape[2]).swapaxes(2, 3))
    s = np.where(there[:, None, None, :], s, -np.inf)
    top = s.max(axis=3, initial=-np.inf, keepdims=True)
    e = np.exp(s - np.where(np.isinf(top), 0.0, top))
    z = e.sum(axis=3, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (top + np.log(z))[..., 0]
    return e / np.where(z > 0, z, 1.0), lse


def cross_forward(q, k, v, there, scale):
    """out [B, N, H, D] and lse [B, H, N]."""
    p, lse = cross_weights(q, k, there, scale)
    return _rows(p @ _heads(v, there, q.shape[2] // k.shape[2])), lse


def cross_backward(q, k, v, there, scale, g):
    """dq, dk, dv of sum(g * out), and the sizes of the terms that they are sums of."""
    B, S, HK, D = k.shape
    G = q.shape[2] // HK
    p, _ = cross_weights(q, k, there, scale)
    q, g, k, v = _rows(q), _rows(g), _heads(k, there, G), _heads(v, there, G)

    def shared(t):
        return t.reshape(B, HK, G, S, D).sum(axis=2).transpose(0, 2, 1, 3)
    out = p @ v
    ds = p * (g @ v.swapaxes(2, 3) - (g * out).sum(3, keepdims=True))
    grads = {"dq": scale * _rows(ds @ k), "dk": scale * shared(ds.swapaxes(2, 3) @ q), "dv": shared(p.swapaxes(2, 3) @ g)}
    av, ag = np.abs(v), np.abs(g)
    size = p @ av
    terms = p * (ag @ av.swapaxes(2, 3) + (ag * size).sum(3, keepdims=True))
    sizes = {"out": _rows(size), "dq": scale * _rows(terms @ np.abs(k)), "dk": scale * shared(terms.swapaxes(2, 3) @ np.abs(q)),
             "dv": shared(p.swapaxes(2, 3) @ ag)}
    return grads, sizes


def _sigmoid(a):
    return 0.5 * (1.0 + np.tanh(0.5 * a))


def sandwich_forward(f, x, gate, w, eps):
    """y and LN(y); the latter None without w["gamma_pre"]."""
    _, m = norm_forward(f, None, w["gamma_post"], w["beta_post"], eps)
    y = x + w["scale"] * m * (1.0 if gate is None else _sigmoid(gate))
    if w.get("gamma_pre") is None:
        return y, None
    return y, norm_forward(y, None, w["gamma_pre"], w["beta_pre"], eps)[1]


def sandwich_backward(f, y, gate, gy, gn, w, eps):
    """df, dx, dgate and the parameters' gradients of sum(gy * y) + sum(gn * LN(y))."""
    grads = {}
    dy = np.zeros_like(f) if gy is None else gy
    if gn is not None:
        dy, grads["gamma_pre"], grads["beta_pre"] = norm_backward(y, gn, dy, w["gamma_pre"], eps)
    _, m = norm_forward(f, None, w["gamma_post"], w["beta_post"], eps)
    s = 1.0 if gate is None else _sigmoid(gate)
    grads["scale"] = (dy * s * m).sum(0)
    if gate is not None:
        grads["dgate"] = dy * w["scale"] * m * s * _sigmoid(-gate)
    df, grads["gamma_post"], grads["beta_post"] = norm_backward(f, dy * w["scale"] * s, None, w["gamma_post"], eps)
    return dict(grads, df=df, dx=dy)


NEWTON_SCHULZ = (3.4445, -4.7750, 2.0315)


def orthogonalise(g, steps=5, eps=1e-7):
    """The polynomial of the steps applied to the singular values of g [.., rows, cols]."""
    a, b, c = NEWTON_SCHULZ
    u, s, vt = np.linalg.svd(g, full_matrices=False)
    with np.errstate(invalid="ignore"):
        s = s / (np.sqrt((g * g).sum(axis=(-2, -1)))[..., None] + eps)
    for _ in range(steps):
        s = a * s + b * s ** 3 + c * s ** 5
    return (u * s[..., None, :]) @ vt


def newton_schulz(g, steps=5, eps=1e-7):
    """The same by the products of the definition."""
    a, b, c = NEWTON_SCHULZ
    x = g / (math.sqrt((g * g).sum()) + eps)
    for _ in range(steps):
        gram = x @ x.T
        x = a * x + (b * gram + c * gram @ gram) @ x
    return x
