"""Python face of libts3's training operators (include/ts3.h): the gated feed-forward,
the residual LayerNorm and the clipping of gradients by their global norm.  Argument
marshalling only; every step runs in the library's HIP kernels."""
from __future__ import annotations

import ctypes as ct

import torch

from . import _lib as L
from .layer import _DTYPES

_ACTIVATIONS = {"silu": L.TS3_SILU, "gelu": L.TS3_GELU}


# The current stream of a device, as an integer, without building a Stream object (a microsecond
# of a call of ten), and the current device.
_raw_stream = torch._C._cuda_getCurrentRawStream
_current_device = torch._C._cuda_getDevice


def _ptr(t):
    return None if t is None else t.data_ptr()


class _Handle:
    """Owns a library object: self.h, released by ts3_<kind>_free.  It lives on the device that was
    current when it was made, where its calls run and its tensors have to be."""

    _free = None
    h = None

    def _create(self, *desc):
        h = ct.c_void_p()
        create = self._free.replace("_free", "_create")
        L.check(getattr(L.lib(), create)(*desc, ct.byref(h)), create)
        self.h, self.device = h, _current_device()

    def _call(self, name, *args):
        """The library's function on the handle and the current stream of its device."""
        call = getattr(L.lib(), name)
        if _current_device() == self.device:  # the library launches on the current device
            status = call(self.h, *args, _raw_stream(self.device))
        else:
            with torch.cuda.device(self.device):
                status = call(self.h, *args, _raw_stream(self.device))
        L.check(status, name)

    def close(self):
        if self.h:
            L.check(getattr(L.lib(), self._free)(self.h), self._free)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()

    def _rows(self, t, name, n=None):
        """Checks that t is [n, C] of the operator's type and on its device; returns n."""
        shape = t.shape
        if not (t.get_device() == self.device and t.dtype is self.torch_dtype and len(shape) == 2 and shape[1] == self.C
                and (n is None or shape[0] == n) and t.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous cuda {self.torch_dtype} tensor "
                             f"[{'n' if n is None else n}, {self.C}] on cuda:{self.device}")
        return shape[0]

    def _vector(self, t, name):
        if not (t.get_device() == self.device and t.dtype is torch.float32 and t.is_contiguous() and t.shape == (self.C,)):
            raise ValueError(f"{name} must be a contiguous cuda float32 tensor [{self.C}] on cuda:{self.device}")


class GatedWeights:
    """Device copies, in the operator's type ("bf16" or "fp32"), of Wg, Wu [C, F], Wd [F, C]
    and the biases bg, bu [F], bd [C], which may be absent.  Tensors that already are
    contiguous device tensors of that type are used as they are, not copied."""

    def __init__(self, weights: dict, dtype="bf16", device="cuda"):
        _, self.torch_dtype = _DTYPES[dtype]
        self.t = {}
        for n in L.GATED_NAMES:
            v = weights.get(n)
            self.t[n] = v if v is None else torch.as_tensor(v).to(device=device, dtype=self.torch_dtype).contiguous()
        for n in ("Wg", "Wu", "Wd"):
            if self.t[n] is None:
                raise ValueError(f"{n} is missing")
        self.C, self.F = self.t["Wg"].shape
        for n, shape in (("Wu", (self.C, self.F)), ("Wd", (self.F, self.C)), ("bg", (self.F,)), ("bu", (self.F,)),
                         ("bd", (self.C,))):
            if self.t[n] is not None and self.t[n].shape != shape:
                raise ValueError(f"{n} must be {list(shape)}, not {list(self.t[n].shape)}")


class GatedFeedForward(_Handle):
    """out = (act(x Wg + bg) * (x Wu + bu)) Wd + bd for points x [n, C], and its gradient.

    load() lays a GatedWeights out for the kernels: once for serving, after every change of
    the weights in training.  Everything the operator takes and gives is of its dtype."""

    _free = "ts3_gated_free"

    def __init__(self, C, F, activation="silu", dtype="bf16"):
        self.C, self.F = C, F
        code, self.torch_dtype = _DTYPES[dtype]
        self.desc = L.GatedDesc(C=C, F=F, activation=_ACTIVATIONS[activation], io_dtype=code)
        self._create(ct.byref(self.desc))

    def bytes(self) -> int:
        b = ct.c_int64()
        L.check(L.lib().ts3_gated_bytes(self.h, ct.byref(b)), "ts3_gated_bytes")
        return b.value

    def default_tile(self) -> int:
        row = 3 * ((self.F + 31) // 32 * 32) * (2 if self.torch_dtype is torch.bfloat16 else 4)
        return max(min(1 << 18, (1 << 33) // row), (1 << 31) // row)

    def load(self, w: GatedWeights):
        if (w.C, w.F, w.torch_dtype) != (self.C, self.F, self.torch_dtype):
            raise ValueError(f"weights of C={w.C}, F={w.F}, {w.torch_dtype} for an operator of C={self.C}, F={self.F}, "
                             f"{self.torch_dtype}")
        if any(t is not None and t.get_device() != self.device for t in w.t.values()):
            raise ValueError(f"the weights must be on cuda:{self.device}")
        s = L.GatedWeights(**{n: (t.data_ptr() if t is not None else None) for n, t in w.t.items()})
        self._call("ts3_gated_load", ct.byref(s))

    def forward(self, x, out=None):
        n = self._rows(x, "x")
        if out is None:
            out = torch.empty_like(x)
        else:
            self._rows(out, "out", n)
        self._call("ts3_gated_forward", x.data_ptr(), n, out.data_ptr())
        return out

    def backward(self, x, g, tile: int | None = None, dx=None):
        """Gradients of sum(g * out) at the loaded weights: (dx, {dWg, dbg, dWu, dbu, dWd, dbd}).
        forward(x) need not have run.  `tile` points pass at a time, and their da, du and h are
        kept: by default as many as take 2 GiB, 262,144 at least if those take no more than 8.
        Longer tiles gain up to a tenth at small widths, shorter ones lose: 65,536 points of
        C = 128, F = 512 in bfloat16 1.07 ms per 500,000 points, 262,144 1.02 ms, 1,048,576
        0.93 ms."""
        if tile is None:
            tile = self.default_tile()
        n = self._rows(x, "x")
        self._rows(g, "g", n)
        if dx is None:
            dx = torch.empty_like(x)
        else:
            self._rows(dx, "dx", n)
        C, F = self.C, self.F
        # one buffer, the matrices first
        flat = torch.empty(3 * C * F + 2 * F + C, device=x.device, dtype=self.torch_dtype)
        grads, at = {}, 0
        for name, shape in (("dWg", (C, F)), ("dWu", (C, F)), ("dWd", (F, C)), ("dbg", (F,)), ("dbu", (F,)), ("dbd", (C,))):
            size = shape[0] * shape[1] if len(shape) == 2 else shape[0]
            grads[name] = flat[at:at + size].view(shape)
            at += size
        gs = L.GatedGrads(**{k: t.data_ptr() for k, t in grads.items()})
        self._call("ts3_gated_backward", x.data_ptr(), g.data_ptr(), n, tile, dx.data_ptr(), ct.byref(gs))
        return dx, grads


class ResidualNorm(_Handle):
    """y = x + residual and the LayerNorm of y over C channels, and the gradient of both."""

    _free = "ts3_norm_free"

    def __init__(self, C, dtype="bf16", eps=1e-5):
        self.C = C
        code, self.torch_dtype = _DTYPES[dtype]
        self.desc = L.NormDesc(C=C, io_dtype=code, eps=eps)
        self._create(ct.byref(self.desc))

    def forward(self, x, gamma, beta, residual=None, y=None, out=None):
        """(y, LayerNorm of y).  Without a residual, y is x itself unless a tensor is given for it."""
        n = self._rows(x, "x")
        self._vector(gamma, "gamma")
        self._vector(beta, "beta")
        if residual is not None:
            self._rows(residual, "residual", n)
        if y is not None:
            self._rows(y, "y", n)
        elif residual is not None:
            y = torch.empty_like(x)
        if out is None:
            out = torch.empty_like(x)
        else:
            self._rows(out, "out", n)
        self._call("ts3_norm_forward", x.data_ptr(), _ptr(residual), gamma.data_ptr(), beta.data_ptr(), n, _ptr(y),
                   out.data_ptr())
        return (x if y is None else y), out

    def backward(self, y, g, gamma, residual_grad=None, dx=None):
        """Gradients of sum(g * out) + sum(residual_grad * y): (dx, dgamma, dbeta); dx is that
        of the forward's x and of its residual alike."""
        n = self._rows(y, "y")
        self._rows(g, "g", n)
        self._vector(gamma, "gamma")
        if residual_grad is not None:
            self._rows(residual_grad, "residual_grad", n)
        if dx is None:
            dx = torch.empty_like(y)
        else:
            self._rows(dx, "dx", n)
        d = torch.empty((2, self.C), device=y.device, dtype=torch.float32)
        dgamma, dbeta = d.unbind()
        self._call("ts3_norm_backward", y.data_ptr(), g.data_ptr(), _ptr(residual_grad), gamma.data_ptr(), n,
                   dx.data_ptr(), dgamma.data_ptr(), dbeta.data_ptr())
        return dx, dgamma, dbeta


class GradClip(_Handle):
    """Scales a list of gradients (float32 and bfloat16) so that their global norm is at most
    max_norm: clip(grads, max_norm) -> the norm before, a float32 device scalar."""

    _free = "ts3_clip_free"

    def __init__(self):
        try:
            from . import _tensors
        except ImportError as e:
            raise RuntimeError("_tensors.so is missing or unusable: build it with __graft_entry__.build()") from e
        self._table = _tensors.clip_table
        self._create()

    def __call__(self, grads, max_norm: float, out=None):
        """grads, a list: in place, or into the tensors of the list `out`, one of the same size and
        type for each.  No tensor may come twice or share memory with another, as those of tied
        parameters would: pass it once."""
        table, device = self._table(grads, out)
        if device >= 0 and device != self.device:
            raise ValueError(f"gradients must be on cuda:{self.device}, where the GradClip was made")
        norm = torch.empty((), device=self.device, dtype=torch.float32)
        self._call("ts3_clip_gradients", table, len(grads), max_norm, norm.data_ptr())
        return norm
