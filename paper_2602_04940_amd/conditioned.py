"""Python face of libts3's operators of a conditioned block (include/ts3.h): attention to an
encoder's states, the norms around a block and orthogonalised updates.  Argument marshalling
only; every step runs in the library's HIP kernels."""
from __future__ import annotations

import ctypes as ct
import math
import struct

import torch

from . import _lib as L
from .layer import _DTYPES
from .train import _Handle, _ptr

# ts3_cross_inputs and ts3_view as bytes: a fraction of the time that ctypes takes for their fields.
_INPUTS = struct.Struct("=3i4x14q")
_VIEW = struct.Struct("=4q")


class CrossAttention(_Handle):
    """softmax(scale q k^T) v of points [B, N, heads, head_dim] over an encoder's states
    [B, S, kv_heads, head_dim], and its gradient; heads / kv_heads query heads in a row share a
    head of keys and values.  The scale is 1 / sqrt(head_dim) unless given.

    q, k, v and the output's gradient may be views, of one projection for instance: the last
    dimension contiguous, the other strides multiples of 16 bytes.  `lengths` (int32 [B]: the
    states from there on are absent) and `mask` (bool [B, S], False is absent) say which states
    there are; a sample of none gives zeros."""

    _free = "ts3_cross_free"

    def __init__(self, heads, head_dim, kv_heads=None, dtype="bf16", scale=None):
        self.H, self.D, self.Hkv = heads, head_dim, heads if kv_heads is None else kv_heads
        code, self.torch_dtype = _DTYPES[dtype]
        if scale is not None and not (math.isfinite(scale) and ct.c_float(scale).value > 0.0):
            raise ValueError("scale must be finite and > 0")
        self.desc = L.CrossDesc(H=self.H, Hkv=self.Hkv, D=self.D, io_dtype=code, scale=scale or 0.0)
        self._create(ct.byref(self.desc))

    def bytes(self) -> int:
        b = ct.c_int64()
        L.check(L.lib().ts3_cross_bytes(self.h, ct.byref(b)), "ts3_cross_bytes")
        return b.value

    def _view(self, t, name, B, n, heads):
        """(address, strides) of t [B, n, heads, D]."""
        if not (t.get_device() == self.device and t.dtype is self.torch_dtype and t.shape == (B, n, heads, self.D)):
            raise ValueError(f"{name} must be a cuda {self.torch_dtype} tensor [{B}, {n}, {heads}, {self.D}] on "
                             f"cuda:{self.device}")
        sb, sr, sh, sd = t.stride()
        if sd != 1:
            raise ValueError(f"{name}: the last dimension must be contiguous")
        # A dimension of one is never stepped along, whatever its stride says.
        return t.data_ptr(), sb if B > 1 else 0, sr if n > 1 else 0, sh if heads > 1 else 0

    def _whole(self, t, name, shape, dtype):
        if not (t.get_device() == self.device and t.dtype is dtype and t.shape == shape and t.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous cuda {dtype} tensor {list(shape)} on cuda:{self.device}")
        return t.data_ptr()

    def _inputs(self, q, k, v, lengths, mask):
        if q.dim() != 4 or k.dim() != 4:
            raise ValueError("q, k and v must be [samples, points or states, heads, head_dim]")
        B, N, S = q.shape[0], q.shape[1], k.shape[1]
        if mask is not None and mask.dtype is not torch.bool:
            raise ValueError("mask must be a bool tensor")
        packed = _INPUTS.pack(B, N, S, *self._view(q, "q", B, N, self.H), *self._view(k, "k", B, S, self.Hkv),
                              *self._view(v, "v", B, S, self.Hkv),
                              0 if lengths is None else self._whole(lengths, "lengths", (B,), torch.int32),
                              0 if mask is None else self._whole(mask, "mask", (B, S), torch.bool))
        return packed, B, N, S

    def forward(self, q, k, v, lengths=None, mask=None, out=None, lse=None):
        """(out, lse): the output as q, contiguous, and the float32 logarithms of the sums of
        exponentials [B, heads, N], which the backward reads."""
        packed, B, N, _ = self._inputs(q, k, v, lengths, mask)
        if out is None:
            out = torch.empty((B, N, self.H, self.D), device=q.device, dtype=self.torch_dtype)
        else:
            self._whole(out, "out", (B, N, self.H, self.D), self.torch_dtype)
        if lse is None:
            lse = torch.empty((B, self.H, N), device=q.device, dtype=torch.float32)
        else:
            self._whole(lse, "lse", (B, self.H, N), torch.float32)
        self._call("ts3_cross_forward", packed, out.data_ptr(), lse.data_ptr())
        return out, lse

    def backward(self, q, k, v, out, lse, g, lengths=None, mask=None, dq=None):
        """(dq, dk, dv), contiguous: gradients of sum(g * out) for the forward's inputs, out and
        lse.  Those of absent states are zero, and of shared heads the sums over their sharers."""
        packed, B, N, S = self._inputs(q, k, v, lengths, mask)
        rows, states = (B, N, self.H, self.D), (B, S, self.Hkv, self.D)
        po, pl = self._whole(out, "out", rows, self.torch_dtype), self._whole(lse, "lse", (B, self.H, N), torch.float32)
        pg = _VIEW.pack(*self._view(g, "g", B, N, self.H))
        if dq is None:
            dq = torch.empty(rows, device=q.device, dtype=self.torch_dtype)
        else:
            self._whole(dq, "dq", rows, self.torch_dtype)
        dk, dv = (torch.empty(states, device=q.device, dtype=self.torch_dtype) for _ in range(2))
        self._call("ts3_cross_backward", packed, po, pl, pg, dq.data_ptr(), dk.data_ptr(), dv.data_ptr())
        return dq, dk, dv


class SandwichNorm(_Handle):
    """The norms around a block of C channels, with its gate and residual scale, and their gradient:

        y   = x + scale * sigmoid(gate) * (LN(f) gamma_post + beta_post)
        out = LN(y) gamma_pre + beta_pre

    for the block's output f and the residual stream x [n, C]; the gate [n, C] and the second
    norm may be absent."""

    _free = "ts3_sandwich_free"

    def __init__(self, C, dtype="bf16", eps=1e-5):
        self.C = C
        code, self.torch_dtype = _DTYPES[dtype]
        self.desc = L.SandwichDesc(C=C, io_dtype=code, eps=eps)
        self._create(ct.byref(self.desc))

    def forward(self, f, x, gamma_post, beta_post, scale, gate=None, gamma_pre=None, beta_pre=None, y=None, out=None):
        """(y, out); out is None without gamma_pre and beta_pre.  y may be given as x."""
        n = self._rows(f, "f")
        self._rows(x, "x", n)
        if gate is not None:
            self._rows(gate, "gate", n)
        pre = gamma_pre is not None
        if pre is not (beta_pre is not None) or (out is not None and not pre):
            raise ValueError("gamma_pre and beta_pre come together, and out with them")
        params = {"gamma_post": gamma_post, "beta_post": beta_post, "scale": scale}
        if pre:
            params.update(gamma_pre=gamma_pre, beta_pre=beta_pre)
        for name, t in params.items():
            self._vector(t, name)
        if y is None:
            y = torch.empty_like(x)
        else:
            self._rows(y, "y", n)
        if out is not None:
            self._rows(out, "out", n)
        elif pre:
            out = torch.empty_like(x)
        p = L.SandwichParams(*(t.data_ptr() for t in params.values()))
        self._call("ts3_sandwich_forward", f.data_ptr(), x.data_ptr(), _ptr(gate), ct.byref(p), n, y.data_ptr(), _ptr(out))
        return y, out

    def backward(self, f, y, gy, gamma_post, beta_post, scale, gate=None, gn=None, gamma_pre=None, dx=None):
        """Gradients of sum(gy * y) + sum(gn * out) for the forward's f, y and gate: (df, dx, dgate,
        {gamma_post, beta_post, scale, gamma_pre, beta_pre}).  gy may be None (zero).  gn goes with
        gamma_pre; without them there is no second norm and y may be None.  dgate and the last two
        gradients are None where their operands are."""
        n = self._rows(f, "f")
        for name, t in (("y", y), ("gy", gy), ("gate", gate), ("gn", gn), ("dx", dx)):
            if t is not None:
                self._rows(t, name, n)
        pre = gn is not None
        if pre is not (gamma_pre is not None) or (pre and y is None) or (gy is None and not pre):
            raise ValueError("gn, gamma_pre and y come together, and gy may be None only with them")
        params = {"gamma_post": gamma_post, "beta_post": beta_post, "scale": scale}
        if pre:
            params["gamma_pre"] = gamma_pre
        for name, t in params.items():
            self._vector(t, name)
        df = torch.empty_like(f)
        if dx is None:
            dx = torch.empty_like(f)
        dgate = None if gate is None else torch.empty_like(f)
        sums = torch.empty((5, self.C), device=f.device, dtype=torch.float32)
        base, row = sums.data_ptr(), 4 * self.C
        p = L.SandwichParams(*(t.data_ptr() for t in params.values()))
        d = L.SandwichParams(*(base + i * row for i in range(5 if pre else 3)))
        self._call("ts3_sandwich_backward", f.data_ptr(), _ptr(y), _ptr(gate), _ptr(gy), _ptr(gn), ct.byref(p), n,
                   df.data_ptr(), dx.data_ptr(), _ptr(dgate), ct.byref(d))
        grads = dict(zip(L.SANDWICH_NAMES, sums.unbind()))
        if not pre:
            grads.update(gamma_pre=None, beta_pre=None)
        return df, dx, dgate, grads


class Orthogonalizer(_Handle):
    """Orthogonalised updates of a list of gradients, as the Muon optimiser takes them: each matrix G
    becomes the result of `steps` Newton-Schulz steps

        X <- a X + (b A + c A A) X,  A = X X^T,  (a, b, c) = (3.4445, -4.7750, 2.0315)

    from X = G / (|G| + eps).  Tensors of more than two dimensions are batches of matrices."""

    _free = "ts3_orth_free"

    def __init__(self, steps=5, eps=1e-7):
        try:
            from . import _tensors
            self._table = _tensors.matrix_table
        except (ImportError, AttributeError) as e:
            raise RuntimeError("_tensors.so is missing or unusable: build it with __graft_entry__.build()") from e
        self.desc = L.OrthDesc(steps=steps, eps=eps)
        self._create(ct.byref(self.desc))

    def bytes(self) -> int:
        b = ct.c_int64()
        L.check(L.lib().ts3_orth_bytes(self.h, ct.byref(b)), "ts3_orth_bytes")
        return b.value

    def __call__(self, updates, out=None):
        """The list of results, of each tensor's type (float32 or bfloat16) and shape: new tensors, or
        those of the list `out`, which may be `updates` itself.  A result may share no memory with
        another tensor of either list."""
        if out is None:
            out = [torch.empty_like(t) for t in updates]
        table, device = self._table(updates, out)
        if device >= 0 and device != self.device:
            raise ValueError(f"tensors must be on cuda:{self.device}, where the Orthogonalizer was made")
        self._call("ts3_orth_matrices", table, len(updates))
        return out
