"""ctypes binding of include/ts3.h: argument marshalling only.

Every computation happens in libts3.so's HIP kernels.  The library must have
been built (``__graft_entry__.build()``); loading fails loudly otherwise.
"""
from __future__ import annotations

import ctypes as ct
import os

from .build import LIB

TS3_OK, TS3_ERR_INVALID_ARG, TS3_ERR_BAD_STATE, TS3_ERR_OUT_OF_MEMORY, TS3_ERR_HIP, TS3_ERR_UNSUPPORTED = range(6)
TS3_FP32, TS3_BF16 = 0, 1
TS3_S_RAW, TS3_D, TS3_S, TS3_S1, TS3_ZP, TS3_T_RAW = range(6)


TS3_ACCUM_FP32, TS3_ACCUM_FP64 = 0, 1


class Desc(ct.Structure):
    _fields_ = [("C", ct.c_int32), ("H", ct.c_int32), ("M", ct.c_int32), ("dh", ct.c_int32),
                ("temperature", ct.c_float), ("eps", ct.c_float), ("io_dtype", ct.c_int32),
                ("accum", ct.c_int32), ("group_span", ct.c_int64), ("max_points", ct.c_int64)]


class Weights(ct.Structure):
    _fields_ = [(n, ct.c_void_p) for n in ("W2", "b2", "W1", "b1", "Wq", "Wk", "Wv", "W3", "b3")]


WEIGHT_NAMES = [n for n, _ in Weights._fields_]


class Grads(ct.Structure):
    _fields_ = [(n, ct.c_void_p) for n in ("dW2", "db2", "dW1", "db1", "dWq", "dWk", "dWv", "dW3", "db3")]


GRAD_NAMES = [n for n, _ in Grads._fields_]

BLOCK_EXTRA_NAMES = ("ln1_g", "ln1_b", "ln2_g", "ln2_b", "Wa", "ba", "Wb", "bb")


class BlockWeights(ct.Structure):
    _fields_ = [("pa", Weights)] + [(n, ct.c_void_p) for n in BLOCK_EXTRA_NAMES]


TS3_SILU, TS3_GELU = 0, 1


class GatedDesc(ct.Structure):
    _fields_ = [("C", ct.c_int32), ("F", ct.c_int32), ("activation", ct.c_int32), ("io_dtype", ct.c_int32)]


GATED_NAMES = ("Wg", "bg", "Wu", "bu", "Wd", "bd")


class GatedWeights(ct.Structure):
    _fields_ = [(n, ct.c_void_p) for n in GATED_NAMES]


class GatedGrads(ct.Structure):
    _fields_ = [("d" + n, ct.c_void_p) for n in GATED_NAMES]


class NormDesc(ct.Structure):
    _fields_ = [("C", ct.c_int32), ("io_dtype", ct.c_int32), ("eps", ct.c_float)]


class ClipTensor(ct.Structure):
    _fields_ = [("src", ct.c_void_p), ("dst", ct.c_void_p), ("n", ct.c_int64), ("dtype", ct.c_int32),
                ("reserved", ct.c_int32)]


class CrossDesc(ct.Structure):
    _fields_ = [("H", ct.c_int32), ("Hkv", ct.c_int32), ("D", ct.c_int32), ("io_dtype", ct.c_int32), ("scale", ct.c_float)]


class View(ct.Structure):
    _fields_ = [("p", ct.c_void_p), ("batch", ct.c_int64), ("row", ct.c_int64), ("head", ct.c_int64)]


class CrossInputs(ct.Structure):
    _fields_ = [("B", ct.c_int32), ("N", ct.c_int32), ("S", ct.c_int32), ("q", View), ("k", View), ("v", View),
                ("lengths", ct.c_void_p), ("mask", ct.c_void_p)]


class SandwichDesc(ct.Structure):
    _fields_ = [("C", ct.c_int32), ("io_dtype", ct.c_int32), ("eps", ct.c_float)]


SANDWICH_NAMES = ("gamma_post", "beta_post", "scale", "gamma_pre", "beta_pre")


class SandwichParams(ct.Structure):
    """Of the parameters, and of their gradients."""
    _fields_ = [(n, ct.c_void_p) for n in SANDWICH_NAMES]


class OrthDesc(ct.Structure):
    _fields_ = [("steps", ct.c_int32), ("eps", ct.c_float)]


class Matrix(ct.Structure):
    _fields_ = [("src", ct.c_void_p), ("dst", ct.c_void_p), ("rows", ct.c_int32), ("cols", ct.c_int32),
                ("batch", ct.c_int32), ("dtype", ct.c_int32)]


_P = ct.c_void_p
# name -> (restype, argtypes); must match include/ts3.h
SIGNATURES = {
    "ts3_state_create": (ct.c_int, [ct.POINTER(Desc), ct.POINTER(_P)]),
    "ts3_state_free": (ct.c_int, [_P]),
    "ts3_state_bytes": (ct.c_int, [_P, ct.POINTER(ct.c_int64)]),
    "ts3_state_projected": (ct.c_int, [_P, ct.POINTER(ct.c_int32)]),
    "ts3_state_reset": (ct.c_int, [_P, _P]),
    "ts3_slice_accumulate": (ct.c_int, [_P, ct.POINTER(Weights), _P, ct.c_int64, ct.c_int64, _P]),
    "ts3_slice_finalize": (ct.c_int, [_P, ct.POINTER(Weights), _P]),
    "ts3_token_attention": (ct.c_int, [_P, ct.POINTER(Weights), _P]),
    "ts3_deslice": (ct.c_int, [_P, ct.POINTER(Weights), _P, ct.c_int64, _P, _P]),
    "ts3_layer_forward": (ct.c_int, [_P, ct.POINTER(Weights), _P, ct.c_int64, ct.c_int64, ct.c_int64, _P, _P]),
    "ts3_layer_forward_noalloc": (ct.c_int, [ct.POINTER(Desc), ct.POINTER(Weights), _P, ct.c_int64, ct.c_int64,
                                             ct.c_int64, _P, _P]),
    "ts3_layer_backward": (ct.c_int, [_P, ct.POINTER(Weights), _P, _P, ct.c_int64, ct.c_int64, _P,
                                      ct.POINTER(Grads), _P]),
    "ts3_state_get": (ct.c_int, [_P, ct.c_int32, _P, ct.c_int64, _P]),
    "ts3_state_get_spans": (ct.c_int, [_P, ct.c_int64, ct.c_int64, _P, ct.c_int64, _P]),
    "ts3_state_set": (ct.c_int, [_P, ct.POINTER(Weights), ct.c_int32, _P, ct.c_int64, _P, _P]),
    "ts3_stack_create": (ct.c_int, [ct.POINTER(Desc), ct.c_int32, ct.c_int32, ct.POINTER(_P)]),
    "ts3_stack_free": (ct.c_int, [_P]),
    "ts3_stack_bytes": (ct.c_int, [_P, ct.POINTER(ct.c_int64)]),
    "ts3_stack_layer": (ct.c_int, [_P, ct.c_int32, ct.POINTER(_P)]),
    "ts3_stack_forward": (ct.c_int, [_P, ct.POINTER(BlockWeights), _P, ct.c_int64, ct.c_int64, ct.c_int64, _P]),
    "ts3_stack_decode": (ct.c_int, [_P, ct.POINTER(BlockWeights), _P, ct.c_int64, ct.c_int64, _P]),
    "ts3_stack_feedforward": (ct.c_int, [_P, ct.POINTER(BlockWeights), ct.c_int32, _P, _P, ct.c_int64, _P, _P]),
    "ts3_gated_create": (ct.c_int, [ct.POINTER(GatedDesc), ct.POINTER(_P)]),
    "ts3_gated_free": (ct.c_int, [_P]),
    "ts3_gated_bytes": (ct.c_int, [_P, ct.POINTER(ct.c_int64)]),
    "ts3_gated_load": (ct.c_int, [_P, ct.POINTER(GatedWeights), _P]),
    "ts3_gated_forward": (ct.c_int, [_P, _P, ct.c_int64, _P, _P]),
    "ts3_gated_backward": (ct.c_int, [_P, _P, _P, ct.c_int64, ct.c_int64, _P, ct.POINTER(GatedGrads), _P]),
    "ts3_norm_create": (ct.c_int, [ct.POINTER(NormDesc), ct.POINTER(_P)]),
    "ts3_norm_free": (ct.c_int, [_P]),
    "ts3_norm_forward": (ct.c_int, [_P, _P, _P, _P, _P, ct.c_int64, _P, _P, _P]),
    "ts3_norm_backward": (ct.c_int, [_P, _P, _P, _P, _P, ct.c_int64, _P, _P, _P, _P]),
    "ts3_clip_create": (ct.c_int, [ct.POINTER(_P)]),
    "ts3_clip_free": (ct.c_int, [_P]),
    "ts3_clip_gradients": (ct.c_int, [_P, _P, ct.c_int32, ct.c_float, _P, _P]),
    "ts3_cross_create": (ct.c_int, [ct.POINTER(CrossDesc), ct.POINTER(_P)]),
    "ts3_cross_free": (ct.c_int, [_P]),
    "ts3_cross_bytes": (ct.c_int, [_P, ct.POINTER(ct.c_int64)]),
    "ts3_cross_forward": (ct.c_int, [_P, _P, _P, _P, _P]),
    "ts3_cross_backward": (ct.c_int, [_P, _P, _P, _P, _P, _P, _P, _P, _P]),
    "ts3_sandwich_create": (ct.c_int, [ct.POINTER(SandwichDesc), ct.POINTER(_P)]),
    "ts3_sandwich_free": (ct.c_int, [_P]),
    "ts3_sandwich_forward": (ct.c_int, [_P, _P, _P, _P, _P, ct.c_int64, _P, _P, _P]),
    "ts3_sandwich_backward": (ct.c_int, [_P, _P, _P, _P, _P, _P, _P, ct.c_int64, _P, _P, _P, _P, _P]),
    "ts3_orth_create": (ct.c_int, [ct.POINTER(OrthDesc), ct.POINTER(_P)]),
    "ts3_orth_free": (ct.c_int, [_P]),
    "ts3_orth_bytes": (ct.c_int, [_P, ct.POINTER(ct.c_int64)]),
    "ts3_orth_matrices": (ct.c_int, [_P, _P, ct.c_int32, _P]),
    "ts3_status_string": (ct.c_char_p, [ct.c_int]),
    "ts3_last_error": (ct.c_char_p, []),
}

_lib = None


class TS3Error(RuntimeError):
    def __init__(self, status: int, where: str, detail: str):
        super().__init__(f"{where}: status {status} ({detail})")
        self.status = status


def lib() -> ct.CDLL:
    """The loaded library; TS3_LIB may name another build of it (default: in-tree)."""
    global _lib
    if _lib is None:
        path = os.environ.get("TS3_LIB", LIB)
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: build it with __graft_entry__.build() "
                               "(the layer has no fallback path)")
        L = ct.CDLL(path)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _lib = L
    return _lib


def check(status: int, where: str) -> None:
    if status != TS3_OK:
        L = lib()
        raise TS3Error(status, where, f"{L.ts3_status_string(status).decode()}: {L.ts3_last_error().decode()}")
