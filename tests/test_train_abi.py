"""The training operators' refusals and layouts that need no GPU: bad descriptors and
arguments are rejected before any device call, with the documented status."""
import ctypes as ct

import pytest
import torch

from paper_2602_04940_amd import _lib as L

FAKE = 0x10000  # aligned, never dereferenced: the calls fail before touching it


def test_struct_layouts_match_header():
    assert ct.sizeof(L.GatedDesc) == 16 and ct.sizeof(L.NormDesc) == 12
    assert ct.sizeof(L.GatedWeights) == ct.sizeof(L.GatedGrads) == 6 * ct.sizeof(ct.c_void_p)
    assert ct.sizeof(L.ClipTensor) == 32 and L.ClipTensor.n.offset == 16 and L.ClipTensor.dtype.offset == 24


@pytest.mark.parametrize("kw,status", [
    (dict(C=0), L.TS3_ERR_INVALID_ARG),
    (dict(F=0), L.TS3_ERR_INVALID_ARG),
    (dict(F=-5), L.TS3_ERR_INVALID_ARG),
    (dict(C=40), L.TS3_ERR_UNSUPPORTED),      # not a multiple of 16
    (dict(C=272), L.TS3_ERR_UNSUPPORTED),
    (dict(F=65537), L.TS3_ERR_UNSUPPORTED),
    (dict(activation=2), L.TS3_ERR_INVALID_ARG),
    (dict(io_dtype=2), L.TS3_ERR_INVALID_ARG),
])
def test_bad_gated_descriptor(kw, status):
    d = dict(C=128, F=512, activation=L.TS3_SILU, io_dtype=L.TS3_BF16)
    d.update(kw)
    h = ct.c_void_p(1)
    assert L.lib().ts3_gated_create(ct.byref(L.GatedDesc(**d)), ct.byref(h)) == status
    assert h.value is None and L.lib().ts3_last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(C=0), L.TS3_ERR_INVALID_ARG),
    (dict(C=24), L.TS3_ERR_UNSUPPORTED),
    (dict(C=528), L.TS3_ERR_UNSUPPORTED),
    (dict(io_dtype=-1), L.TS3_ERR_INVALID_ARG),
    (dict(eps=-1e-5), L.TS3_ERR_INVALID_ARG),
    (dict(eps=float("nan")), L.TS3_ERR_INVALID_ARG),
    (dict(eps=float("inf")), L.TS3_ERR_INVALID_ARG),
])
def test_bad_norm_descriptor(kw, status):
    d = dict(C=128, io_dtype=L.TS3_BF16, eps=1e-5)
    d.update(kw)
    h = ct.c_void_p(1)
    assert L.lib().ts3_norm_create(ct.byref(L.NormDesc(**d)), ct.byref(h)) == status
    assert h.value is None


def test_null_handles():
    lib = L.lib()
    bad = L.TS3_ERR_INVALID_ARG
    assert lib.ts3_gated_create(None, None) == lib.ts3_norm_create(None, None) == lib.ts3_clip_create(None) == bad
    assert lib.ts3_gated_free(None) == lib.ts3_norm_free(None) == lib.ts3_clip_free(None) == L.TS3_OK
    assert lib.ts3_gated_bytes(None, None) == bad
    assert lib.ts3_gated_load(None, None, None) == bad
    assert lib.ts3_gated_forward(None, FAKE, 1, FAKE, None) == bad
    assert lib.ts3_gated_backward(None, FAKE, FAKE, 1, 1, FAKE, None, None) == bad
    assert lib.ts3_norm_forward(None, FAKE, None, FAKE, FAKE, 1, None, FAKE, None) == bad
    assert lib.ts3_norm_backward(None, FAKE, FAKE, None, FAKE, 1, FAKE, FAKE, FAKE, None) == bad
    assert lib.ts3_clip_gradients(None, None, 0, 1.0, None, None) == bad


def test_python_faces_check_their_tensors():
    from paper_2602_04940_amd import GatedWeights
    w = {"Wg": torch.zeros(16, 8), "Wu": torch.zeros(16, 8), "Wd": torch.zeros(8, 16)}
    assert GatedWeights(w, "fp32", "cpu").F == 8
    with pytest.raises(ValueError, match="Wd is missing"):
        GatedWeights({k: w[k] for k in ("Wg", "Wu")}, "fp32", "cpu")
    with pytest.raises(ValueError, match="Wd must be"):
        GatedWeights(dict(w, Wd=torch.zeros(16, 8)), "fp32", "cpu")
    with pytest.raises(ValueError, match="bg must be"):
        GatedWeights(dict(w, bg=torch.zeros(16)), "fp32", "cpu")
    with pytest.raises(KeyError):
        GatedWeights(w, "fp16", "cpu")


def test_tensor_tables_are_refused_before_any_device_call():
    from paper_2602_04940_amd import _tensors
    assert _tensors.clip_table([], None) == (b"", -1)
    for grads, out, error in (([torch.zeros(3)], None, ValueError), ([3.0], None, TypeError), ([], [torch.zeros(1)], ValueError),
                              (None, None, TypeError), ([], 5, TypeError)):
        with pytest.raises(error):
            _tensors.clip_table(grads, out)


@pytest.mark.parametrize("F", [1, 24, 512, 1024, 5000, 65536])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_default_tile_bounds_the_store(F, dtype):
    from paper_2602_04940_amd import GatedFeedForward
    ff = GatedFeedForward.__new__(GatedFeedForward)
    ff.F, ff.torch_dtype = F, dtype
    tile, row = ff.default_tile(), 3 * ((F + 31) // 32 * 32) * (2 if dtype is torch.bfloat16 else 4)
    assert tile >= 8192 and tile * row <= 1 << 33
    assert tile >= 1 << 18 or F >= 2048
