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


class _OnGpu:
    """What the operators ask of a tensor, without a GPU."""

    def __init__(self, shape, dtype, index, address=1 << 20):
        self.shape, self.dtype, self.is_cuda = shape, dtype, True
        self.device, self._address = torch.device("cuda", index), address

    def get_device(self):
        return self.device.index

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self._address


def _handle(kind, device, **fields):
    h = kind.__new__(kind)
    h.device, h.h = device, None
    for k, v in fields.items():
        setattr(h, k, v)
    return h


def test_tensors_of_another_device_are_refused():
    from paper_2602_04940_amd import GatedFeedForward, GatedWeights, GradClip, ResidualNorm
    bf = torch.bfloat16

    def rows(i):
        return _OnGpu((4, 16), bf, i)

    def vector(i):
        return _OnGpu((16,), torch.float32, i)
    ff = _handle(GatedFeedForward, 1, C=16, F=8, torch_dtype=bf)
    norm = _handle(ResidualNorm, 1, C=16, torch_dtype=bf)
    here, away, gm = rows(1), rows(0), vector(1)
    weights = GatedWeights.__new__(GatedWeights)
    weights.C, weights.F, weights.torch_dtype = 16, 8, bf
    weights.t = {n: _OnGpu((1,), bf, 0 if n == "bd" else 1) for n in L.GATED_NAMES}
    for call in (lambda: ff.forward(away), lambda: ff.forward(here, out=away), lambda: ff.backward(here, away),
                 lambda: ff.backward(away, here), lambda: ff.backward(here, here, dx=away), lambda: ff.load(weights),
                 lambda: norm.forward(away, gm, gm), lambda: norm.forward(here, vector(0), gm),
                 lambda: norm.forward(here, gm, vector(0)), lambda: norm.forward(here, gm, gm, residual=away),
                 lambda: norm.forward(here, gm, gm, y=away), lambda: norm.forward(here, gm, gm, out=away),
                 lambda: norm.backward(here, away, gm), lambda: norm.backward(here, here, vector(0)),
                 lambda: norm.backward(here, here, gm, residual_grad=away), lambda: norm.backward(here, here, gm, dx=away),
                 lambda: _handle(GradClip, 1, _table=lambda grads, out: (b"", 0))([None], 1.0)):
        with pytest.raises(ValueError, match="cuda:1"):
            call()
    host = GatedWeights({"Wg": torch.zeros(16, 8), "Wu": torch.zeros(16, 8), "Wd": torch.zeros(8, 16)}, "bf16", "cpu")
    with pytest.raises(ValueError, match="cuda:1"):
        ff.load(host)


def test_calls_run_on_the_handles_device(monkeypatch):
    """The library launches on the current device: a call on a handle of another one switches to
    it, takes that device's stream, and switches back."""
    from paper_2602_04940_amd import GatedFeedForward, train
    current, calls = [0], []

    class Device:
        def __init__(self, i):
            self.i = i

        def __enter__(self):
            self.before, current[0] = current[0], self.i

        def __exit__(self, *a):
            current[0] = self.before

    class Library:
        def ts3_gated_forward(self, *args):
            calls.append((current[0], args))
            return L.TS3_OK
    monkeypatch.setattr(train, "_current_device", lambda: current[0])
    monkeypatch.setattr(train, "_raw_stream", lambda i: 100 * current[0] + i)
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(L, "lib", Library)
    for device in (0, 1):
        ff = _handle(GatedFeedForward, device, C=16, F=8, torch_dtype=torch.bfloat16)
        x, out = (_OnGpu((4, 16), torch.bfloat16, device, a) for a in (1 << 20, 1 << 21))
        assert ff.forward(x, out=out) is out
        assert calls.pop() == (device, (None, 1 << 20, 4, 1 << 21, 101 * device)) and current == [0]
