"""Refusals and layouts of a conditioned block's operators that need no GPU: bad descriptors and
arguments are rejected before any device call, with the documented status.  The library looks at
addresses only here; none is read."""
import ctypes as ct

import pytest
import torch

from paper_2602_04940_amd import _lib as L
from test_train_abi import _handle, _OnGpu

BAD, UNSUPPORTED = L.TS3_ERR_INVALID_ARG, L.TS3_ERR_UNSUPPORTED
MB = 1 << 20


def test_struct_layouts_match_header_and_packing():
    from paper_2602_04940_amd import conditioned as C
    assert ct.sizeof(L.View) == C._VIEW.size == 32
    assert ct.sizeof(L.CrossInputs) == C._INPUTS.size == 128 and L.CrossInputs.q.offset == 16
    assert L.CrossInputs.lengths.offset == 112 and ct.sizeof(L.CrossDesc) == 20
    assert ct.sizeof(L.SandwichDesc) == 12 and ct.sizeof(L.SandwichParams) == 40
    assert ct.sizeof(L.OrthDesc) == 8 and ct.sizeof(L.Matrix) == 32 and L.Matrix.dtype.offset == 28
    packed = C._INPUTS.pack(1, 2, 3, *range(10, 24))
    s = L.CrossInputs.from_buffer_copy(packed)
    assert (s.B, s.N, s.S, s.q.p, s.k.batch, s.v.head, s.lengths, s.mask) == (1, 2, 3, 10, 15, 21, 22, 23)


@pytest.mark.parametrize("kw,status", [
    (dict(H=0), BAD), (dict(Hkv=0), BAD), (dict(D=-16), BAD), (dict(Hkv=3), BAD), (dict(io_dtype=2), BAD),
    (dict(scale=-1.0), BAD), (dict(scale=float("nan")), BAD), (dict(scale=float("inf")), BAD),
    (dict(D=24), UNSUPPORTED), (dict(D=144), UNSUPPORTED), (dict(H=2048, Hkv=2048), UNSUPPORTED),
])
def test_bad_cross_descriptor(kw, status):
    h = ct.c_void_p(1)
    d = L.CrossDesc(**dict(dict(H=8, Hkv=4, D=32, io_dtype=L.TS3_BF16, scale=0.0), **kw))
    assert L.lib().ts3_cross_create(ct.byref(d), ct.byref(h)) == status
    assert h.value is None and L.lib().ts3_last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(C=0), BAD), (dict(C=24), UNSUPPORTED), (dict(C=528), UNSUPPORTED), (dict(io_dtype=5), BAD), (dict(eps=-1.0), BAD),
    (dict(eps=float("nan")), BAD),
])
def test_bad_sandwich_descriptor(kw, status):
    h = ct.c_void_p(1)
    d = L.SandwichDesc(**dict(dict(C=128, io_dtype=L.TS3_BF16, eps=1e-5), **kw))
    assert L.lib().ts3_sandwich_create(ct.byref(d), ct.byref(h)) == status and h.value is None


@pytest.mark.parametrize("kw", [dict(steps=0), dict(steps=65), dict(eps=-1.0), dict(eps=float("inf"))])
def test_bad_orth_descriptor(kw):
    h = ct.c_void_p(1)
    assert L.lib().ts3_orth_create(ct.byref(L.OrthDesc(**dict(dict(steps=5, eps=1e-7), **kw))), ct.byref(h)) == BAD
    assert h.value is None


def _cross(**kw):
    """A handle, which takes no device memory before its first split call."""
    h = ct.c_void_p()
    d = L.CrossDesc(**dict(dict(H=8, Hkv=4, D=32, io_dtype=L.TS3_BF16, scale=0.0), **kw))
    assert L.lib().ts3_cross_create(ct.byref(d), ct.byref(h)) == L.TS3_OK
    return h


def _cross_inputs(**kw):
    """Arrays 16 MB apart, contiguous, of 2 samples of 3 points and 5 states."""
    row, kv = 8 * 32, 4 * 32
    f = dict(B=2, N=3, S=5, q=L.View(16 * MB, 3 * row, row, 32), k=L.View(32 * MB, 5 * kv, kv, 32),
             v=L.View(48 * MB, 5 * kv, kv, 32), lengths=None, mask=None)
    f.update(kw)
    return L.CrossInputs(**f)


OUT, LSE = 64 * MB, 80 * MB


@pytest.mark.parametrize("kw,out,lse,status", [
    (dict(B=-1), OUT, LSE, BAD), (dict(N=-1), OUT, LSE, BAD), (dict(S=-1), OUT, LSE, BAD),
    (dict(q=L.View(0, 768, 256, 32)), OUT, LSE, BAD),
    (dict(q=L.View(16 * MB + 8, 768, 256, 32)), OUT, LSE, BAD),           # not 16-byte aligned
    (dict(q=L.View(16 * MB, 768, 257, 32)), OUT, LSE, BAD),               # a stride that is not
    (dict(q=L.View(16 * MB, 768, -256, 32)), OUT, LSE, BAD),
    (dict(k=L.View(32 * MB, 1 << 41, 128, 32)), OUT, LSE, BAD),
    (dict(v=L.View(0, 640, 128, 32)), OUT, LSE, BAD),
    (dict(lengths=96 * MB + 2), OUT, LSE, BAD),
    (dict(), 0, LSE, BAD), (dict(), OUT + 8, LSE, BAD), (dict(), OUT, 0, BAD), (dict(), OUT, LSE + 2, BAD),
    (dict(), 16 * MB, LSE, BAD), (dict(), 16 * MB + 1536 * 2 - 16, LSE, BAD),   # out over q's end
    (dict(), OUT, OUT, BAD), (dict(), OUT, 32 * MB, BAD), (dict(lengths=OUT + 16), OUT, LSE, BAD),
    (dict(mask=LSE + 4), OUT, LSE, BAD),
    (dict(N=(1 << 30) - 400), OUT, LSE, UNSUPPORTED), (dict(S=(1 << 31) - 1000), OUT, LSE, UNSUPPORTED),
    (dict(B=1 << 23), OUT, LSE, UNSUPPORTED), (dict(B=8, N=1 << 28), OUT, LSE, UNSUPPORTED),
])
def test_cross_forward_refusals(kw, out, lse, status):
    h = _cross()
    assert L.lib().ts3_cross_forward(h, ct.byref(_cross_inputs(**kw)), out, lse, None) == status
    assert L.lib().ts3_last_error()


def test_cross_backward_refusals_and_calls_of_nothing():
    lib, h = L.lib(), _cross()
    g, ok = L.View(96 * MB, 768, 256, 32), (OUT, LSE, 112 * MB, 128 * MB, 144 * MB)

    def call(inputs=None, g=g, args=ok):
        out, lse, dq, dk, dv = args
        return lib.ts3_cross_backward(h, ct.byref(inputs or _cross_inputs()), out, lse, ct.byref(g), dq, dk, dv, None)
    for i in range(5):
        for bad in (0, ok[i] + 2):
            assert call(args=ok[:i] + (bad,) + ok[i + 1:]) == BAD
    for i in (2, 3, 4):  # an output over an input, or over another output
        for over in (16 * MB, 32 * MB, 48 * MB, 96 * MB, OUT, LSE, ok[2 + (i - 1) % 3]):
            assert call(args=ok[:i] + (over,) + ok[i + 1:]) == BAD
    assert call(g=L.View(96 * MB, 768, 255, 32)) == BAD and call(g=L.View(0, 768, 256, 32)) == BAD
    assert call(inputs=_cross_inputs(B=0), args=(0, 0, 0, 0, 0)) == L.TS3_OK
    assert lib.ts3_cross_forward(h, ct.byref(_cross_inputs(B=0)), 0, 0, None) == L.TS3_OK
    assert lib.ts3_cross_forward(h, ct.byref(_cross_inputs(N=0)), 0, 0, None) == L.TS3_OK


def test_null_handles():
    lib = L.lib()
    assert lib.ts3_cross_create(None, None) == lib.ts3_sandwich_create(None, None) == lib.ts3_orth_create(None, None) == BAD
    assert lib.ts3_cross_free(None) == lib.ts3_sandwich_free(None) == lib.ts3_orth_free(None) == L.TS3_OK
    assert lib.ts3_cross_bytes(None, None) == lib.ts3_orth_bytes(None, None) == BAD
    assert lib.ts3_cross_forward(None, None, MB, MB, None) == lib.ts3_cross_forward(_cross(), None, MB, MB, None) == BAD
    assert lib.ts3_cross_backward(None, None, MB, MB, None, MB, MB, MB, None) == BAD
    assert lib.ts3_sandwich_forward(None, MB, MB, None, None, 1, MB, None, None) == BAD
    assert lib.ts3_sandwich_backward(None, MB, MB, None, MB, None, None, 1, MB, MB, None, None, None) == BAD
    assert lib.ts3_orth_matrices(None, None, 0, None) == BAD


def _orth():
    h = ct.c_void_p()
    assert L.lib().ts3_orth_create(ct.byref(L.OrthDesc(steps=5, eps=1e-7)), ct.byref(h)) == L.TS3_OK
    return h


def _matrices(*rows):
    fields = [dict(dict(src=MB, dst=64 * MB, rows=4, cols=6, batch=1, dtype=L.TS3_FP32), **r) for r in rows]
    return (L.Matrix * len(fields))(*(L.Matrix(**f) for f in fields)), len(fields)


@pytest.mark.parametrize("row,status", [
    (dict(src=0), BAD), (dict(dst=0), BAD), (dict(src=MB + 2), BAD), (dict(dst=MB + 1, dtype=L.TS3_BF16), BAD),
    (dict(rows=-1), BAD), (dict(cols=-1), BAD), (dict(batch=-1), BAD), (dict(dtype=2), BAD), (dict(rows=32769), UNSUPPORTED),
    (dict(cols=32769), UNSUPPORTED), (dict(batch=1 << 24, dst=1 << 40), UNSUPPORTED),
    (dict(rows=32768, cols=32768, batch=(1 << 31) - 1), UNSUPPORTED),
])
def test_orth_refusals(row, status):
    assert L.lib().ts3_orth_matrices(_orth(), *_matrices(row), None) == status and L.lib().ts3_last_error()


def test_orth_results_that_overlap_and_empty_lists():
    lib, h = L.lib(), _orth()
    for second in (dict(), dict(dst=64 * MB + 92), dict(src=2 * MB, dst=64 * MB - 4), dict(src=2 * MB, dst=MB + 92),
                   dict(src=64 * MB + 92, dst=2 * MB), dict(src=2 * MB, dst=2 * MB + 4)):
        assert lib.ts3_orth_matrices(h, *_matrices(dict(), second), None) == BAD
    assert lib.ts3_orth_matrices(h, None, 0, None) == L.TS3_OK
    assert lib.ts3_orth_matrices(h, *_matrices(dict(rows=0), dict(batch=0, src=0, dst=0)), None) == L.TS3_OK
    assert lib.ts3_orth_matrices(h, None, 1, None) == lib.ts3_orth_matrices(h, *_matrices(dict())[:1], -1, None) == BAD
    assert lib.ts3_orth_matrices(h, _matrices(dict())[0], 16385, None) == BAD


def test_matrix_tables():
    from paper_2602_04940_amd import _tensors
    assert _tensors.matrix_table([], []) == (b"", -1)
    t = torch.zeros(3, 4)
    for a, b, error in (([t], [t], ValueError), ([3.0], [t], TypeError), ([t], [], ValueError), (None, [], TypeError),
                        ([], None, TypeError), ([t], 5, TypeError)):
        with pytest.raises(error):
            _tensors.matrix_table(a, b)


class _View(_OnGpu):
    def __init__(self, shape, dtype, index, stride=None):
        super().__init__(shape, dtype, index)
        self.shape = torch.Size(shape)
        self._stride = stride or tuple(int(torch.Size(shape[i + 1:]).numel()) for i in range(len(shape)))

    def stride(self):
        return self._stride

    def dim(self):
        return len(self.shape)


def test_python_faces_refuse_wrong_tensors():
    from paper_2602_04940_amd import CrossAttention, SandwichNorm
    bf = torch.bfloat16
    a = _handle(CrossAttention, 1, H=4, Hkv=2, D=16, torch_dtype=bf)

    def q(i=1, **kw):
        return _View(**dict(dict(shape=(2, 3, 4, 16), dtype=bf, index=i), **kw))

    def k(i=1, **kw):
        return _View(**dict(dict(shape=(2, 5, 2, 16), dtype=bf, index=i), **kw))
    lse, lens, mask = _View((2, 4, 3), torch.float32, 1), _View((2,), torch.int32, 1), _View((2, 5), torch.bool, 1)
    calls = [dict(q=q(0)), dict(k=k(0)), dict(v=k(0)), dict(q=q(dtype=torch.float32)), dict(v=k(shape=(2, 6, 2, 16))),
             dict(k=k(shape=(2, 5, 4, 16))), dict(q=q(shape=(2, 3, 64))), dict(q=q(stride=(384, 128, 32, 2))),
             dict(lengths=_View((3,), torch.int32, 1)), dict(lengths=_View((2,), torch.int64, 1)),
             dict(lengths=_View((2,), torch.int32, 0)), dict(mask=_View((2, 5), torch.uint8, 1)),
             dict(mask=_View((2, 4), torch.bool, 1)), dict(mask=_View((2, 5), torch.bool, 0)), dict(out=q(0)),
             dict(out=q(), lse=_View((2, 3, 4), torch.float32, 1))]
    for kw in calls:
        with pytest.raises(ValueError):
            a.forward(**dict(dict(q=q(), k=k(), v=k(), lengths=lens, mask=mask), **kw))
    for kw in (dict(out=q(0)), dict(lse=_View((2, 4, 3), torch.float32, 0)), dict(g=q(0)), dict(g=k()), dict(dq=q(0))):
        with pytest.raises(ValueError):
            a.backward(**dict(dict(q=q(), k=k(), v=k(), out=q(), lse=lse, g=q()), **kw))
    for scale in (0.0, -1.0, float("nan"), float("inf"), 1e-60):
        with pytest.raises(ValueError):
            CrossAttention(4, 16, scale=scale)
    n = _handle(SandwichNorm, 1, C=16, torch_dtype=bf)

    def rows(i=1):
        return _OnGpu((4, 16), bf, i)

    def vec(i=1):
        return _OnGpu((16,), torch.float32, i)
    good = dict(f=rows(), x=rows(), gamma_post=vec(), beta_post=vec(), scale=vec(), gate=rows(), gamma_pre=vec(), beta_pre=vec(),
                y=rows())
    for kw in [{name: (rows if name in ("f", "x", "gate", "y") else vec)(0)} for name in good] + [
            dict(beta_pre=None), dict(gamma_pre=None), dict(gamma_pre=None, beta_pre=None, out=rows()), dict(out=rows(0))]:
        with pytest.raises(ValueError):
            n.forward(**dict(good, **kw))
    good = dict(f=rows(), y=rows(), gy=rows(), gamma_post=vec(), beta_post=vec(), scale=vec(), gate=rows(), gn=rows(),
                gamma_pre=vec())
    for kw in [{name: (rows if name in ("f", "y", "gy", "gate", "gn") else vec)(0)} for name in good] + [
            dict(gn=None), dict(gamma_pre=None), dict(y=None), dict(gy=None, gn=None, gamma_pre=None), dict(dx=rows(0))]:
        with pytest.raises(ValueError):
            n.backward(**dict(good, **kw))
