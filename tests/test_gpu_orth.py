"""Orthogonalised updates on the GPU by tiles of 128, which the lists of test_gpu_conditioned.py are too short for, against
the float64 reference.  Bars as there, from the products' operands and sums."""
import math

import numpy as np
import pytest

from gpu_helpers import banner, to_host
from orth_shapes import STREAM
from test_gpu_conditioned import U, _flat, _frobenius

pytestmark = pytest.mark.gpu


def _bar(shape, norm, dtype):
    r, c = min(shape[-2:]), max(shape[-2:])
    delta = 2.0 ** -22 + math.sqrt(r + c) * U
    bar = 16 * delta if c >= 2 * r else 6 * 3.4445 ** 5 * delta / norm
    return bar + (2.0 ** -8 if dtype == "bf16" else 0.0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shapes", STREAM)
def test_lists_of_many_or_large_matrices(shapes, dtype):
    import torch
    from oracle import conditioned as R
    from paper_2602_04940_amd import Orthogonalizer
    banner(f"orth {len(shapes)} tensors, first {shapes[0]} {dtype}")
    parts, views, _ = _flat(shapes, dtype, 5, scale=1e-3)
    with Orthogonalizer() as orth:
        out = orth(views)
        again = orth(views)
        torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, again))
    worst = 0.0
    for p, t in zip(parts, out):
        ref, got = R.orthogonalise(p), to_host(t)
        assert got.shape == p.shape
        for g, e in zip(got.reshape(-1, *p.shape[-2:]), ref.reshape(-1, *p.shape[-2:])):
            err, bar = _frobenius(g, e), _bar(p.shape, np.linalg.norm(e), dtype)
            worst = max(worst, err / bar)
            assert err <= bar, (p.shape, err, bar)
    print(f"worst of the bars {worst:.3f}", flush=True)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_bad_matrices_stay_alone_in_a_long_list(dtype):
    """A tile of a matrix of 64 rows reads 64 rows of the next matrix, or behind the last one: not-a-numbers there reach
    nothing but their own matrix, bit for bit."""
    import torch
    from paper_2602_04940_amd import Orthogonalizer
    _, views, _ = _flat([(64, 128)] * 200, dtype, 6)
    bad = [0, 1, 50, 199]
    with Orthogonalizer() as orth:
        clean = orth(views)
        for i in bad:
            views[i][3, 5] = math.nan
        out = orth(views)
        for i in bad:
            views[i].zero_()
        zeros = orth(views)
        torch.cuda.synchronize()
    for i in range(200):
        if i in bad:
            assert out[i].isnan().any() and (zeros[i] == 0).all()
        else:
            assert torch.equal(out[i], clean[i]) and torch.equal(zeros[i], clean[i]), i
