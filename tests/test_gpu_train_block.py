"""A pre-norm block with a gated feed-forward, as the training example puts it together from
the library's operators: its output and every gradient against the float64 oracle, and a
short training run that the clipping keeps in bounds.

The bar is the float32 acceptance bar, 1e-4 normwise: the gradients pass through the slice
softmax and its normalisation, whose conditioning the sums' rounding meets."""
import os
import sys

import numpy as np
import pytest

from gpu_helpers import banner, normwise, to_host

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("C,H,M,F,N,kind", [(64, 4, 32, 171, 3001, "silu"), (128, 8, 16, 96, 1500, "gelu")])
def test_block_against_the_oracle(C, H, M, F, N, kind):
    import torch

    import train_gated_block as example
    from oracle import backward as BW
    from oracle import physics_attention as PA
    from oracle import train as T
    banner(f"block C={C} H={H} M={M} F={F} N={N} {kind}")
    x, _ = example.surface(N, C)
    g = np.random.default_rng(1).standard_normal((N, C)).astype(np.float32)
    block = example.GatedBlock(C, H, M, F, N, seed=3, activation=kind, group_span=512)
    out = block.forward(torch.from_numpy(x).cuda())
    dx, grads = block.backward(torch.from_numpy(g).cuda())
    torch.cuda.synchronize()
    w = {k: to_host(v) for k, v in block.p.items()}
    x64, g64 = x.astype(np.float64), g.astype(np.float64)
    _, h1 = T.norm_forward(x64, None, w["g1"], w["n1"], 1e-5)
    a = PA.layer_forward_fast(h1, w, H, M, 2.0)
    y, h2 = T.norm_forward(a, x64, w["g2"], w["n2"], 1e-5)
    ref_out = y + T.gated_forward(h2, w, kind)
    ref = T.gated_backward(h2, w, kind, g64)
    dy, ref["dg2"], ref["dn2"] = T.norm_backward(y, ref.pop("dx"), g64, w["g2"], 1e-5)
    layer = BW.layer_backward(h1, w, dy, H, M, 2.0)
    ref_dx, ref["dg1"], ref["dn1"] = T.norm_backward(x64, layer.pop("dx"), dy, w["g1"], 1e-5)
    ref.update(layer)
    errors = {"out": normwise(to_host(out), ref_out), "dx": normwise(to_host(dx), ref_dx)}
    errors.update({k: normwise(to_host(v).reshape(ref["d" + k].shape), ref["d" + k]) for k, v in grads.items()})
    block.close()
    print({k: f"{v:.1e}" for k, v in errors.items()}, flush=True)
    assert set(grads) == set(w)
    assert max(errors.values()) <= 1e-4, errors


def test_training_lowers_the_loss_and_clips():
    import train_gated_block as example
    losses, norms = example.train(points=4000, steps=30)
    assert np.isfinite(losses).all() and np.isfinite(norms).all()
    assert losses[-1] < 0.7 * losses[0], losses
