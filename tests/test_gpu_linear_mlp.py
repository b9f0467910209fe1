"""A gated MLP from the 8-bit operators together, and its training with MuonBP."""

import numpy as np
import pytest

from oracle import linear_oracle as O
from tests.gpu_harness import announce

pytestmark = pytest.mark.gpu


def _mlp(tokens, width, hidden, seed):
    import torch
    from examples.mlp_8bit import Mlp8
    from paper_2510_16981_amd import muonbp as mb
    g = torch.Generator(device="cuda").manual_seed(seed)
    linear = mb.Linear()
    w = [(torch.randn(r, c, generator=g, device="cuda") / r ** 0.5).bfloat16()
         for r, c in ((width, hidden), (width, hidden), (hidden, width))]
    x = torch.randn(tokens, width, generator=g, device="cuda").bfloat16()
    dy = (1e-3 * torch.randn(tokens, width, generator=g, device="cuda")).bfloat16()
    return linear, Mlp8(linear, w), x, dy


@pytest.mark.parametrize("sizes", [(1, 128, 256), (77, 200, 333), (700, 512, 1408)], ids=str)
def test_mlp_against_the_64_bit_chain(sizes):
    """Every result against the 64-bit chain that starts from what the forward
    pass kept in 8 bits.

    A result of n roundings to bf16 (2^-8 at most each) is within n 2^-8 in the
    2-norm: y has one; the weights' gradients three (dh, dgate or dup, dW).  dx
    goes through dgate and dup in 8 bits: a value that is d off rounds to
    another multiple of the step D with chance d / D, so the square of what the
    rounding moves is d D on average; two bf16 roundings (d = 2^-8 at most in
    all, rms) and a step of at most 2^-3 of the value give sqrt(2^-11) = 2.2%.
    A wrong operand, transpose or sign is off by 100%."""
    import torch
    announce(f"mlp {sizes}")
    linear, mlp, x, dy = _mlp(*sizes, seed=1)
    y, kept = mlp.forward(x)
    grads, dx = mlp.backward(dy, kept)

    def r8(v):
        return O.values(*O.quantize(v), v.shape[1])

    def w8(w):
        v = w.double().cpu().numpy()
        return O.values(*O.quantize(v, tile=True), v.shape[1])

    wg, wu, wd = (w8(w) for w in mlp.weights)
    xr, h, gate, up = (linear.restore(v, dtype=torch.float32).double().cpu().numpy() for v in kept)
    x64, dy64 = x.double().cpu().numpy(), dy.double().cpu().numpy()
    np.testing.assert_array_equal(xr, r8(x64))
    dh = r8(dy64) @ wd.T
    dgate, dup = O.gated_backward(dh, gate, up)
    want = {"y": (y, h @ wd, 2.0 ** -8),
            "dgate": (grads[0], xr.T @ dgate, 3 * 2.0 ** -8), "dup": (grads[1], xr.T @ dup, 3 * 2.0 ** -8),
            "ddown": (grads[2], h.T @ dy64, 2.0 ** -8),
            "dx": (dx, r8(dgate) @ wg.T + r8(dup) @ wu.T, 2.0 ** -5.5 + 2 * 2.0 ** -8)}
    for name, (got, ref, bound) in want.items():
        err = np.linalg.norm(got.double().cpu().numpy() - ref) / np.linalg.norm(ref)
        announce(f"{name} {err:.2e} of {bound:.2e}")
        assert err < bound, (name, err)
    linear.close()


def test_training_lowers_the_loss():
    from examples.mlp_8bit import train
    losses = train(tokens=256, width=256, hidden=704, steps=25)
    announce(f"losses {losses[0]:.4f} {losses[-1]:.4f}")
    assert np.isfinite(losses).all() and losses[-1] < 0.5 * losses[0]
