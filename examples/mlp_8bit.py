"""Train a gated MLP with 8-bit linear layers and MuonBP.

    python examples/mlp_8bit.py [--tokens 512] [--width 512] [--hidden 1408] [--steps 30]

The MLP learns the outputs of another one (y = W_down^T (silu(W_gate^T x) W_up^T
x)) on a fixed batch of inputs.  Its bf16 weights are requantized after each step; the
activations that the backward pass needs are kept in 8 bits:

    forward    x8 = quantize(x); gate, up = product(x8, w8^T)
               h8, gate8, up8 = gated_forward(gate, up); y = product(h8, down8^T)
    backward   dy8 = quantize(dy); dh = product(dy8, down8)
               dgate, dup, dgate8, dup8 = gated_backward(dh, gate8, up8)
               dW = weight_grad(x8 or h8, dy, dgate or dup)
               dx = product(dgate8, gate8) + product(dup8, up8)
    update     MuonBP on the three weights
"""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2510_16981_amd import muonbp as mb  # noqa: E402


class Mlp8:
    """W_gate, W_up (width x hidden) and W_down (hidden x width), bf16, with
    their 8-bit forms: w[k] for the input gradient, wt[k] for the forward."""

    def __init__(self, linear, weights):
        self.linear, self.weights = linear, weights
        self.quantize()

    def quantize(self):
        self.w, self.wt = zip(*(self.linear.quantize_weight(w) for w in self.weights))

    def forward(self, x):
        lin = self.linear
        x8 = lin.quantize(x)
        gate, up = lin.product(x8, self.wt[0]), lin.product(x8, self.wt[1])
        h8, gate8, up8 = lin.gated_forward(gate, up, blocks=True)
        return lin.product(h8, self.wt[2]), (x8, h8, gate8, up8)

    def backward(self, dy, kept, input_grad=True):
        """(gradients of the weights, dx)."""
        lin, (x8, h8, gate8, up8) = self.linear, kept
        dh = lin.product(lin.quantize(dy), self.w[2])
        dgate, dup, dgate8, dup8 = lin.gated_backward(dh, gate8, up8, blocks=True)
        grads = [lin.weight_grad(x8, dgate), lin.weight_grad(x8, dup), lin.weight_grad(h8, dy)]
        dx = None
        if input_grad:  # summed in fp32, rounded by the caller
            dx = lin.product(dgate8, self.w[0], dtype=torch.float32)
            lin.product(dup8, self.w[1], out=dx, accumulate=True)
        return grads, dx


def train(tokens=512, width=512, hidden=1408, steps=30, lr=0.02, seed=0):
    """The losses of `steps` steps."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def weights(scale):
        return [(scale * torch.randn(r, c, generator=g, device="cuda") / r ** 0.5).bfloat16()
                for r, c in ((width, hidden), (width, hidden), (hidden, width))]

    linear = mb.Linear()
    teacher, student = Mlp8(linear, weights(1.0)), Mlp8(linear, weights(0.5))
    opt = mb.MuonBP([(width, hidden, 1, 4), (width, hidden, 1, 4), (hidden, width, 4, 1)], period=5,
                    lr_block=lr / 2, lr_full=lr, momentum=0.9,
                    options=mb.options_default(scale_mode=1, rms_beta=0.2))
    losses = []
    x = torch.randn(tokens, width, generator=g, device="cuda").bfloat16()
    want, _ = teacher.forward(x)
    for t in range(steps):
        y, kept = student.forward(x)
        diff = y.float() - want.float()
        losses.append(float(diff.square().mean()))
        grads, _ = student.backward((2.0 / diff.numel() * diff).bfloat16(), kept, input_grad=False)
        opt.step(student.weights, grads, t)
        student.quantize()
    opt.close()
    linear.close()
    return losses


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--tokens", type=int, default=512)
    p.add_argument("--width", type=int, default=512)
    p.add_argument("--hidden", type=int, default=1408)
    p.add_argument("--steps", type=int, default=30)
    a = p.parse_args()
    for t, loss in enumerate(train(a.tokens, a.width, a.hidden, a.steps)):
        if t % 5 == 0 or t == a.steps - 1:
            print(f"step {t:3d}  loss {loss:.5f}", flush=True)


if __name__ == "__main__":
    main()
