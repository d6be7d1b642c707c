"""Training steps of one pipeline stage: its layers, compressor and optimizer.

The stage holds a feed-forward block and a gated one, each with its residual:

    a  = gelu(x W1^T + b1)         y = a W2^T + b2 + x
    h  = silu(g) * u, [g u] = y Wg^T       z = h W3^T + y

A step does what a stage does under compressed communication: forward
(occ_linear_fwd, occ_gated_fwd), the activation gradient as it comes from the
next stage, as factors (occ_step by the sender, occ_decompress_ex here),
backward (occ_linear_bwd, occ_gated_bwd), compression of the weight gradients
(occ_step_batched_noalloc; between data-parallel ranks the factors would be
averaged here), and AdamW straight from those factors (occ_adamw_step), with
fp32 weights, their bf16 copies and 8-bit moments.  The residuals' gradients
are added with torch.

    python examples/stage_step.py [--steps 60] [--hidden 512] [--tokens 1024]
"""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2301_09830_amd import optcc  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32


class Weight:
    """A matrix with what its gradient's compressor and its optimizer keep."""

    def __init__(self, rows, cols, rank, gen):
        def randn(*shape):
            return torch.randn(*shape, generator=gen, device="cuda")

        self.value = randn(rows, cols) * cols ** -0.5
        self.bf16 = self.value.to(BF16)
        self.grad = torch.empty(rows, cols, dtype=BF16, device="cuda")
        self.err = torch.zeros(rows, cols, device="cuda")
        self.P, self.Q = torch.empty(rows, rank, device="cuda"), randn(cols, rank)
        self.m, self.v = (torch.zeros(rows, cols, dtype=torch.uint8, device="cuda") for _ in "mv")
        runs = -(-cols // optcc.OCC_SCALE_RUN)
        self.m_scale, self.v_scale = (torch.zeros(rows, runs, device="cuda") for _ in "mv")

    def param(self):
        return optcc.make_param(self.value, self.m, self.v, P=self.P, Q=self.Q, W16=self.bf16,
                                m_scale=self.m_scale, v_scale=self.v_scale, decay=0.01)


class Bias:
    """A vector: its gradient is exchanged as it is, its moments are fp32."""

    def __init__(self, n):
        self.value, self.grad, self.m, self.v = (torch.zeros(n, device="cuda") for _ in range(4))

    def param(self):
        return optcc.make_param(self.value, self.m, self.v, G=self.grad)


class Stage:
    def __init__(self, hidden, tokens, rank, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        h = hidden
        self.W1, self.W2 = Weight(4 * h, h, rank, gen), Weight(h, 4 * h, rank, gen)
        self.Wg, self.W3 = Weight(4 * h, h, rank, gen), Weight(h, 2 * h, rank, gen)
        self.b1, self.b2 = Bias(4 * h), Bias(h)
        self.weights = [self.W1, self.W2, self.Wg, self.W3]
        self.params = optcc.make_params(p.param() for p in self.weights + [self.b1, self.b2])
        self.flags = torch.zeros(1, dtype=torch.int32, device="cuda")

        def empty(cols):
            return torch.empty(tokens, cols, dtype=BF16, device="cuda")

        self.z1, self.a, self.y = empty(4 * h), empty(4 * h), empty(h)
        self.gu, self.h, self.z = empty(4 * h), empty(2 * h), empty(h)
        self.dh, self.dy, self.da, self.dx = empty(2 * h), empty(h), empty(4 * h), empty(h)

    def forward(self, x):
        o = optcc
        self.x = x
        o.occ_linear_fwd(x, self.W1.bf16, bias=self.b1.value, act=o.OCC_ACT_GELU, Z=self.z1, Y=self.a)
        o.occ_linear_fwd(self.a, self.W2.bf16, bias=self.b2.value, R=x, Y=self.y)
        o.occ_gated_fwd(self.y, self.Wg.bf16, act=o.OCC_ACT_SILU, Z=self.gu, Y=self.h)
        o.occ_linear_fwd(self.h, self.W3.bf16, R=self.y, Y=self.z)
        return self.z

    def backward(self, dz):
        """Gradients of every weight; returns the activation gradient for the stage before."""
        o = optcc
        o.occ_linear_bwd(dz, self.h, self.W3.bf16, dX=self.dh, dW=self.W3.grad)
        o.occ_gated_bwd(self.dh, self.y, self.Wg.bf16, Z=self.gu, act=o.OCC_ACT_SILU, dX=self.dy,
                        dW=self.Wg.grad)
        self.dy += dz          # the residual's way round the gated block
        o.occ_linear_bwd(self.dy, self.a, self.W2.bf16, dX=self.da, dW=self.W2.grad,
                         dbias=self.b2.grad)
        o.occ_linear_bwd(self.da, self.x, self.W1.bf16, Z=self.z1, act=o.OCC_ACT_GELU, dX=self.dx,
                         dW=self.W1.grad, dbias=self.b1.grad)
        self.dx += self.dy
        return self.dx

    def update(self, rank, step, lr):
        """Compresses the weight gradients and takes an optimizer step from the factors."""
        self.flags.zero_()
        optcc.occ_step_batched_noalloc([(w.grad, w.err, w.Q, w.P, None) for w in self.weights],
                                       rank, 1, write_mhat=False, flags_out=self.flags)
        optcc.occ_adamw_step(self.params, lr=lr, step=step, seed=step, flags=self.flags)


def run(steps=60, hidden=512, tokens=1024, rank=16, lr=1e-3, report=None):
    """Fits the stage to another one's outputs; returns the loss of each step."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    stage, teacher = Stage(hidden, tokens, rank), Stage(hidden, tokens, rank, seed=1)
    # the next stage sends its activation gradient as factors, with error feedback
    err = torch.zeros(tokens, hidden, device="cuda")
    Q = torch.randn(hidden, 4 * rank, generator=gen, device="cuda")
    P = torch.empty(tokens, 4 * rank, device="cuda")
    ws = optcc.alloc_workspace(optcc.occ_workspace_bytes([(tokens, hidden)], 4 * rank, 1,
                                                         optcc.OCC_BF16))
    x = torch.randn(tokens, hidden, generator=gen, device="cuda").to(BF16)
    target = teacher.forward(x).float()
    losses = []
    for step in range(1, steps + 1):
        diff = stage.forward(x).float() - target
        losses.append(float(diff.square().mean()))
        if report:
            report(step, losses[-1])
        gradient = (diff * (2.0 / hidden)).to(BF16)
        optcc.occ_step(gradient, err, Q, 4 * rank, 1, P=P, write_mhat=False, ws=ws)   # the sender
        dz = optcc.occ_decompress_ex(P, Q, optcc.OCC_DEC_SPLIT_BF16 | optcc.OCC_DEC_OUT_BF16)
        stage.backward(dz)
        stage.update(rank, step, lr)
    return losses


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--hidden", type=int, default=512)
    ap.add_argument("--tokens", type=int, default=1024)
    ap.add_argument("--rank", type=int, default=16)
    ap.add_argument("--lr", type=float, default=1e-3)
    a = ap.parse_args()

    def report(step, loss):
        if step == 1 or step % 10 == 0:
            print(f"step {step:4d}  loss {loss:.5f}", flush=True)

    run(a.steps, a.hidden, a.tokens, a.rank, a.lr, report)


if __name__ == "__main__":
    main()
