"""The feed-forward block of a language model in microscaled formats: trained for a few steps, then served token by token.

    y = x + W2 (silu(Wg h) * (Wu h)),   h = layer norm of x

Products run on 4-bit operands; what the backward pass reads again -- the norm's input, the layers' inputs, the gate and what it
gates -- is kept in 8 bits.  Weights are fp32 between the steps and quantised once per step (when served: once).

    python examples/feed_forward.py [--tokens 4096] [--width 1024] [--hidden 4096] [--steps 16]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2105_11010_amd as sq  # noqa: E402

EPS = 1e-5


def empty(*shape, dtype=torch.bfloat16):
    return torch.empty(*shape, dtype=dtype, device="cuda")


def coded(rows, K, bits):
    """Codes and scales of [rows][K]."""
    return (empty(rows, sq.sparq_mx_code_bytes(K, bits), dtype=torch.uint8),
            empty(rows, sq.sparq_mx_scale_bytes(K), dtype=torch.uint8))


class Linear:
    """A layer [N][K] for M rows: fp32 weights, their 4-bit form, and the buffers a step needs."""

    def __init__(self, M, N, K):
        self.K = K
        self.w = torch.randn(N, K, device="cuda") * K ** -0.5
        self.dw = empty(N, K, dtype=torch.float32)
        self.w4, self.x4, self.x8 = coded(N, K, 4), coded(M, K, 4), coded(M, K, 8)
        self.workspace = empty(max(sq.sparq_mx_gemm_workspace_bytes(M, N, K), sq.sparq_mx_linear_workspace_bytes(M, N, K),
                                   sq.sparq_mx_linear_dx_workspace_bytes(M, N, K), sq.sparq_mx_linear_dw_workspace_bytes(M, N, K)),
                               dtype=torch.uint8)
        self.quantize()

    def quantize(self):
        sq.sparq_mx_quantize(self.w, *self.w4)

    def forward(self, x, y):
        """y = x W^T; x is kept for the backward pass."""
        sq.sparq_mx_quantize(x, *self.x4, *self.x8)
        sq.sparq_mx_gemm(*self.x4, *self.w4, self.K, y, workspace=self.workspace)

    def serve(self, x, y):
        sq.sparq_mx_linear(x, *self.w4, y, workspace=self.workspace)

    def backward(self, dy, dx):
        sq.sparq_mx_linear_dx(dy, *self.w4, dx, workspace=self.workspace)
        sq.sparq_mx_linear_dw(dy, *self.x8, self.dw, workspace=self.workspace)


class FeedForward:
    def __init__(self, tokens, width, hidden):
        self.gamma, self.beta = torch.ones(width, device="cuda"), torch.zeros(width, device="cuda")
        self.dgamma, self.dbeta = torch.empty_like(self.gamma), torch.empty_like(self.beta)
        self.up, self.down = Linear(tokens, 2 * hidden, width), Linear(tokens, width, hidden)        # (gate and up in one product)
        self.hidden, self.kept = hidden, coded(tokens, width, 8)
        self.kept_gate, self.kept_up = coded(tokens, hidden, 8), coded(tokens, hidden, 8)
        self.mean, self.rstd = empty(tokens, dtype=torch.float32), empty(tokens, dtype=torch.float32)
        self.workspace = empty(sq.sparq_mx_norm_grad_workspace_bytes(tokens, width), dtype=torch.uint8)

    def forward(self, x):
        h, both, a, y = empty(*x.shape), empty(len(x), 2 * self.hidden), empty(len(x), self.hidden), empty(*x.shape)
        sq.sparq_mx_norm(x, self.gamma, self.beta, EPS, h, mean=self.mean, rstd=self.rstd, codes=self.kept[0], scales=self.kept[1])
        self.up.forward(h, both)
        sq.sparq_mx_act("silu", both[:, :self.hidden], a, up=both[:, self.hidden:], gate_codes=self.kept_gate[0],
                        gate_scales=self.kept_gate[1], up_codes=self.kept_up[0], up_scales=self.kept_up[1])
        self.down.forward(a, y)
        return x + y

    def backward(self, dy):
        """The weights' gradients (in dw, dgamma, dbeta) and dx."""
        da, dboth, dh, dx = empty(len(dy), self.hidden), empty(len(dy), 2 * self.hidden), empty(*dy.shape), empty(*dy.shape)
        self.down.backward(dy, da)
        sq.sparq_mx_act_grad("silu", da, *self.kept_gate, dboth[:, :self.hidden], up_codes=self.kept_up[0], up_scales=self.kept_up[1],
                             dup=dboth[:, self.hidden:])
        self.up.backward(dboth, dh)
        sq.sparq_mx_norm_grad(dh, *self.kept, self.mean, self.rstd, self.gamma, dx, dgamma=self.dgamma, dbeta=self.dbeta,
                              workspace=self.workspace)
        return dy + dx

    def step(self, rate):
        for w, dw in ((self.up.w, self.up.dw), (self.down.w, self.down.dw), (self.gamma, self.dgamma), (self.beta, self.dbeta)):
            w.sub_(dw, alpha=rate)
        self.up.quantize()
        self.down.quantize()

    def serve(self, x):
        h, both, a, y = empty(*x.shape), empty(len(x), 2 * self.hidden), empty(len(x), self.hidden), empty(*x.shape)
        sq.sparq_mx_norm(x, self.gamma, self.beta, EPS, h)
        self.up.serve(h, both)
        sq.sparq_mx_act("silu", both[:, :self.hidden], a, up=both[:, self.hidden:])
        self.down.serve(a, y)
        return x + y


def train_and_serve(tokens, width, hidden, steps, rate=0.2):
    """Fits the block to x + 0.5 x R, R a random rotation of the channels; the losses, and the largest difference between the batch's
    outputs and the same tokens served one by one."""
    torch.manual_seed(0)
    block = FeedForward(tokens, width, hidden)
    x = torch.randn(tokens, width, device="cuda").bfloat16()
    rotation = torch.linalg.qr(torch.randn(width, width, device="cuda"))[0]
    target = x.float() + 0.5 * x.float() @ rotation
    losses = []
    for _ in range(steps):
        off = block.forward(x).float() - target
        losses.append(float((off * off).sum(1).mean()))
        block.backward((off * (2 / tokens)).bfloat16())
        block.step(rate)
    batch = block.forward(x)
    apart = max(float((block.serve(x[i:i + 1]) - batch[i:i + 1]).abs().max()) for i in range(min(tokens, 4)))
    return losses, apart


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("tokens", 4096), ("width", 1024), ("hidden", 4096), ("steps", 16)):
        p.add_argument("--" + name, type=int, default=default)
    a = p.parse_args()
    losses, apart = train_and_serve(a.tokens, a.width, a.hidden, a.steps)
    print("loss per token:", " ".join("%.4g" % v for v in losses))
    print("a token served alone differs from the batch by at most %.3g" % apart)


if __name__ == "__main__":
    main()
