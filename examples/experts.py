"""A feed-forward block with experts in microscaled formats, forward and backward, on the library's entry points alone.

    y = x + dropout(sum_j w_j W2[e_j] gelu(W1[e_j] x + b1[e_j]))

over each token's chosen experts e_j and their weights w_j, which a router gives.  Rows go to their experts in 4 bits for the product and in 8 for its backward
pass; how many rows an expert has the host never learns, so that a step can be captured into a graph.

    python examples/experts.py [--tokens 4096] [--per 2] [--experts 8] [--width 1024] [--hidden 2048]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2105_11010_amd as sq  # noqa: E402

SEED = 17


def empty(*shape, dtype=torch.bfloat16):
    return torch.empty(*shape, dtype=dtype, device="cuda")


def coded(rows, K, bits):
    """Codes and scales of [rows][K]."""
    return (empty(rows, sq.sparq_mx_code_bytes(K, bits), dtype=torch.uint8),
            empty(rows, sq.sparq_mx_scale_bytes(K), dtype=torch.uint8))


class Block:
    """Weights [experts][hidden][width] and [experts][width][hidden], and the buffers of a step of `tokens` tokens with `per` experts each."""

    def __init__(self, tokens, per, experts, width, hidden):
        rows, f32 = tokens * per, torch.float32
        g = torch.Generator(device="cuda").manual_seed(3)
        self.width, self.hidden = width, hidden
        self.w1 = torch.randn(experts * hidden, width, generator=g, device="cuda") * width ** -0.5
        self.w2 = torch.randn(experts * width, hidden, generator=g, device="cuda") * hidden ** -0.5
        self.b1 = torch.randn(experts, hidden, generator=g, device="cuda")
        self.w1q, self.w2q = coded(experts * hidden, width, 4), coded(experts * width, hidden, 4)
        sq.sparq_mx_quantize(self.w1, *self.w1q)
        sq.sparq_mx_quantize(self.w2, *self.w2q)
        self.offsets, self.place = empty(experts + 1, dtype=torch.int32), empty(tokens, per, dtype=torch.int32)
        self.x4, self.x8, self.z8 = coded(rows, width, 4), coded(rows, width, 8), coded(rows, hidden, 8)
        self.a4, self.a8 = coded(rows, hidden, 4), coded(rows, hidden, 8)
        # (rows that nobody has are read by the codec alone)
        self.a, self.o, self.da = torch.zeros_like(empty(rows, hidden)), empty(rows, width), torch.zeros_like(empty(rows, hidden))
        self.z8[0].zero_(), self.z8[1].zero_()
        self.c, self.y, self.dc, self.dx = (empty(tokens, width) for _ in range(4))
        self.do, self.dz, self.dr = empty(rows, width), empty(rows, hidden), empty(rows, width)
        self.dweights, self.db1 = empty(tokens, per, dtype=f32), empty(experts, hidden, dtype=f32)
        self.dw1, self.dw2 = torch.empty_like(self.w1), torch.empty_like(self.w2)
        need = [sq.sparq_mx_sort_workspace_bytes(rows, experts)]
        for n, k in ((hidden, width), (width, hidden)):
            need += [sq.sparq_mx_experts_gemm_workspace_bytes(rows, n, k, experts), sq.sparq_mx_experts_dx_workspace_bytes(rows, n, k, experts),
                     sq.sparq_mx_experts_dw_workspace_bytes(rows, n, k, experts)]
        self.ws = empty(max(need), dtype=torch.uint8)

    def forward(self, x, chosen, weights, p=0.0, step=None):
        """chosen: int32 [tokens][per], a number outside of the experts' is a choice refused; weights: fp32 [tokens][per]; step: dropout's, in device memory."""
        sq.sparq_mx_sort(chosen, self.offsets, self.place, workspace=self.ws)
        sq.sparq_mx_gather(x, self.place, codes4=self.x4[0], scales4=self.x4[1], codes8=self.x8[0], scales8=self.x8[1])
        sq.sparq_mx_experts_gemm(*self.x4, *self.w1q, self.width, self.a, offsets=self.offsets, bias=self.b1, function="gelu",
                                 kept_codes=self.z8[0], kept_scales=self.z8[1], workspace=self.ws)
        sq.sparq_mx_quantize(self.a, *self.a4, *self.a8)
        sq.sparq_mx_experts_gemm(*self.a4, *self.w2q, self.hidden, self.o, offsets=self.offsets, workspace=self.ws)
        sq.sparq_mx_combine(self.o, self.place, self.c, weights=weights)
        sq.sparq_mx_dropout(self.c, p, SEED, self.y, residual=x, step=step)
        return self.y

    def backward(self, dy, weights, p=0.0, step=None):
        """dx; the weights' gradients are in dw1, dw2 and db1, the router's in dweights."""
        sq.sparq_mx_dropout(dy, p, SEED, self.dc, step=step)
        sq.sparq_mx_combine_grad(self.dc, self.place, weights, dx=self.do, x=self.o, dweights=self.dweights)
        sq.sparq_mx_experts_dx(self.do, self.offsets, *self.w2q, self.da, workspace=self.ws)
        sq.sparq_mx_experts_dw(self.do, self.offsets, *self.a8, self.dw2, workspace=self.ws)
        sq.sparq_mx_act_grad("gelu", self.da, *self.z8, self.dz)
        sq.sparq_mx_experts_dx(self.dz, self.offsets, *self.w1q, self.dr, workspace=self.ws)
        sq.sparq_mx_experts_dw(self.dz, self.offsets, *self.x8, self.dw1, db=self.db1, workspace=self.ws)
        sq.sparq_mx_combine(self.dr, self.place, self.dx, residual=dy)
        return self.dx

    def results(self):
        return {k: getattr(self, k) for k in ("offsets", "place", "y", "dx", "dweights", "dw1", "dw2", "db1")}


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("tokens", 4096), ("per", 2), ("experts", 8), ("width", 1024), ("hidden", 2048)):
        p.add_argument("--" + name, type=int, default=default)
    a = p.parse_args()
    block = Block(a.tokens, a.per, a.experts, a.width, a.hidden)
    x = torch.randn(a.tokens, a.width, device="cuda").bfloat16()
    top, chosen = torch.topk(torch.randn(a.tokens, a.experts, device="cuda"), a.per, dim=1)
    chosen, weights = chosen.int().contiguous(), torch.softmax(top, 1).contiguous()
    block.forward(x, chosen, weights, p=0.1)
    block.backward(torch.randn_like(x), weights, p=0.1)
    print("rows of each expert:", block.offsets.diff().tolist())
    for k, v in block.results().items():
        if v.dtype.is_floating_point:
            print("%s: root of the mean square %.4g" % (k, float(v.float().square().mean().sqrt())))


if __name__ == "__main__":
    main()
