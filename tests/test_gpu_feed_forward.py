"""The example that runs the microscaled operators together: a feed-forward block that trains and serves."""
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ff():
    assert torch.cuda.is_available(), "GPU tests need a device"
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import feed_forward
    return feed_forward


def test_trains_and_serves(ff):
    losses, apart = ff.train_and_serve(512, 256, 512, 12)
    assert all(b < a for a, b in zip(losses, losses[1:])) and losses[-1] < 0.8 * losses[0], losses
    assert apart < 0.1


def test_gradients_against_autograd(ff):
    """The block's gradients beside those of the same block in fp32, whose inputs, weights and activations are not quantised: they point
    the same way.  4-bit operands have steps of a quarter to a half, an error of about 0.1 of a value: a cosine of 0.99 a product, two or three
    products on the way."""
    torch.manual_seed(1)
    tokens, width, hidden = 384, 256, 320
    block = ff.FeedForward(tokens, width, hidden)
    x = torch.randn(tokens, width, device="cuda").bfloat16()
    dy = (torch.randn(tokens, width, device="cuda") / tokens).bfloat16()
    block.forward(x)
    dx = block.backward(dy)
    p = [t.clone().requires_grad_() for t in (x.float(), block.gamma, block.beta, block.up.w, block.down.w)]
    h = torch.nn.functional.layer_norm(p[0], (width,), p[1], p[2], ff.EPS)
    both = h @ p[3].t()
    y = p[0] + (torch.nn.functional.silu(both[:, :hidden]) * both[:, hidden:]) @ p[4].t()
    y.backward(dy.float())
    for name, got, ref in zip(("dx", "dgamma", "dbeta", "dw up", "dw down"), (dx, block.dgamma, block.dbeta, block.up.dw, block.down.dw), p):
        cosine = torch.nn.functional.cosine_similarity(got.float().flatten(), ref.grad.flatten(), 0)
        assert cosine > 0.95, (name, float(cosine))
