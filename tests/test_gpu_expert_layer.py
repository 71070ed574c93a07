"""The operators together: the example's layer trains and serves, and its gradients are those of the same layer in 32 bits."""
from __future__ import annotations

import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_example_trains_and_serves():
    import expert_layer
    losses, off = expert_layer.main(20)
    assert losses[-1] < 0.8 * losses[0]
    # roundings to bfloat16 (2^-9 rms each) of the inner rows, the sums, the projection and the result
    assert off < 8 * 2.0 ** -8


def test_gradients_of_the_layer():
    """Against autograd through the layer in 32 bits, with the routing held at the choice that was made."""
    import expert_layer as ex
    layer = ex.Layer(3)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    x = torch.randn((200, ex.H), generator=g, device="cuda").to(torch.bfloat16)
    y, kept = layer.forward(x)
    gy = torch.randn(y.shape, generator=g, device="cuda").to(torch.bfloat16)
    gx, grads = layer.backward(gy, kept)
    w, _, R = kept[:3]
    leaf = {n: t.float().requires_grad_() for n, t in w.items()}
    xf = x.float().requires_grad_()
    cols = R.colidx.view(-1, ex.K).long()
    v = torch.softmax((xf @ leaf["router"].T).gather(1, cols), 1)
    out = 0
    for j in range(ex.K):
        up = torch.einsum("th,tfh->tf", xf, leaf["up"][cols[:, j]])
        out = out + v[:, j, None] * torch.einsum("tf,thf->th", torch.relu(up), leaf["down"][cols[:, j]])
    out.backward(gy.float())
    # a handful of roundings to bfloat16 (relative 2^-9 rms) on every way, and relu's sign at values that rounding moved
    for got, want in [(y, out.detach()), (gx, xf.grad)] + [(grads[n], leaf[n].grad) for n in leaf]:
        assert float((got.float() - want).norm() / want.norm()) < 12 * 2.0 ** -8
