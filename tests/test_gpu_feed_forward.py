"""The operators of a block in a run, as examples/feed_forward.py uses them: its gradients against those of the same block in 64 bits, and its training step."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import feed_forward  # noqa: E402
from paper_1805_10692_amd import binding as B  # noqa: E402

pytestmark = pytest.mark.gpu


def plain(layer, x, params, mask):
    """The block in 64 bits, of tensors that record their gradients."""
    W, b, before, after, gate, following = params
    u = x * torch.rsqrt((x * x).mean(1, keepdim=True) + 1e-6) * before
    z = u @ W.t() + b
    f = (z * torch.sigmoid(z) * mask) @ layer.V.double().t()
    h = layer.scale * x + gate * (f * torch.rsqrt((f * f).mean(1, keepdim=True) + 1e-6) * after)
    return h, h * torch.rsqrt((h * h).mean(1, keepdim=True) + 1e-6) * following


@pytest.mark.parametrize("tokens,n,hidden", [(37, 96, 160), (130, 257, 130), (1, 64, 96)])
def test_gradients(tokens, n, hidden):
    layer = feed_forward.FeedForward(n, hidden, bits=4, p=0.25, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(5)
    x, dh, dy = (torch.randn((tokens, n), generator=gen, device="cuda") for _ in range(3))
    layer.b.normal_(generator=gen).mul_(0.1)
    for w in (layer.before, layer.after, layer.following, layer.gate):
        w.add_(0.1 * torch.randn(n, generator=gen, device="cuda"))
    ones = torch.ones((tokens, hidden), device="cuda")
    B.dropout_add(ones, ones, layer.key, layer.p)
    h, y = layer.forward(x, train=True)
    dx, grads = layer.backward(dh, dy)
    leaves = [p.double().requires_grad_() for p in [x] + layer.parameters()]
    want_h, want_y = plain(layer, leaves[0], leaves[1:], ones.double())
    want = torch.autograd.grad((want_h * dh.double()).sum() + (want_y * dy.double()).sum(), leaves)
    # each of some ten steps, the longest sum of `hidden` terms among them, is off by (hidden + 200) 2^-23 of its terms' sizes at most; sizes over results: below 8 for these random numbers
    most = 10 * 8 * (hidden + tokens + 200) * 2.0 ** -23
    for got, exact in zip((h, y, dx, *grads), (want_h, want_y, *want)):
        exact = exact.detach()
        assert float((got.double() - exact).norm()) <= most * float(exact.norm()), most


def test_without_dropout_the_served_block_is_the_trained_one():
    layer = feed_forward.FeedForward(64, 96, bits=4, p=0.0)
    x = torch.randn((20, 64), generator=torch.Generator(device="cuda").manual_seed(6), device="cuda")
    trained, served = layer.forward(x, train=True), layer.forward(x, train=False)
    assert torch.equal(trained[0], served[0]) and torch.equal(trained[1], served[1])


def test_runs():
    losses = feed_forward.main(n=128, hidden=192, tokens=70, steps=4)
    assert len(losses) == 4 and all(math.isfinite(v) for v in losses)
