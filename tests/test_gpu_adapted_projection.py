"""The operators together, as examples/adapted_projection.py uses them: one step's gradients against a plain implementation in 64 bits, the training's
progress, and a decode step beside the same tokens within a batch."""
import importlib.util
import os

import pytest
import torch

from paper_1805_10692_amd import binding as B

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("adapted_projection", os.path.join(ROOT, "examples", "adapted_projection.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_gradients_of_a_step(example):
    gen = torch.Generator(device="cuda").manual_seed(3)
    m, n, tokens = 96, 130, 75
    layer = example.AdaptedProjection(torch.randn((m, n), generator=gen, device="cuda"), bits=4, tasks=3, rank=5)
    layer.Bm.normal_(generator=gen)
    layer.weight.normal_(generator=gen)
    x = torch.randn((tokens, n), generator=gen, device="cuda")
    index = torch.tensor([0] * 30 + [2] * 20 + [-1] * 10 + [1] * 15, dtype=torch.int32, device="cuda")
    dy = torch.randn((m, tokens), generator=gen, device="cuda").t()
    y = layer.forward(x, index)
    dx, dA, dB, dweight = layer.backward(dy)
    W = torch.empty((m, n), device="cuda")
    B.cer_decode_device(layer.handle, W)
    # 64 bits, by torch's differentiation
    p = [t.detach().cpu().double().requires_grad_() for t in (x, layer.A, layer.Bm, layer.weight)]
    hat = p[0] * torch.rsqrt(p[0].square().mean(1, keepdim=True) + 1e-6) * p[3]
    want = hat @ W.cpu().double().t()
    rows = []
    for t in range(tokens):
        a = int(index[t])
        rows.append(want[t] if a < 0 else want[t] + 2.0 * (p[2][a] @ (p[1][a] @ hat[t])))
    want = torch.stack(rows)
    want.backward(dy.cpu().double())
    # sums of at most 130 + 96 + 75 products of size 1 in 32 bits, errors of either sign: within 300 . 2^-23 of the largest element
    for got, w in ((y, want.detach()), *zip((dx, dA, dB, dweight), (q.grad for q in p))):
        assert float((got.cpu().double() - w).abs().max()) <= 300 * 2.0 ** -23 * float(w.abs().max())


def test_training_and_serving(example):
    losses = example.main(m=160, n=192, tasks=3, rank=4, steps=40)
    assert losses[-1] < 0.5 * losses[0] and all(v == v for v in losses)


def test_decode_step_gives_what_the_batch_gave(example):
    gen = torch.Generator(device="cuda").manual_seed(4)
    layer = example.AdaptedProjection(torch.randn((64, 96), generator=gen, device="cuda"), bits=3, tasks=2, rank=3)
    layer.Bm.normal_(generator=gen)
    x = torch.randn((300, 96), generator=gen, device="cuda")
    index = torch.tensor([0] * 140 + [1] * 160, dtype=torch.int32, device="cuda")
    whole = layer.forward(x, index).clone()
    at = torch.tensor([0, 139, 140, 299], device="cuda")
    few = layer.forward(x[at], index[at])
    # the same sums in another order: 96 + 3 products twice, in 32 bits
    assert float((whole[at] - few).abs().max()) <= 200 * 2.0 ** -23 * float(whole.abs().max())
