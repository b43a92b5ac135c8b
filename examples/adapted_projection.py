"""A frozen, compressed projection with low-rank adapters beside it: trained, then served.

    python examples/adapted_projection.py

The projection's weights are quantized and kept in CER form; they cannot be trained.  What is trained for each of a few tasks is an adapter beside
them, and the weight of the norm in front:

    x (tokens, n) -> rms_norm -> columns -> cer_matmul(W) + adapter_matmul -> y (tokens, m)

A step goes back the same way -- cer_matmul with the transposed matrix's handle, adapter_backward, rms_norm_backward -- and the gradients
are clipped together.  Serving runs the same three calls on a batch of single tokens that belong to different tasks, or to none.
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1805_10692_amd import binding as B  # noqa: E402


class AdaptedProjection:
    def __init__(self, W: torch.Tensor, bits: int, tasks: int, rank: int, seed: int = 0):
        """W: fp32 device tensor (m, n), quantized here to `bits` bits."""
        self.m, self.n = W.shape
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.handle, codebook = B.cer_quantize_encode_device(W.contiguous(), self.m, self.n, bits)
        dense = torch.empty((self.m, self.n), dtype=torch.float32, device="cuda")
        B.cer_decode_device(self.handle, dense)
        self.back = B.cer_encode_device(dense.t().contiguous(), self.n, self.m, codebook)
        self.A = torch.randn((tasks, rank, self.n), generator=gen, device="cuda") / self.n ** 0.5
        self.Bm = torch.zeros((tasks, self.m, rank), device="cuda")  # an adapter starts as no change
        self.scales = torch.full((tasks,), 2.0, device="cuda")
        self.weight = torch.ones(self.n, device="cuda")
        self.norm = torch.empty(1, device="cuda")

    def forward(self, x: torch.Tensor, index: torch.Tensor) -> torch.Tensor:
        """x: (tokens, n); index: each token's task, -1 for none.  Returns y as (tokens, m); keeps what backward needs."""
        tokens = x.shape[0]
        columns = torch.empty((self.n, tokens), device="cuda")
        y = torch.empty((self.m, tokens), device="cuda")
        rstd, hidden = torch.empty(tokens, device="cuda"), torch.empty((tokens, self.A.shape[1]), device="cuda")
        B.rms_norm(x, columns.t(), self.weight, rstd=rstd)
        B.cer_matmul(self.handle, columns, y, tokens)
        B.adapter_matmul(self.A, self.Bm, index, columns.t(), y.t(), scales=self.scales, base=y.t(), hidden=hidden)
        self.kept = (x, index, columns, rstd, hidden)
        return y.t()

    def backward(self, dy: torch.Tensor):
        """dy: (tokens, m) as the transposed view of a contiguous (m, tokens) tensor.  Returns the gradients of x, A, B and the norm's weight."""
        x, index, columns, rstd, hidden = self.kept
        tokens = x.shape[0]
        dcolumns = torch.empty((self.n, tokens), device="cuda")
        dA, dB, dx, dweight = torch.empty_like(self.A), torch.empty_like(self.Bm), torch.empty_like(x), torch.empty_like(self.weight)
        B.cer_matmul(self.back, dy.t(), dcolumns, tokens)
        B.adapter_backward(self.A, self.Bm, index, dy, columns.t(), hidden, scales=self.scales, base=dcolumns.t(), dX=dcolumns.t(), dA=dA, dB=dB)
        B.rms_norm_backward(dcolumns.t(), x, rstd, dx, self.weight, dweight=dweight)
        return dx, dA, dB, dweight

    def step(self, x, index, target, rate: float, most: float) -> float:
        """One step of gradient descent on the mean squared error; returns the loss before it."""
        off = self.forward(x, index) - target
        _, *grads = self.backward((off / x.shape[0]).t().contiguous().t())
        B.grad_clip(grads, most, self.norm)
        for p, g in zip((self.A, self.Bm, self.weight), grads):
            p.sub_(g, alpha=rate)
        return float(off.square().sum()) / x.shape[0] / 2


def main(m: int = 512, n: int = 512, tasks: int = 3, rank: int = 8, steps: int = 60) -> list:
    gen = torch.Generator(device="cuda").manual_seed(1)
    W = torch.randn((m, n), generator=gen, device="cuda") / n ** 0.5
    layer = AdaptedProjection(W, bits=4, tasks=tasks, rank=rank)
    # each task wants the projection changed by a matrix of low rank
    wanted = [torch.randn((m, 2), generator=gen, device="cuda") @ torch.randn((2, n), generator=gen, device="cuda") / n ** 0.5 for _ in range(tasks)]
    lengths = [70, 33, 101, 20, 64, 55]
    index = torch.tensor(np.repeat([0, 2, 1, -1, 0, 2], lengths), dtype=torch.int32, device="cuda")
    x = torch.randn((sum(lengths), n), generator=gen, device="cuda")
    plain = layer.forward(x, index).clone()
    hat = x * torch.rsqrt(x.square().mean(1, keepdim=True) + 1e-6)
    target = plain + sum((index == k)[:, None] * (hat @ wanted[k].t()) for k in range(tasks))
    losses = [layer.step(x, index, target, rate=0.05, most=25.0) for _ in range(steps)]
    print("loss: " + " ".join(f"{v:.2f}" for v in losses[:: max(1, steps // 6)]))
    # a decode step: one token of each of five requests, the last one without an adapter
    tokens, tasks_of = x[:5].contiguous(), torch.tensor([2, 0, 1, 0, -1], dtype=torch.int32, device="cuda")
    served = layer.forward(tokens, tasks_of)
    print("served " + ", ".join(f"task {int(k)}: |y| {float(v):.2f}" for k, v in zip(tasks_of, served.norm(dim=1))))
    return losses


if __name__ == "__main__":
    main()
