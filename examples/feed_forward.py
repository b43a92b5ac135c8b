"""A feed-forward block with one trained and one compressed projection: its training step, and serving.

    python examples/feed_forward.py

    x (tokens, n) -> rms_norm -> linear_matmul(W, b, silu) -> dropout_add -> cer_matmul(V) -> block_norm(x, gate) -> h, y

W is dense and trained; V is quantized, kept in CER form and frozen.  Everything between the norms is in columns, cer_matmul's order; the residual
stream x -> h is in rows.  y is what the next block reads.  A step goes back the same way, with the same dropout mask formed again from its key.
Calls that need memory take temporaries of their own: on the null stream.  On another one they take a workspace (binding.linear_workspace_bytes, block_workspace_bytes).
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1805_10692_amd import binding as B  # noqa: E402


def columns(features: int, tokens: int) -> torch.Tensor:
    """(tokens, features), feature after feature in memory."""
    return torch.empty((features, tokens), device="cuda").t()


class FeedForward:
    NAMES = ("W", "b", "before", "after", "gate", "following")

    def __init__(self, n: int, hidden: int, bits: int, p: float, seed: int = 0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        V = torch.randn((n, hidden), generator=gen, device="cuda") / hidden ** 0.5
        self.n, self.hidden, self.p, self.scale = n, hidden, p, 0.9
        self.handle, codebook = B.cer_quantize_encode_device(V, n, hidden, bits)
        self.V = torch.empty_like(V)
        B.cer_decode_device(self.handle, self.V)
        self.back = B.cer_encode_device(self.V.t().contiguous(), hidden, n, codebook)
        self.W = torch.randn((hidden, n), generator=gen, device="cuda") / n ** 0.5
        self.b = torch.zeros(hidden, device="cuda")
        self.before, self.after, self.following = (torch.ones(n, device="cuda") for _ in range(3))  # the norms' weights
        self.gate = torch.full((n,), 0.5, device="cuda")
        self.key = torch.tensor([seed, 0], dtype=torch.int64, device="cuda")
        self.norm = torch.empty(1, device="cuda")

    def parameters(self):
        return [getattr(self, k) for k in self.NAMES]

    def forward(self, x: torch.Tensor, train: bool):
        """Returns h and y, and keeps what backward needs."""
        t = x.shape[0]
        u, z, a, f, h, y = columns(self.n, t), columns(self.hidden, t), columns(self.hidden, t), columns(self.n, t), torch.empty_like(x), torch.empty_like(x)
        r, r_post, r_pre = (torch.empty(t, device="cuda") for _ in range(3))
        B.rms_norm(x, u, self.before, rstd=r)
        B.linear_matmul(self.W, u, a, bias=self.b, activation="silu", pre=z if train else None)
        if train:
            B.dropout_add(a, a, self.key, self.p)
        B.cer_matmul(self.handle, a.t(), f.t(), t)
        B.block_norm(x, f, h, y, gate=self.gate, post_weight=self.after, pre_weight=self.following, scale=self.scale, rstd_post=r_post, rstd_pre=r_pre)
        self.kept = (x, u, z, f, h, r, r_post, r_pre)
        return h, y

    def backward(self, dh: torch.Tensor, dy: torch.Tensor):
        """Returns the gradient of x and those of the parameters, in their order."""
        x, u, z, f, h, r, r_post, r_pre = self.kept
        t = x.shape[0]
        dx, df, da, du = torch.empty_like(x), columns(self.n, t), columns(self.hidden, t), columns(self.n, t)
        dW, db, dbefore, dafter, dgate, dfollowing = (torch.empty_like(p) for p in self.parameters())
        B.block_norm_backward(dy, h, f, r_pre, dx, df, rstd_post=r_post, gate=self.gate, post_weight=self.after, pre_weight=self.following, scale=self.scale,
                              dsum=dh, dgate=dgate, dpost_weight=dafter, dpre_weight=dfollowing)
        B.cer_matmul(self.back, df.t(), da.t(), t)
        B.dropout_add(da, da, self.key, self.p)
        B.linear_backward(self.W, da, X=u, activation="silu", pre=z, dX=du, dW=dW, dbias=db)
        B.rms_norm_backward(du, x, r, dx, self.before, dsum=dx, dweight=dbefore)
        return dx, [dW, db, dbefore, dafter, dgate, dfollowing]

    def step(self, x, target, rate: float, most: float) -> float:
        """One step of gradient descent on the mean squared error of y; returns the loss before it."""
        _, y = self.forward(x, train=True)
        off = y - target
        _, grads = self.backward(torch.zeros_like(x), off / x.shape[0])
        B.grad_clip(grads, most, self.norm)
        for p, g in zip(self.parameters(), grads):
            p.sub_(g, alpha=rate)
        self.key[1] += 1  # the next step has another mask
        return float(off.square().sum()) / x.shape[0] / 2


def main(n: int = 384, hidden: int = 640, tokens: int = 300, steps: int = 40) -> list:
    gen = torch.Generator(device="cuda").manual_seed(1)
    layer = FeedForward(n, hidden, bits=4, p=0.1)
    x, target = torch.randn((tokens, n), generator=gen, device="cuda"), torch.randn((tokens, n), generator=gen, device="cuda")
    losses = [layer.step(x, target, rate=0.02, most=25.0) for _ in range(steps)]
    print("loss: " + " ".join(f"{v:.2f}" for v in losses[:: max(1, steps // 6)]))
    _, served = layer.forward(x[:1].contiguous(), train=False)
    print(f"served one token: |y| {float(served.norm()):.2f}")
    return losses


if __name__ == "__main__":
    main()
