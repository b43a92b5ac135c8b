"""The operators of a block where offsets pass 32 bits."""
import numpy as np
import pytest
import torch

from block_reference import HALF, near, philox
from paper_1805_10692_amd import binding as B

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def test_dropout_of_more_than_one_launch():
    """17 GB in place: 2^33 numbers are a launch."""
    n, tokens = 65536, (1 << 17) + 3
    x = torch.ones((tokens, n), dtype=BF16, device="cuda")
    key = torch.tensor([7, 9], dtype=torch.int64, device="cuda")
    B.dropout_add(x, x, key, 0.5)
    for t in (0, 65537, (1 << 17) - 1, 1 << 17, tokens - 1):
        counters = [(at % 2 ** 32, at >> 32, 9, 0) for at in range(t * 8192, t * 8192 + 40)]
        words = np.array(philox(counters, (7, 0)), dtype=np.uint64)
        keep = np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], axis=2).reshape(-1) >= 32768
        assert torch.equal(x[t, :320].cpu() != 0, torch.from_numpy(keep)), t
    del x
    torch.cuda.empty_cache()


def test_block_norm_far_apart():
    tokens, n, ld = 300, 64, 1 << 23  # rows 16 MB apart: 2.5 G numbers
    room = torch.zeros((tokens, ld), dtype=BF16, device="cuda")
    x, f = room[:, 1:n + 1], torch.randn((tokens, n), device="cuda").to(BF16)
    x.copy_(torch.randn((tokens, n), device="cuda"))
    h, y, h2, y2 = (torch.empty((tokens, n), dtype=BF16, device="cuda") for _ in range(4))
    B.block_norm(x.contiguous(), f, h, y)
    B.block_norm(x, f, h2, room[:, 100:100 + n])
    assert torch.equal(h, h2) and torch.equal(y, room[:, 100:100 + n])
    dx, df, dx2, df2 = (torch.empty_like(h) for _ in range(4))
    r = torch.ones(tokens, device="cuda")
    B.block_norm_backward(f, x.contiguous(), f, r, dx, df)
    B.block_norm_backward(f, x, f, r, room[:, 200:200 + n], df2)
    assert torch.equal(dx, room[:, 200:200 + n]) and torch.equal(df, df2)
    del room, x, y2, dx2
    torch.cuda.empty_cache()


def test_linear_of_many_tokens():
    tokens, n, m = 600_001, 4096, 8  # 2.5 G numbers
    x = torch.zeros((tokens, n), dtype=BF16, device="cuda")
    at = torch.tensor([0, 1, 299_999, 524_287, 524_288, 524_289, 600_000], device="cuda")
    x[at] = torch.randn((len(at), n), device="cuda").to(BF16)
    W, y = torch.randn((m, n), device="cuda").to(BF16), torch.empty((tokens, m), dtype=BF16, device="cuda")
    B.linear_matmul(W, x, y)
    want = x[at].double() @ W.double().t().contiguous()
    near(y[at], want, (n + 8) * 2.0 ** -23 * (x[at].double().abs() @ W.double().abs().t().contiguous()), HALF[BF16])
    assert int((y != 0).any(1).sum()) == len(at)
    dW, dx = torch.empty_like(W), x
    B.linear_backward(W, y, X=x, dW=dW)
    exact = y[at].double().t().contiguous() @ x[at].double()
    near(dW, exact, (len(at) + 8) * 2.0 ** -23 * (y[at].double().abs().t().contiguous() @ x[at].double().abs()), HALF[BF16])
    B.linear_backward(W, y, dX=dx)
    near(dx[at], y[at].double() @ W.double(), (m + 8) * 2.0 ** -23 * (y[at].double().abs() @ W.double().abs()), HALF[BF16])
    del x, dx, y
    torch.cuda.empty_cache()
