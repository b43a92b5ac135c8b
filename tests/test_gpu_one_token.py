"""One token of a batch in columns: its features lie a line of tokens apart, so that its order is no choice, while that of matrices with their features side by side is.  A call
may have both.  Tolerances of the product: those of tests/test_gpu_linear.py (one token: the same sums)."""
import itertools

import pytest
import torch

from block_reference import HALF, act, near
from paper_1805_10692_amd import binding as B
from test_gpu_linear import exact_forward, numbers

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
BATCH, AT = 5, 3


def one(seed, n, apart):
    """(1, n): of a batch in columns, or by itself."""
    return numbers(seed, n, BATCH).t()[AT:AT + 1] if apart else numbers(seed, 1, n)


def alone(x, kept):
    """Only the token's own column of its batch was written."""
    if x._base is None:
        return True
    now, kept = x._base.clone(), kept.clone()
    now[:, AT], kept[:, AT] = 0, 0
    return torch.equal(now, kept)


WAYS = list(itertools.product([False, True], repeat=4))


@pytest.mark.parametrize("n,m", [(70, 130), (64, 2048), (130, 1), (1, 130), (1, 1), (4100, 40)])
@pytest.mark.parametrize("ways", WAYS)
def test_linear(n, m, ways):
    W, b = numbers(1, m, n, scale=n ** -0.5), numbers(2, m)
    x, y, r, pre = (one(3 + k, size, way) for k, (size, way) in enumerate(zip((n, m, m, m), ways)))
    kept = [t._base.clone() if t._base is not None else None for t in (y, pre)]
    z, z_slack, want, slack = exact_forward(W, x, b, r, "silu")
    B.linear_matmul(W, x, y, bias=b, residual=r, activation="silu", pre=pre)
    near(y, want, slack, HALF[F32])
    near(pre, z, z_slack, HALF[F32])
    assert alone(y, kept[0]) and alone(pre, kept[1])
    B.linear_matmul(W, x, r, bias=b, residual=r, activation="silu")  # in the residual's own place
    near(r, want, slack, HALF[F32])


@pytest.mark.parametrize("n,m", [(70, 130), (130, 1), (1, 130), (300, 9000)])
@pytest.mark.parametrize("ways", WAYS)
@pytest.mark.parametrize("base", [False, True])
def test_linear_backward(n, m, ways, base):
    W = numbers(1, m, n, scale=n ** -0.5)
    dy, pre, x, dx = (one(3 + k, size, way) for k, (size, way) in enumerate(zip((m, m, n, n), ways)))
    r = one(9, n, ways[0]) if base else None
    dW, db, kept = torch.empty_like(W), torch.empty(m, device="cuda"), dx._base.clone() if dx._base is not None else None
    B.linear_backward(W, dy, X=x, activation="gelu", pre=pre, base=r, dX=dx, dW=dW, dbias=db)
    half, D, A, X = HALF[F32], dy.double().contiguous(), W.double(), x.double().contiguous()
    dz, off = D * act(pre.double().contiguous(), "gelu")[1], 2.0 ** -20 * D.abs()
    rounded = off + half * dz.abs()
    want, slack = dz @ A, rounded @ A.abs() + (m + 8) * 2.0 ** -23 * 1.01 * (dz.abs() @ A.abs())
    if base:
        want, slack = want + r.double(), slack + 2.0 ** -23 * (r.double().abs() + want.abs())
    near(dx, want, slack, half)
    near(dW, dz.t().contiguous() @ X, rounded.t().contiguous() @ X.abs() + 9 * 2.0 ** -23 * 1.01 * (dz.t().contiguous().abs() @ X.abs()), half)
    near(db, dz[0], off[0] + 9 * 2.0 ** -24 * dz[0].abs(), half)
    assert alone(dx, kept)


@pytest.mark.parametrize("n", [1, 8, 75])
@pytest.mark.parametrize("ways", itertools.product([False, True], repeat=3))
def test_dropout(n, ways):
    x, y, r = (one(1 + k, n, way) for k, way in enumerate(ways))
    key, want, kept = torch.tensor([11, 12], dtype=torch.int64, device="cuda"), torch.empty((1, n), device="cuda"), y._base.clone() if y._base is not None else None
    B.dropout_add(x.contiguous(), want, key, 0.4, residual=r.contiguous())
    B.dropout_add(x, y, key, 0.4, residual=r)
    assert torch.equal(y, want) and alone(y, kept)


@pytest.mark.parametrize("n", [1, 8, 515, 9000])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("ways", itertools.product([False, True], repeat=3))
def test_block(n, dtype, ways):
    """The branch's side; the residual stream is in rows."""
    x, g, r, q = numbers(1, 1, n, dtype=dtype), numbers(2, n), torch.rand(1, device="cuda"), torch.rand(1, device="cuda")
    f, y, df = (one(3 + k, n, way) for k, way in enumerate(ways))
    kept = [t._base.clone() if t._base is not None else None for t in (y, df)]
    H, Y, dX, dF, h, dx = (torch.empty_like(t) for t in (x, numbers(4, 1, n), x, numbers(5, 1, n), x, x))
    dy = y.clone().contiguous()
    B.block_norm(x, f.contiguous(), H, Y, gate=g)
    B.block_norm(x, f, h, y, gate=g)
    assert torch.equal(h, H) and torch.equal(y, Y) and alone(y, kept[0])
    y.copy_(dy)
    B.block_norm_backward(dy, x, f.contiguous(), r, dX, dF, rstd_post=q, gate=g)
    B.block_norm_backward(y, x, f, r, dx, df, rstd_post=q, gate=g)
    assert torch.equal(dx, dX) and torch.equal(df, dF) and alone(df, kept[1])


def test_16_bits_in_columns_are_refused():
    x, y, W = numbers(1, BATCH, 8, dtype=BF16, columns=True)[AT:AT + 1], numbers(2, 1, 8, dtype=BF16), numbers(3, 8, 8, dtype=BF16)
    key, r = torch.zeros(2, dtype=torch.int64, device="cuda"), torch.ones(1, device="cuda")
    for call in (lambda: B.linear_matmul(W, x, y), lambda: B.linear_backward(W, x, dX=y), lambda: B.dropout_add(x, y, key, 0.5), lambda: B.block_norm(y, x, y, y.clone()),
                 lambda: B.block_norm_backward(y, y, x, r, y.clone(), y.clone())):
        with pytest.raises(B.CerError):
            call()
