"""The operators beside a projection at sizes where offsets are long and every loop of a kernel goes round, against vectorised forms in 64 bits on the GPU.

The adapters' numbers are small whole ones and their factors powers of two, so that every sum is exact in 32 bits in any order and only an output in 16 bits is rounded:
results are equal to the 64-bit form's, rounded, and not only near them."""
import pytest
import torch

from paper_1805_10692_amd import binding as B
from test_gpu_operators import F32

pytestmark = pytest.mark.gpu


def whole(seed, most, *shape):
    """Whole numbers up to `most` of either sign, as 32-bit floats."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=gen, device="cuda").float()


def order(x, columns):
    """(tokens, features) with the features side by side or the tokens."""
    return x.t().contiguous().t() if columns else x.contiguous()


def equal(got, want, what):
    off = (got != want.to(got.dtype)).nonzero()
    assert len(off) == 0, (what, len(off), off[:3].tolist())


def adapters_exactly(tokens, n, m, N, R, types, columns, index, ranks=None, base=True):
    ta, tw = types
    A, Bm, scales = whole(1, 1, N, R, n).to(tw), whole(2, 1, N, m, R).to(tw), torch.exp2(whole(3, 1, N))
    x, dy = order(whole(4, 1, tokens, n).to(ta), columns), order(whole(5, 1, tokens, m).to(ta), columns)
    hidden = torch.empty((tokens, R), device="cuda")
    y, dx, dA, dB = torch.empty_like(dy), torch.empty_like(x), torch.empty((N, R, n), device="cuda"), torch.empty((N, m, R), device="cuda")
    to_y, to_dx = (order(whole(6, 9, tokens, m).to(ta), columns), order(whole(7, 9, tokens, n).to(ta), columns)) if base else (None, None)
    B.adapter_matmul(A, Bm, index, x, y, scales=scales, ranks=ranks, base=to_y, hidden=hidden)
    B.adapter_backward(A, Bm, index, dy, x, hidden, scales=scales, ranks=ranks, base=to_dx, dX=dx, dA=dA, dB=dB)
    for a in range(-1, N):
        at = (index == a).nonzero()[:, 0]
        r = R if ranks is None or a < 0 else int(ranks[a])
        of_y, of_x = (0.0, 0.0) if to_y is None else (to_y[at].double(), to_dx[at].double())
        if a < 0:
            equal(y[at], torch.zeros_like(y[at]) + of_y, "y, no adapter")
            equal(dx[at], torch.zeros_like(dx[at]) + of_x, "dx, no adapter")
            continue
        xs, ds, w, v, s = x[at].double(), dy[at].double(), A[a, :r].double(), Bm[a, :, :r].double(), float(scales[a])
        h = xs @ w.t().contiguous()
        d = s * (ds @ v.contiguous())
        equal(hidden[at, :r], h, f"hidden {a}")
        equal(y[at], of_y + s * (h @ v.t().contiguous()), f"y {a}")
        equal(dx[at], of_x + d @ w, f"dx {a}")
        equal(dA[a, :r], d.t().contiguous() @ xs, f"dA {a}")
        equal(dB[a, :, :r], s * (ds.t().contiguous() @ h), f"dB {a}")
        assert (dA[a, r:] == 0).all() and (dB[a, :, r:] == 0).all()


def test_columns_of_more_than_four_million_tokens():
    """include/cer.h: up to 2^24 tokens, in either order."""
    tokens = (1 << 22) + 70
    index = (torch.arange(tokens, device="cuda") // 1000 % 4 - 1).to(torch.int32)
    adapters_exactly(tokens, 8, 64, 3, 4, (F32, F32), True, index, base=False)
