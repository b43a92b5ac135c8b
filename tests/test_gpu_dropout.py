"""dropout_add against its generator in whole numbers on the host: the mask has to be equal, the values are off by the product's and the sum's rounding."""
import numpy as np
import pytest
import torch

from block_reference import HALF, SMALLEST, near, numbers16
from paper_1805_10692_amd import binding as B

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
SEED, OFFSET = 0x123456789ABCDEF0 - 2 ** 64 // 4, -5


def numbers(seed, *shape, dtype=F32, columns=False):
    x = torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)
    return x.t().contiguous().t() if columns else x


def key(seed=SEED, offset=OFFSET):
    return torch.tensor([seed, offset], dtype=torch.int64, device="cuda")


def want_of(x, p, r=None, seed=SEED, offset=OFFSET):
    d = int(np.rint(p * 65536))
    keep = torch.from_numpy(numbers16(*x.shape, seed, offset) >= d).cuda()
    y = torch.where(keep, x.double() * (65536 / (65536 - d) if d < 65536 else 0.0), torch.zeros((), dtype=torch.float64, device="cuda"))
    return keep, y if r is None else y + r.double(), 2.0 ** -23 * y.abs() + (0 if r is None else 2.0 ** -24 * (y.abs() + r.double().abs()))


@pytest.mark.parametrize("tokens,n", [(1, 1), (1, 8), (5, 7), (3, 65), (70, 33), (130, 256), (1, 5001), (301, 20)])
@pytest.mark.parametrize("dtype,columns", [(F32, False), (F32, True), (BF16, False), (F16, False)])
@pytest.mark.parametrize("residual", [False, True])
def test_values(tokens, n, dtype, columns, residual):
    x, r = numbers(1, tokens, n, dtype=dtype, columns=columns), numbers(2, tokens, n, dtype=dtype, columns=columns) if residual else None
    y = numbers(3, tokens, n, dtype=dtype, columns=columns)
    B.dropout_add(x, y, key(), 0.3, residual=r)
    keep, want, slack = want_of(x, 0.3, r)
    near(y, want, slack + SMALLEST[dtype], HALF[dtype])
    if not residual:
        assert torch.equal(y != 0, keep & (x != 0))


@pytest.mark.parametrize("p", [0.0, 2.0 ** -18, 2.0 ** -16, 0.5, 1 - 2.0 ** -16, 1.0])
def test_probabilities(p):
    x, y = numbers(4, 40, 100), torch.empty((40, 100), device="cuda")
    B.dropout_add(x, y, key(), p)
    _, want, slack = want_of(x, p)
    near(y, want, slack, HALF[F32])
    if p < 2.0 ** -17:
        assert torch.equal(x, y)


def test_share_and_mean():
    """4 M numbers: the share that is kept has a standard deviation of sqrt(p (1 - p) / 2^22) = 2.0e-4 (six of them are allowed), and pairs of neighbours are independent."""
    x = torch.ones((2048, 2048), device="cuda")
    y = torch.empty_like(x)
    B.dropout_add(x, y, key(), 0.2)
    kept = (y != 0).double()
    assert abs(float(kept.mean()) - (1 - round(0.2 * 65536) / 65536)) < 6 * 2e-4
    assert abs(float((kept[:, 1:] * kept[:, :-1]).mean()) - 0.64) < 6 * 2.4e-4 and abs(float((kept[1:] * kept[:-1]).mean()) - 0.64) < 6 * 2.4e-4
    assert abs(float(y.mean()) - 1) < 6 * 2.5e-4


def test_key_and_call():
    x = torch.ones((30, 50), device="cuda")
    outs = []
    for k, call in ((key(), 0), (key(), 3), (key(offset=OFFSET + 3), 0), (key(seed=SEED + 1), 0), (key(offset=2 ** 63 - 1), 1), (key(offset=-2 ** 63), 0)):
        y = torch.empty_like(x)
        B.dropout_add(x, y, k, 0.5, call=call)
        outs.append(y)
    assert torch.equal(outs[1], outs[2]) and torch.equal(outs[4], outs[5])
    for other in (1, 3, 4):
        assert not torch.equal(outs[0], outs[other])


def test_mask_does_not_depend_on_the_layout():
    x = numbers(5, 37, 91)
    rows, columns, wide, half = torch.empty_like(x), torch.empty((91, 37), device="cuda").t(), torch.full((37, 100), 7.0, device="cuda"), torch.empty((37, 91), dtype=BF16, device="cuda")
    B.dropout_add(x, rows, key(), 0.4)
    B.dropout_add(x.t().contiguous().t(), columns, key(), 0.4)
    B.dropout_add(x, wide[:, 3:94], key(), 0.4)
    B.dropout_add(x.to(BF16), half, key(), 0.4)
    assert torch.equal(rows, columns) and torch.equal(rows, wide[:, 3:94]) and torch.equal(rows != 0, half != 0)
    assert bool((wide[:, :3] == 7).all()) and bool((wide[:, 94:] == 7).all())


def test_in_place_and_broadcast():
    x, r = numbers(6, 20, 30, dtype=BF16), numbers(7, 20, 30, dtype=BF16)
    want, a, b = torch.empty_like(x), x.clone(), r.clone()
    B.dropout_add(x, want, key(), 0.25, residual=r)
    B.dropout_add(a, a, key(), 0.25, residual=r)
    B.dropout_add(x, b, key(), 0.25, residual=b)
    assert torch.equal(a, want) and torch.equal(b, want)
    B.dropout_add(x[:1].expand(20, 30), a, key(), 0.25)
    B.dropout_add(x[:1].expand(20, 30).contiguous(), b, key(), 0.25)
    assert torch.equal(a, b)


def test_dropped_infinities():
    x, r = torch.full((40, 40), float("inf"), device="cuda"), torch.ones((40, 40), device="cuda")
    x[::2] = float("nan")
    y = torch.empty_like(x)
    B.dropout_add(x, y, key(), 0.5, residual=r)
    keep = want_of(x, 0.5)[0]
    assert bool((y[~keep] == 1).all()) and not bool(y[keep].isfinite().any())


def test_backward_is_the_same_call():
    x, dy = numbers(8, 50, 60), numbers(9, 50, 60)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    B.dropout_add(x, y, key(), 0.3)
    B.dropout_add(dy, dx, key(), 0.3)
    ones = torch.empty_like(x)
    B.dropout_add(torch.ones_like(x), ones, key(), 0.3)
    assert torch.equal(dx, dy * ones) and torch.equal(y, x * ones)


def test_no_tokens():
    none = torch.empty((0, 8), device="cuda")
    B.dropout_add(none, none, key(), 0.5)


def test_a_recorded_call_has_new_masks_with_a_new_key():
    x, y, k = numbers(10, 64, 100), torch.empty((64, 100), device="cuda"), key()
    B.dropout_add(x, y, k, 0.5)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.dropout_add(x, y, k, 0.5)
    seen = []
    for step in range(4):
        k[1] += 1
        y.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        seen.append(y.clone())
        want = torch.empty_like(x)
        B.dropout_add(x, want, key(offset=OFFSET + step + 1), 0.5)
        assert torch.equal(y, want)
    assert not torch.equal(seen[0], seen[1])


def test_on_another_stream():
    x = numbers(11, 300, 400)
    want, y, s = torch.empty_like(x), torch.empty_like(x), torch.cuda.Stream()
    B.dropout_add(x, want, key(), 0.5)
    k = key()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        B.dropout_add(x, y, k, 0.5)
    s.synchronize()
    assert torch.equal(y, want)
