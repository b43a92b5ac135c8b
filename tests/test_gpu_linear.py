"""linear_matmul and linear_backward against the formulas in 64 bits, for every type, order and tile.

What a result may be off by: products of two 16-bit numbers are exact in 32 bits, so a sum of k terms is within (k + 8) . 2^-23 of the terms' sizes
(the matrix instruction cuts where it adds); an activation passes on at most 1.13 of that and adds 16 . 2^-24 of |z|; what goes out is rounded once.  In the backward
pass dZ itself has half a step of the type and 2^-20 of dY from the slope."""
import pytest
import torch

from block_reference import HALF, SMALLEST, act, near
from paper_1805_10692_amd import binding as B

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
SIZES = [(1, 1, 1), (1, 8, 8), (16, 3000, 2050), (33, 130, 2), (9, 77, 3001), (31, 700, 18), (70, 66, 3), (257, 72, 258), (3, 5, 7), (2, 4099, 515), (17, 64, 33), (65, 130, 257), (128, 64, 128), (200, 515, 130), (300, 1000, 70)]
LARGE = [(2100, 200, 1900), (4100, 136, 3401),  # tiles of 128 and (16 bits) 256
         (40, 9001, 67), (130, 4100, 1030), (4099, 1032, 4611)]  # parts of the contraction: of all tiles, of the last ones


def numbers(seed, *shape, dtype=F32, columns=False, scale=1.0):
    x = (torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * scale).to(dtype)
    return x.t().contiguous().t() if columns else x


def exact_forward(W, x, bias, r, name):
    X, A = x.double().contiguous(), W.double().t().contiguous()
    z = X @ A
    slack = (W.shape[1] + 8) * 2.0 ** -23 * (X.abs() @ A.abs())
    if bias is not None:
        z = z + bias.double()
        slack = slack + 2.0 ** -23 * bias.double().abs()
    y = act(z, name)[0]
    return z, slack, y if r is None else y + r.double(), 1.13 * slack + 2.0 ** -20 * z.abs() + (0 if r is None else 2.0 ** -23 * (r.double().abs() + y.abs()))


def check_forward(tokens, n, m, dtype, name, bias=True, residual=False, columns=False, keep=True):
    W, x = numbers(1, m, n, dtype=dtype, scale=n ** -0.5), numbers(2, tokens, n, dtype=dtype, columns=columns)
    b = numbers(3, m) if bias else None
    r = numbers(4, tokens, m, dtype=dtype, columns=columns) if residual else None
    y, pre = numbers(5, tokens, m, dtype=dtype, columns=columns), numbers(6, tokens, m, dtype=dtype, columns=columns) if keep else None
    B.linear_matmul(W, x, y, bias=b, residual=r, activation=name, pre=pre)
    z, z_slack, want, slack = exact_forward(W, x, b, r, name)
    near(y, want, slack + SMALLEST[dtype], HALF[dtype])
    if keep:
        near(pre, z, z_slack + SMALLEST[dtype], HALF[dtype])


@pytest.mark.parametrize("tokens,n,m", SIZES + LARGE)
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_forward(tokens, n, m, dtype):
    check_forward(tokens, n, m, dtype, "silu")
    check_forward(tokens, n, m, dtype, "none", bias=False, residual=True, keep=False)


@pytest.mark.parametrize("tokens,n,m", SIZES + LARGE[:1] + LARGE[2:4])
def test_forward_columns(tokens, n, m):
    check_forward(tokens, n, m, F32, "gelu", columns=True, residual=True)


@pytest.mark.parametrize("name", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_activations(name, dtype):
    check_forward(33, 40, 260, dtype, name, residual=True)


@pytest.mark.parametrize("name", ["relu", "gelu", "gelu_tanh", "silu"])
def test_activations_over_their_range(name):
    """One feature in, a weight of 1: Z is X, and the limits are those of the functions."""
    z = torch.cat([torch.linspace(-40, 40, 4001, device="cuda"), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 200.0, -200.0, 1e20, -1e20, 3e38, -3e38], device="cuda")])[:, None]
    W, y = torch.ones((1, 1), device="cuda"), torch.empty_like(z)
    B.linear_matmul(W, z, y, activation=name)
    want = act(z.double(), name)[0]
    want = torch.where(z < -100, torch.zeros_like(want), want)
    # the share of z is exp(u) below: u, down to -104 where it is 0, has a relative error of 2^-21; below the normal numbers it may be cut
    assert bool(((y.double() - want).abs() <= 53 * 2.0 ** -20 * want.abs() + 2.0 ** -125 * z.double().abs()).all())
    ends = torch.tensor([[float("inf")], [float("-inf")], [float("nan")]], device="cuda")
    out = torch.empty_like(ends)
    B.linear_matmul(W, ends, out, activation=name)
    assert out[0] == float("inf") and out[1] == 0 and bool(out[2].isnan())
    dz = torch.empty_like(z)
    B.linear_backward(W, torch.ones_like(z), activation=name, pre=z, dX=dz)
    slopes = torch.where(z < -100, torch.zeros_like(want), torch.where(z > 100, torch.ones_like(want), act(z.double(), name)[1]))
    assert float((dz.double() - slopes).abs().max()) <= 2.0 ** -20
    dz = torch.empty_like(ends)
    B.linear_backward(W, torch.ones_like(ends), activation=name, pre=ends, dX=dz)
    assert dz[0] == 1 and dz[1] == 0 and bool(dz[2].isnan())


def check_backward(tokens, n, m, dtype, name, columns=False, base=False):
    W, x = numbers(11, m, n, dtype=dtype, scale=n ** -0.5), numbers(12, tokens, n, dtype=dtype, columns=columns)
    dy, z = numbers(13, tokens, m, dtype=dtype, columns=columns), numbers(14, tokens, m, dtype=dtype, columns=columns)
    r = numbers(15, tokens, n, dtype=dtype, columns=columns) if base else None
    dx, dW, db = numbers(16, tokens, n, dtype=dtype, columns=columns), numbers(17, m, n, dtype=dtype), numbers(18, m)
    pre = z if name != "none" else None
    B.linear_backward(W, dy, X=x, activation=name, pre=pre, base=r, dX=dx, dW=dW, dbias=db)
    D, A, X = dy.double().contiguous(), W.double(), x.double().contiguous()
    half = HALF[dtype]
    if pre is None:
        dz, off = D, torch.zeros_like(D)
    else:
        dz = D * act(z.double().contiguous(), name)[1]
        off = 2.0 ** -20 * D.abs()
    rounded = off if pre is None else off + half * dz.abs() + SMALLEST[dtype]
    want = dz @ A
    slack = rounded @ A.abs() + (m + 8) * 2.0 ** -23 * (dz.abs() @ A.abs()) * 1.01
    if r is not None:
        want, slack = want + r.double(), slack + 2.0 ** -23 * (r.double().abs() + want.abs())
    near(dx, want, slack + SMALLEST[dtype], half)
    near(dW, dz.t().contiguous() @ X, rounded.t().contiguous() @ X.abs() + (tokens + 8) * 2.0 ** -23 * 1.01 * (dz.t().contiguous().abs() @ X.abs()) + SMALLEST[dtype], half)
    near(db, dz.sum(0), off.sum(0) + (tokens + 8) * 2.0 ** -24 * dz.abs().sum(0), HALF[F32])


@pytest.mark.parametrize("tokens,n,m", SIZES + LARGE)
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_backward(tokens, n, m, dtype):
    check_backward(tokens, n, m, dtype, "gelu_tanh", base=True)
    check_backward(tokens, n, m, dtype, "none")


@pytest.mark.parametrize("tokens,n,m", SIZES + LARGE[:1] + LARGE[2:4])
def test_backward_columns(tokens, n, m):
    check_backward(tokens, n, m, F32, "silu", columns=True, base=True)
    check_backward(tokens, n, m, F32, "none", columns=True)


@pytest.mark.parametrize("name", ["relu", "gelu"])
def test_backward_activations(name):
    check_backward(70, 50, 90, BF16, name)
    check_backward(70, 50, 90, F32, name)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tokens,n,m", [(37, 67, 45), (4, 200, 90)])
def test_strides_and_what_lies_around(tokens, n, m, dtype):
    """Odd leading dimensions and odd addresses; what lies beside an output stays as it was."""
    W, x, r = numbers(21, m, n + 5, dtype=dtype)[:, 3:n + 3], numbers(22, tokens + 1, n + 9, dtype=dtype)[1:, 1:n + 1], numbers(23, tokens, m + 1, dtype=dtype)[:, 1:]
    around = numbers(24, tokens + 2, m + 7, dtype=dtype)
    kept, y = around.clone(), around[1:-1, 3:m + 3]
    B.linear_matmul(W, x, y, residual=r)
    _, _, want, slack = exact_forward(W, x, None, r, "none")
    near(y, want, slack, HALF[dtype])
    kept[1:-1, 3:m + 3] = y
    assert torch.equal(kept, around)
    wide, plain = numbers(25, m + 2, n + 3, dtype=dtype), torch.empty((m, n), dtype=dtype, device="cuda")
    kept, dW, dy = wide.clone(), wide[1:-1, 2:n + 2], numbers(26, tokens, m, dtype=dtype)
    dx, dx2 = numbers(27, tokens, n + 1, dtype=dtype)[:, :n], torch.empty((tokens, n), dtype=dtype, device="cuda")
    B.linear_backward(W, dy, X=x, dX=dx, dW=dW)
    B.linear_backward(W.contiguous(), dy, X=x.contiguous(), dX=dx2, dW=plain)
    kept[1:-1, 2:n + 2] = dW
    assert torch.equal(kept, wide) and torch.equal(dW, plain) and torch.equal(dx, dx2)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_broadcast_inputs_and_in_place(dtype):
    W, x, r = numbers(31, 70, 40, dtype=dtype), numbers(32, 1, 40, dtype=dtype), numbers(33, 50, 70, dtype=dtype)
    y = r.clone()
    B.linear_matmul(W, x.expand(50, 40), y, residual=y, activation="relu")
    _, _, one, slack = exact_forward(W, x.expand(50, 40), None, r, "relu")
    near(y, one, slack, HALF[dtype])
    want = torch.empty_like(y)
    B.linear_matmul(W, x.expand(50, 40).contiguous(), want, residual=r, activation="relu")
    assert torch.equal(y, want)
    dx, base = numbers(34, 50, 40, dtype=dtype), None
    base = dx.clone()
    B.linear_backward(W, r, base=dx, dX=dx)
    two = torch.empty_like(dx)
    B.linear_backward(W, r, base=base, dX=two)
    assert torch.equal(dx, two)
    # a gradient that is the same for all tokens
    B.linear_backward(W, r[:1].expand(50, 70), dX=dx)
    B.linear_backward(W, r[:1].expand(50, 70).contiguous(), dX=two)
    assert torch.equal(dx, two)


@pytest.mark.parametrize("tokens,n,m", [(33, 67, 45), (300, 1000, 70), (2100, 72, 1900)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_infinite_numbers_stay_in_their_rows(tokens, n, m, dtype):
    W, x = numbers(41, m, n, dtype=dtype), numbers(42, tokens, n, dtype=dtype)
    clean, y = torch.empty((tokens, m), dtype=dtype, device="cuda"), torch.empty((tokens, m), dtype=dtype, device="cuda")
    B.linear_matmul(W, x, clean)
    bad_x, bad_W = x.clone(), W.clone()
    bad_x[-1, n - 1], bad_x[tokens // 2, 0], bad_W[m - 1, n - 1] = float("nan"), float("inf"), float("inf")
    B.linear_matmul(bad_W, bad_x, y)
    rows = torch.ones(tokens, dtype=torch.bool, device="cuda")
    rows[-1] = rows[tokens // 2] = False
    assert torch.equal(y[rows][:, :-1], clean[rows][:, :-1])
    assert bool(y[-1].isnan().all()) and bool(y[tokens // 2, :-1].isinf().all()) and bool(y[rows][:, -1].isinf().all())


def test_no_tokens():
    W = numbers(51, 40, 30, dtype=BF16)
    none_in, none_out = torch.empty((0, 30), dtype=BF16, device="cuda"), torch.empty((0, 40), dtype=BF16, device="cuda")
    B.linear_matmul(W, none_in, none_out)
    dW, db = torch.ones_like(W), torch.ones(40, device="cuda")
    B.linear_backward(W, none_out, X=none_in, dX=none_in, dW=dW, dbias=db)
    assert not dW.any() and not db.any()


def test_a_dropped_gradient_takes_nothing_along():
    """Where relu is flat, an infinite dY leaves no trace."""
    W, pre, dy = numbers(61, 5, 4), torch.tensor([[1.0, -1.0, 2.0, -2.0, 0.0]], device="cuda"), torch.tensor([[1.0, float("inf"), 1.0, float("nan"), float("-inf")]], device="cuda")
    dx, db = torch.empty((1, 4), device="cuda"), torch.empty(5, device="cuda")
    B.linear_backward(W, dy, activation="relu", pre=pre, dX=dx, dbias=db)
    assert db.tolist() == [1, 0, 1, 0, 0] and torch.equal(dx, (W[0] + W[2])[None])


@pytest.mark.parametrize("name", ["gelu", "gelu_tanh", "silu"])
def test_gradients_against_differences(name):
    """A central difference with step h is off by h^2 / 6 of a third derivative (below 4 for each of these, times |w|^3) and by rounding 2^-20 / h: h = 2^-6."""
    tokens, n, m, h = 4, 6, 5, 2.0 ** -6
    W, x, b, dy = numbers(71, m, n, scale=0.4), numbers(72, tokens, n, scale=0.5), numbers(73, m, scale=0.3), numbers(74, tokens, m)

    def loss(W, x, b):
        y = torch.empty((tokens, m), device="cuda")
        B.linear_matmul(W, x, y, bias=b, activation=name)
        return float((y.double() * dy.double()).sum())

    y, pre = torch.empty((tokens, m), device="cuda"), torch.empty((tokens, m), device="cuda")
    B.linear_matmul(W, x, y, bias=b, activation=name, pre=pre)
    dx, dW, db = torch.empty_like(x), torch.empty_like(W), torch.empty_like(b)
    B.linear_backward(W, dy, X=x, activation=name, pre=pre, dX=dx, dW=dW, dbias=db)
    for which, got in ((0, dW), (1, dx), (2, db)):
        for at in range(got.numel()):
            both = []
            for sign in (1, -1):
                moved = [W.clone(), x.clone(), b.clone()]
                moved[which].view(-1)[at] += sign * h
                both.append(loss(*moved))
            slack = float(dy.abs().sum()) * (4 * h * h / 6 * max(1.0, float(W.abs().max()), float(x.abs().max())) ** 3 + 4 * 2.0 ** -20 / h)
            assert abs((both[0] - both[1]) / (2 * h) - float(got.view(-1)[at])) <= slack


@pytest.mark.parametrize("tokens", [50, 1200])
@pytest.mark.parametrize("dtype,columns", [(BF16, False), (F32, False), (F32, True)])
def test_gradients_that_are_not_wanted(tokens, dtype, columns):
    n, m = 90, 130
    W, x = numbers(81, m, n, dtype=dtype), numbers(82, tokens, n, dtype=dtype, columns=columns)
    dy, z = numbers(83, tokens, m, dtype=dtype, columns=columns), numbers(84, tokens, m, dtype=dtype, columns=columns)
    every = {"dX": torch.empty_like(x), "dW": torch.empty_like(W), "dbias": torch.empty(m, device="cuda")}
    for name, pre in (("silu", z), ("none", None)):
        B.linear_backward(W, dy, X=x, activation=name, pre=pre, **every)
        for k, want in every.items():
            one = torch.empty_like(want)
            B.linear_backward(W, dy, X=x if k == "dW" else None, activation=name, pre=pre, **{k: one})
            assert torch.equal(one, want), (name, k)
    B.linear_backward(W, dy)  # nothing is wanted


def at_offset(x, offset):
    room = torch.full((x.numel() + offset,), float("nan"), dtype=x.dtype, device="cuda")
    to = room[offset:].view(x.shape)
    to.copy_(x)
    return to


# One step of 128 bytes of the contraction, fewer and more of them than are under way, with and without a rest; one workgroup to a compute unit and several; each tile.
@pytest.mark.parametrize("tokens,n,m", [(70, 64, 80), (70, 128, 80), (70, 192, 66), (70, 320, 66), (65, 456, 70), (1000, 64, 1030), (1000, 200, 1030), (1030, 512, 4100), (2050, 264, 4100), (4097, 192, 4700)])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_where_the_operands_lie_changes_nothing(tokens, n, m, dtype):
    """Rows on 16 bytes and rows that are not go different ways into LDS: the same sums in the same order."""
    W, x = numbers(1, m, n, dtype=dtype), numbers(2, tokens, n, dtype=dtype)
    got = [torch.empty((tokens, m), dtype=dtype, device="cuda") for _ in range(3)]
    B.linear_matmul(W, x, got[0])
    B.linear_matmul(at_offset(W, 1), x, got[1])
    B.linear_matmul(W, at_offset(x, 3), got[2])
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])
    want = x.double() @ W.double().t().contiguous()
    near(got[0], want, (n + 8) * 2.0 ** -23 * (x.double().abs() @ W.double().abs().t().contiguous()) + SMALLEST[dtype], HALF[dtype])


@pytest.mark.parametrize("tokens,n,m", [(64, 72, 64), (128, 80, 128), (192, 72, 192), (328, 64, 456), (72, 1032, 1000), (520, 2056, 264), (200, 4104, 1032), (4168, 264, 1032), (264, 4616, 4104)])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("columns", [False, True])
def test_where_the_operands_of_gradients_lie_changes_nothing(tokens, n, m, dtype, columns):
    """An operand that is turned where it is read, and one that is turned on its way."""
    if columns and dtype != F32:
        dtype = F32
        tokens, n, m = n, tokens, m  # another order of the sizes instead of a type that has no columns
    W, x, dy = numbers(1, m, n, dtype=dtype), numbers(2, *((n, tokens) if columns else (tokens, n)), dtype=dtype), numbers(3, *((m, tokens) if columns else (tokens, m)), dtype=dtype)
    turned = (lambda t: t.t()) if columns else (lambda t: t)

    def gradients(W, x, dy):
        dx, dw = torch.empty_like(x), torch.empty_like(W)
        B.linear_backward(W, turned(dy), X=turned(x), dX=turned(dx), dW=dw)
        return turned(dx), dw

    want = gradients(W, x, dy)
    for other in ((at_offset(W, 1), x, dy), (W, at_offset(x, 3), dy), (W, x, at_offset(dy, 1))):
        for a, b in zip(want, gradients(*other)):
            assert torch.equal(a, b)
    W, x, dy = W.double(), turned(x).double().contiguous(), turned(dy).double().contiguous()
    near(want[0], dy @ W, (m + 8) * 2.0 ** -23 * (dy.abs() @ W.abs()) + SMALLEST[dtype], HALF[dtype])
    d = dy.t().contiguous()
    near(want[1], d @ x, (tokens + 8) * 2.0 ** -23 * (d.abs() @ x.abs()) + SMALLEST[dtype], HALF[dtype])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("ld", [(1 << 21) - 8, 1 << 21, (1 << 21) + 8])
def test_rows_far_apart(ld, dtype):
    tokens, n, m = 200, 264, 136
    W, x, dy = numbers(1, m, n, dtype=dtype), numbers(2, tokens, n, dtype=dtype), numbers(3, tokens, m, dtype=dtype)
    room = torch.empty((tokens, ld), dtype=dtype, device="cuda")
    far = room[:, :n].copy_(x)
    want, got = (torch.empty((tokens, m), dtype=dtype, device="cuda") for _ in range(2))
    B.linear_matmul(W, x, want)
    B.linear_matmul(W, far, got)
    assert torch.equal(want, got)
    want, got = torch.empty_like(W), torch.empty_like(W)
    B.linear_backward(W, dy, X=x, dW=want)
    B.linear_backward(W, dy, X=far, dW=got)
    assert torch.equal(want, got)
    far = room[:m, 8:n + 8].copy_(W)
    want, got = torch.empty_like(x), torch.empty_like(x)
    B.linear_backward(W, dy, dX=want)
    B.linear_backward(far, dy, dX=got)
    assert torch.equal(want, got)


@pytest.mark.parametrize("bias_type", [BF16, F16])
@pytest.mark.parametrize("tokens,columns", [(3, False), (100, False), (3, True), (100, True)])
def test_types_of_the_bias(tokens, columns, bias_type):
    W, x, b = numbers(91, 70, 40), numbers(92, tokens, 40, columns=columns), numbers(93, 70, dtype=bias_type)
    y, want = numbers(94, tokens, 70, columns=columns), numbers(95, tokens, 70, columns=columns)
    B.linear_matmul(W, x, y, bias=b)
    B.linear_matmul(W, x, want, bias=b.float())
    assert torch.equal(y, want)


def test_arguments_are_checked():
    W, x, y = numbers(1, 6, 4), numbers(2, 3, 4), numbers(3, 3, 6)
    for bad in (lambda: B.linear_matmul(W, x, x), lambda: B.linear_matmul(W, y, y), lambda: B.linear_matmul(W.to(BF16), x, y), lambda: B.linear_matmul(W, x, y, bias=numbers(4, 5)),
                lambda: B.linear_matmul(W, x, y, activation="tanh"), lambda: B.linear_matmul(W, x, y, activation=1), lambda: B.linear_matmul(W.t(), y, x), lambda: B.linear_matmul(W[0], x, y),
                lambda: B.linear_matmul(W, x, y, workspace=torch.empty(4, dtype=BF16, device="cuda")), lambda: B.linear_backward(W, y, X=x, dW=numbers(5, 4, 6)),
                lambda: B.linear_backward(W, y, X=x, dbias=numbers(6, 6, dtype=BF16)), lambda: B.linear_backward(W, y, dW=W.clone()), lambda: B.linear_backward(W, y, activation="relu", dX=x)):
        with pytest.raises((ValueError, B.CerError)):
            bad()
