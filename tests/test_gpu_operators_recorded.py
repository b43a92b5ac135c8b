"""The operators beside a projection recorded into a HIP graph where they use temporaries of their own: replays between eager work, on new numbers, give what eager calls give."""
import pytest
import torch

from paper_1805_10692_amd import binding as B

pytestmark = pytest.mark.gpu
TOKENS, IN, OUT, RANK, N = 99, 520, 300, 8, 3


def numbers(seed, *shape, columns=False):
    x = torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")
    return x.t().contiguous().t() if columns else x


def norm(x_columns, y_columns):
    x, y, rstd = numbers(1, TOKENS, IN, columns=x_columns), numbers(2, TOKENS, IN, columns=y_columns), torch.empty(TOKENS, device="cuda")
    return lambda: B.rms_norm(x, y, rstd=rstd), [x], [y, rstd]


def norm_backward(dy_columns, h_columns):
    dy, h, dx = numbers(3, TOKENS, IN, columns=dy_columns), numbers(4, TOKENS, IN, columns=h_columns), numbers(5, TOKENS, IN, columns=h_columns)
    rstd, dw = torch.ones(TOKENS, device="cuda"), torch.empty(IN, device="cuda")
    return lambda: B.rms_norm_backward(dy, h, rstd, dx, dweight=dw), [dy, h], [dx, dw]


def adapters(columns, backward):
    A, Bm, index = numbers(6, N, RANK, IN), numbers(7, N, OUT, RANK), (torch.arange(TOKENS, device="cuda") // 20 % (N + 1) - 1).int()
    x, y, hidden = numbers(8, TOKENS, IN, columns=columns), numbers(9, TOKENS, OUT, columns=columns), numbers(10, TOKENS, RANK)
    if not backward:
        return lambda: B.adapter_matmul(A, Bm, index, x, y, hidden=hidden), [x, A], [y, hidden]
    dx, dA, dB = torch.empty_like(x), torch.empty_like(A), torch.empty_like(Bm)
    return lambda: B.adapter_backward(A, Bm, index, y, x, hidden, dX=dx, dA=dA, dB=dB), [y, x], [dx, dA, dB]


def clip():
    g, out, total = numbers(11, 70_001), torch.empty(70_001, device="cuda"), torch.empty(1, device="cuda")
    return lambda: B.grad_clip([g], 1.0, total, outs=[out]), [g], [out, total]


CALLS = {"rows to columns": lambda: norm(False, True), "columns to columns": lambda: norm(True, True), "columns to rows": lambda: norm(True, False),
         "gradient, rows": lambda: norm_backward(False, False), "gradient, columns": lambda: norm_backward(True, True), "gradient, mixed": lambda: norm_backward(True, False),
         "adapters, rows": lambda: adapters(False, False), "adapters, columns": lambda: adapters(True, False), "adapters' gradients, rows": lambda: adapters(False, True),
         "adapters' gradients, columns": lambda: adapters(True, True), "clipping": clip}


@pytest.mark.parametrize("name", CALLS)
def test_recorded(name):
    call, inputs, outputs = CALLS[name]()
    call()  # once eagerly: what is set up at a first call
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(4):
        for x in inputs:
            x.mul_(0.75).add_(0.1 * (k + 1))
        for y in outputs:
            y.fill_(-1.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [y.clone() for y in outputs]
        for y in outputs:
            y.fill_(-2.0)
        call()
        torch.cuda.synchronize()
        for a, b in zip(got, outputs):
            assert torch.equal(a, b), (name, k)
