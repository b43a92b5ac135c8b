"""The operators beside a projection at sizes where offsets are long and every loop of a kernel goes round, against vectorised forms in 64 bits on the GPU.

The adapters' numbers are small whole ones and their factors powers of two, so that every sum is exact in 32 bits in any order and only an output in 16 bits is rounded:
results are equal to the 64-bit form's, rounded, and not only near them.  Norm and clipping: bounds as in test_gpu_operators.py."""
import pytest
import torch

from paper_1805_10692_amd import binding as B
from test_gpu_operators import BF16, F8, F16, F32, STEP, TINY, U

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


def close(got, want, bound, what):
    over = (got.double() - want).abs() - bound
    assert float(over.max()) <= 0, (what, float(over.max()))


def stored(value, dtype, exact_bound):
    return exact_bound + STEP[dtype] * (value.abs() + exact_bound) + TINY[dtype]


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


# tokens, features, adapters, rank: a wave of the product back to the long axis has blocks of it behind one another, the contraction over the long axis goes round its
# buffers, and one workgroup goes through more tokens than one list of them holds
@pytest.mark.parametrize("types", [(F32, F32, True), (F32, BF16, True), (F32, F16, True), (F32, F32, False), (F32, BF16, False), (F32, F16, False), (BF16, BF16, False), (F16, F16, False)],
                         ids=lambda t: f"{t[0]}-{t[1]}-{int(t[2])}".replace("torch.", ""))
@pytest.mark.parametrize("shape", [(8261, 2600, 2570, 60, 16), (8300, 2580, 2630, 55, 36), (8257, 2600, 2600, 48, 64), (8200, 1540, 2600, 50, 100), (8193, 2570, 2580, 3, 24), (4300, 1600, 640, 2, 200)],
                         ids=lambda s: "-".join(map(str, s)))
def test_many_tokens(shape, types):
    tokens, n, m, N, R = shape
    gen = torch.Generator().manual_seed(tokens)
    cuts = torch.sort(torch.randint(0, tokens, (2 * N,), generator=gen))[0]
    index = ((torch.searchsorted(cuts, torch.arange(tokens), right=True) * 7) % (N + 1) - 1).to(torch.int32).cuda()
    ranks = None if N % 2 else torch.randint(0, R + 1, (N,), generator=gen).to(torch.int32).cuda()
    adapters_exactly(tokens, n, m, N, R, types[:2], types[2], index, ranks)


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (F16, F32), (BF16, F8)], ids=str)
def test_norm_of_more_than_a_million_tokens(types):
    """More tokens than the launch has workgroups.  Sums of 8 squares: 16 . 2^-23 with the root and the products (the scale's maximum and quotients: as much again)."""
    tx, ty = types
    tokens, n = (1 << 20) + 3, 8
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, r, w = (torch.randn(s, generator=gen, device="cuda").to(t) for s, t in (((tokens, n), tx), ((tokens, n), tx), ((n,), F32)))
    y, total, rstd = torch.zeros((tokens, n), dtype=torch.uint8, device="cuda").view(F8) if ty == F8 else torch.empty((tokens, n), dtype=ty, device="cuda"), torch.empty_like(x), torch.empty(tokens, device="cuda")
    scale = torch.empty(tokens, device="cuda") if ty == F8 else None
    B.rms_norm(x, y, w, residual=r, sum=total, scale=scale, rstd=rstd)
    h = x.double() + r.double()
    rs = 1.0 / torch.sqrt((h * h).mean(1) + 1e-6)
    want = h * rs[:, None] * w.double()
    close(total, h, stored(h, tx, U * h.abs()), "sum")
    close(rstd, rs, 16 * U * rs, "rstd")
    if ty == F8:
        s = scale.double()[:, None]
        close(scale, want.abs().amax(1) / 448, 32 * U * want.abs().amax(1) / 448, "scale")
        close(y.float().double() * s, want, stored(want / s, F8, 32 * U * (want / s).abs()) * s, "y")
    else:
        close(y, want, stored(want, ty, 16 * U * want.abs()), "y")
    dy, dx, dw = torch.randn((tokens, n), generator=gen, device="cuda").to(tx), torch.empty_like(x), torch.empty(n, device="cuda")
    B.rms_norm_backward(dy, total, rstd, dx, w, dweight=dw)
    hat, g = total.double() * rstd.double()[:, None], dy.double() * w.double()
    c, size = (g * hat).mean(1, keepdim=True), (g * hat).abs().mean(1, keepdim=True)
    rs = rstd.double()[:, None]
    close(dx, rs * (g - hat * c), stored(rs * (g - hat * c), tx, 32 * U * rs * (g.abs() + hat.abs() * size)), "dx")
    # a workgroup adds up every 512th token, the second launch 512 sums in a tree of at most 8 and 6 levels
    close(dw, (dy.double() * hat).sum(0), (tokens // 512 + 20) * U * (dy.double() * hat).abs().sum(0), "dw")


def test_clipping_past_the_caches():
    """More than 256 MiB of gradients and outputs: stores that do not stay in the caches; odd lengths and places."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    sizes = [(30_000_001, F32, 1), (20_000_003, BF16, 1), (8192 * 5, F16, 0), (1_000_001, F16, 3), (77, F32, 0)]
    G = [torch.randn(k + off, generator=gen, device="cuda").to(t)[off:] for k, t, off in sizes]
    outs, norm = [torch.empty(k + off, dtype=t, device="cuda")[off:] for k, t, off in sizes], torch.empty(1, device="cuda")
    B.grad_clip(G, 1000.0, norm, outs=outs)
    want = float(sum((g.double() ** 2).sum() for g in G)) ** 0.5
    assert want > 1000 and abs(float(norm) - want) <= 2 * U * want
    c = 1000.0 / (want + 1e-6)
    for g, o in zip(G, outs):
        close(o, g.double() * c, stored(g.double() * c, o.dtype, 4 * U * g.double().abs() * c), "out")
    kept = [o.clone() for o in outs]
    B.grad_clip(G, 1000.0, norm)  # in place: below 256 MiB together
    assert all(torch.equal(g, o) for g, o in zip(G, kept))
