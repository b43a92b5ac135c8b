"""The operators beside a projection against plain implementations in 64 bits on the CPU.

Bounds.  Sums of k products in 32 bits, in any order, are within k . 2^-23 of the sum of the products' magnitudes (an addition of the matrix cores
counted as 2^-23, twice what a rounded one is off); what is stored in fewer bits is off by half a step more: 2^-8 of a value in bf16, 2^-11 in
fp16 (2^-25 where that is subnormal), 2^-4 in e4m3 (2^-10 of the scale below its normal range)."""
import numpy as np
import pytest
import torch

from paper_1805_10692_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16, F16, F8 = torch.float32, torch.bfloat16, torch.float16, torch.float8_e4m3fn
STEP = {F32: 2.0 ** -23, BF16: 2.0 ** -8, F16: 2.0 ** -11, F8: 2.0 ** -4}
TINY = {F32: 0.0, BF16: 0.0, F16: 2.0 ** -25, F8: 2.0 ** -10}
U = 2.0 ** -23
NAN = float("nan")


def put(x, dtype, columns=False, pad=0, off=0):
    """A CPU tensor on the GPU as (tokens, features) of `dtype`: columns or rows, `pad` elements between them, `off` elements into its memory."""
    x = x.t() if columns else x
    room = torch.full((x.shape[0] * (x.shape[1] + pad) + off + 1,), NAN, dtype=F32).to(dtype).cuda()
    view = room[off:off + x.shape[0] * (x.shape[1] + pad)].view(x.shape[0], x.shape[1] + pad)[:, :x.shape[1]]
    view.copy_(x.to(dtype))
    return view.t() if columns else view


def room_for(tokens, n, dtype, columns=False, pad=0, off=0):
    if dtype == F8:
        room = torch.zeros(tokens * (n + pad) + off, dtype=torch.uint8, device="cuda").view(F8)
        return room[off:].view(tokens, n + pad)[:, :n]
    return put(torch.full((tokens, n), 7.0), dtype, columns, pad, off)


def host(x):
    return x.detach().to(F32).cpu().double() if x.dtype == F8 else x.detach().cpu().double()


def near(got, want, bound, what=""):
    got, want = host(got), want.double()
    assert got.shape == want.shape
    fine = torch.isfinite(want)
    assert torch.equal(fine, torch.isfinite(got)), what
    over = ((got - want).abs() - bound)[fine]
    assert over.numel() == 0 or float(over.max()) <= 0, (what, float(over.max()))


def stored(value, dtype, exact_bound):
    """Bound of a value that is off by exact_bound and then stored as dtype."""
    return exact_bound + STEP[dtype] * (value.abs() + exact_bound) + TINY[dtype]


def rand(gen, *shape):
    return torch.randn(shape, generator=gen)


# ---- norm -----------------------------------------------------------------------------------------------------------------------
NORM_SHAPES = [(1, 1), (1, 4096), (2, 7), (3, 64), (5, 1023), (17, 4097), (64, 130), (65, 63), (99, 520), (130, 2048), (2, 8193), (1, 40000), (3, 65536), (700, 33)]
NORM_FORMS = [(F32, F32, False, False), (BF16, BF16, False, False), (F16, F16, False, False), (BF16, F32, False, False), (F32, F8, False, False), (BF16, F8, False, False),
              (F16, F8, False, False), (F32, F32, True, True), (F32, F32, True, False), (F32, F32, False, True), (BF16, F32, False, True), (F16, F32, False, True)]


def norm_oracle(x, r, w, eps):
    h = x if r is None else x + r
    rstd = 1.0 / torch.sqrt((h * h).sum(1) / h.shape[1] + eps)
    return h, rstd, h * rstd[:, None] * (1.0 if w is None else w)


@pytest.mark.parametrize("form", NORM_FORMS, ids=lambda f: f"{f[0]}-{f[1]}-{int(f[2])}{int(f[3])}".replace("torch.", ""))
@pytest.mark.parametrize("shape", NORM_SHAPES, ids=lambda s: f"{s[0]}x{s[1]}")
def test_rms_norm(shape, form):
    (tokens, n), (tx, ty, from_columns, to_columns) = shape, form
    gen = torch.Generator().manual_seed(tokens * 1000 + n)
    case = tokens + n
    eps, pad, off = 1e-5, case % 3, case % 2
    x, r = rand(gen, tokens, n).to(tx).double(), rand(gen, tokens, n).to(tx).double() if case % 4 else None
    tw = (F32, BF16, F16)[case % 3]
    w = (1 + 0.2 * rand(gen, n)).to(tw) if case % 5 else None
    X, R = put(x, tx, from_columns, pad, off), put(r, tx, from_columns, 2 * pad, off) if r is not None else None
    Y, S = room_for(tokens, n, ty, to_columns, pad, off), room_for(tokens, n, tx, from_columns, pad + 1, off)
    scale = torch.empty(tokens, device="cuda") if ty == F8 else None
    rstd = torch.empty(tokens, device="cuda")
    B.rms_norm(X, Y, None if w is None else w.cuda(), residual=R, sum=S, eps=eps, scale=scale, rstd=rstd)
    h, rs, y = norm_oracle(x, r, None if w is None else w.double(), eps)
    near(S, h, stored(h, tx, U * h.abs()), "sum")
    # at most 64 terms one after the other in a thread, and levels over them, half of it in the root
    off32 = 100 * U
    near(rstd, rs, off32 * rs, "rstd")
    if ty != F8:
        near(Y, y, stored(y, ty, off32 * y.abs()), "y")
        return
    most = y.abs().amax(1)
    near(scale, most / 448, 2 * off32 * most / 448, "scale")
    s = host(scale)[:, None]
    near(host(Y) * s, y, stored(y / s, F8, 2 * off32 * (y / s).abs()) * s, "y")


def test_rms_norm_in_place_and_special_tokens():
    gen = torch.Generator().manual_seed(3)
    for tx, columns in ((F32, False), (BF16, False), (F32, True)):
        for to_columns in ((False, True) if tx == F32 else (False, True)):
            x, r = rand(gen, 33, 200).to(tx).double(), rand(gen, 33, 200).to(tx).double()
            x[4], r[4] = 0.0, 0.0
            x[7, 13] = NAN
            x[9, 100] = float("inf")
            h, rs, y = norm_oracle(x, r, None, 1e-6)
            y[9, :] = 0.0  # finite elements over an infinite root
            y[9, 100] = NAN
            X, R = put(x, tx, columns), put(r, tx, columns)
            Y = room_for(33, 200, F32, to_columns)
            B.rms_norm(X, Y, residual=R, sum=R)  # the residual stream updated in its place
            near(R, h, stored(h, tx, U * h.abs()), "sum")
            near(Y, y, 100 * U * y.abs(), "y")
    x = rand(gen, 4, 96)
    x[1] = 0.0
    x[2, 5] = NAN
    Y, scale = room_for(4, 96, F8), torch.empty(4, device="cuda")
    B.rms_norm(put(x, F32), Y, scale=scale)
    s, got = host(scale), host(Y)
    assert s[1] == 1.0 and (got[1] == 0).all()
    assert torch.isnan(s[2]) and torch.isfinite(s[[0, 1, 3]]).all()
    assert float(got[0].abs().max()) == 448.0


def test_rms_norm_empty_batch():
    x = torch.empty((0, 64), device="cuda")
    B.rms_norm(x, torch.empty_like(x))
    dw = torch.full((64,), 5.0, device="cuda")
    B.rms_norm_backward(x, x, torch.empty(0, device="cuda"), torch.empty_like(x), dweight=dw)
    assert (dw == 0).all()


BACK_FORMS = [(F32, F32, False, False), (BF16, BF16, False, False), (F16, F16, False, False), (F32, BF16, False, False), (F32, F32, True, True), (F32, BF16, True, False),
              (F32, F32, True, False)]


def norm_backward_oracle(dy, h, rstd, w, dsum):
    hat = h * rstd[:, None]
    g = dy if w is None else dy * w
    c = (g * hat).mean(1, keepdim=True)
    dx = rstd[:, None] * (g - hat * c) + (0.0 if dsum is None else dsum)
    size = rstd[:, None] * (g.abs() + hat.abs() * (g * hat).abs().mean(1, keepdim=True)) + (0.0 if dsum is None else dsum.abs())
    return dx, size, (dy * hat).sum(0), (dy * hat).abs().sum(0)


@pytest.mark.parametrize("form", BACK_FORMS, ids=lambda f: f"{f[0]}-{f[1]}-{int(f[2])}{int(f[3])}".replace("torch.", ""))
@pytest.mark.parametrize("shape", NORM_SHAPES + [(1500, 48)], ids=lambda s: f"{s[0]}x{s[1]}")
def test_rms_norm_backward(shape, form):
    (tokens, n), (td, th, dy_columns, h_columns) = shape, form
    gen = torch.Generator().manual_seed(tokens * 1000 + n + 1)
    case = tokens + n
    pad, off = case % 3, case % 2
    dy, h = rand(gen, tokens, n).to(td).double(), (2 * rand(gen, tokens, n)).to(th).double()
    dsum = rand(gen, tokens, n).to(th).double() if case % 4 else None
    w = (1 + 0.2 * rand(gen, n)).to((F32, BF16, F16)[case % 3]) if case % 5 else None
    rstd = (1.0 / torch.sqrt((h * h).mean(1) + 1e-5)).float()
    DX, dw = room_for(tokens, n, th, h_columns, pad + 1, off), torch.empty(n, device="cuda")
    DS = put(dsum, th, h_columns, pad, off) if dsum is not None else None
    B.rms_norm_backward(put(dy, td, dy_columns, pad, off), put(h, th, h_columns, pad, off), rstd.cuda(), DX, None if w is None else w.cuda(), dsum=DS, dweight=dw)
    dx, size, want_w, size_w = norm_backward_oracle(dy, h, rstd.double(), None if w is None else w.double(), dsum)
    near(DX, dx, stored(dx, th, 100 * U * size), "dx")
    near(dw, want_w, 100 * U * size_w, "dw")


def test_rms_norm_backward_against_differences():
    """d/dx and d/dw of sum(c . y) by central differences of the forward pass in 64 bits; the kernel's gradients on the same inputs."""
    gen = torch.Generator().manual_seed(11)
    x, c, w = rand(gen, 6, 40).double(), rand(gen, 6, 40).double(), 1 + 0.3 * rand(gen, 40).double()
    x, c, w = x.float().double(), c.float().double(), w.float().double()
    _, rstd, _ = norm_oracle(x, None, w, 1e-5)
    dx, dw = room_for(6, 40, F32), torch.empty(40, device="cuda")
    B.rms_norm_backward(put(c, F32), put(x, F32), rstd.float().cuda(), dx, w.float().cuda(), dweight=dw)
    f = lambda x, w: float((c * norm_oracle(x, None, w, 1e-5)[2]).sum())  # noqa: E731
    step = 1e-5  # differences are off by step^2 times the third derivative (of order 1), and by 2^-52 . |f| / step
    for t, i in ((0, 0), (3, 17), (5, 39)):
        e = torch.zeros_like(x)
        e[t, i] = step
        assert abs((f(x + e, w) - f(x - e, w)) / (2 * step) - float(dx[t, i])) < 1e-4
    for i in (0, 21, 39):
        e = torch.zeros_like(w)
        e[i] = step
        assert abs((f(x, w + e) - f(x, w - e)) / (2 * step) - float(dw[i])) < 1e-4


# ---- adapters -------------------------------------------------------------------------------------------------------------------
def adapters_oracle(A, Bm, scales, ranks, index, x, base):
    """(y, hidden, magnitude of y's terms) in 64 bits."""
    tokens, (N, R, n), m = x.shape[0], A.shape, Bm.shape[1]
    y = base.clone() if base is not None else torch.zeros((tokens, m), dtype=torch.float64)
    size, hidden = y.abs(), torch.zeros((tokens, R), dtype=torch.float64)
    for t in range(tokens):
        a = int(index[t])
        if not 0 <= a < N:
            continue
        r = R if ranks is None else int(ranks[a])
        s = 1.0 if scales is None else float(scales[a])
        hidden[t, :r] = A[a, :r] @ x[t]
        y[t] += s * (Bm[a, :, :r] @ hidden[t, :r])
        size[t] += abs(s) * (Bm[a, :, :r].abs() @ (A[a, :r].abs() @ x[t].abs()))
    return y, hidden, size


def backward_oracle(A, Bm, scales, ranks, index, dy, x, hidden, base):
    tokens, (N, R, n), m = x.shape[0], A.shape, Bm.shape[1]
    dx = base.clone() if base is not None else torch.zeros((tokens, n), dtype=torch.float64)
    dA, dB = torch.zeros_like(A), torch.zeros_like(Bm)
    sx, sA, sB = dx.abs(), torch.zeros_like(A), torch.zeros_like(Bm)
    for t in range(tokens):
        a = int(index[t])
        if not 0 <= a < N:
            continue
        r = R if ranks is None else int(ranks[a])
        s = 1.0 if scales is None else float(scales[a])
        d, size = s * (dy[t] @ Bm[a, :, :r]), abs(s) * (dy[t].abs() @ Bm[a, :, :r].abs())
        dx[t] += d @ A[a, :r]
        sx[t] += size @ A[a, :r].abs()
        dA[a, :r] += torch.outer(d, x[t])
        sA[a, :r] += torch.outer(size, x[t].abs())
        dB[a, :, :r] += s * torch.outer(dy[t], hidden[t, :r])
        sB[a, :, :r] += abs(s) * torch.outer(dy[t].abs(), hidden[t, :r].abs())
    return dx, sx, dA, sA, dB, sB


def index_of(kind, tokens, N, seed):
    rng = np.random.RandomState(seed)
    if kind == "runs":
        cuts = np.sort(rng.randint(0, tokens + 1, 5))
        which = rng.randint(-1, N, 6)
        return torch.tensor(np.repeat(which, np.diff(np.concatenate([[0], cuts, [tokens]]))), dtype=torch.int32)
    if kind == "any":
        return torch.tensor(rng.randint(-2, N + 2, tokens), dtype=torch.int32)  # also outside 0 .. N - 1
    if kind == "none":
        return torch.full((tokens,), -1, dtype=torch.int32)
    return torch.full((tokens,), N - 1, dtype=torch.int32)


ADAPTER_TYPES = [(F32, F32, False), (F32, F32, True), (F32, BF16, True), (F32, F16, True), (F32, BF16, False), (F32, F16, False), (BF16, BF16, False), (F16, F16, False)]
#: tokens, in, out, adapters, rank, index
ADAPTER_SHAPES = [(1, 64, 64, 1, 16, "last"), (1, 257, 131, 3, 5, "last"), (2, 1, 1, 2, 1, "any"), (7, 700, 190, 4, 8, "any"), (16, 96, 1000, 20, 17, "any"), (64, 320, 256, 70, 16, "any"),
                  (65, 33, 65, 2, 33, "runs"), (130, 512, 64, 3, 64, "none"), (257, 129, 96, 5, 24, "runs"), (300, 200, 320, 9, 100, "any"), (1030, 70, 90, 3, 16, "runs"),
                  (1100, 40, 72, 2, 130, "runs"), (2100, 64, 40, 3, 8, "any"), (40, 300, 80, 2, 256, "runs")]
#: many tokens: whole and broken tiles of 64 by 64, ranks in eights and not, more adapters in a tile than are taken together
WIDE_SHAPES = [(320, 256, 128, 4, 16, "runs"), (513, 200, 193, 3, 24, "any"), (449, 640, 330, 6, 40, "runs"), (385, 129, 257, 5, 64, "any"), (300, 65, 200, 2, 72, "runs"), (640, 320, 64, 1, 128, "last"),
               (260, 140, 150, 2, 200, "runs"), (333, 90, 100, 3, 36, "any"), (700, 1100, 70, 90, 8, "any"),
               (400, 130, 192, 3, 4, "runs"), (330, 192, 130, 2, 12, "runs"), (350, 100, 128, 2, 100, "runs")]


def make_adapters(shape, types, ragged):
    tokens, n, m, N, R, kind = shape
    ta, tw, columns = types
    gen = torch.Generator().manual_seed(tokens + n)
    A, Bm = (rand(gen, N, R, n) / n ** 0.5).to(tw).double(), (rand(gen, N, m, R) / R ** 0.5).to(tw).double()
    scales = (rand(gen, N) + 0.1) if tokens % 3 else None
    ranks = torch.randint(0, R + 1, (N,), generator=gen, dtype=torch.int32) if ragged else None
    return gen, A, Bm, scales, ranks, index_of(kind, tokens, N, tokens)


def on_gpu(w, tw, pad, ranks=None, rank_dim=None):
    """Adapters with gaps between rows, NaN in the gaps and past every adapter's own rank."""
    N, p, q = w.shape
    out = torch.full((N, p + 1, q + pad), NAN).to(tw).cuda()
    w = w.clone()
    if ranks is not None:
        for a in range(N):
            w.select(0, a).narrow(rank_dim - 1, int(ranks[a]), w.shape[rank_dim] - int(ranks[a])).fill_(NAN)
    out[:, :p, :q] = w.to(tw).cuda()
    return out[:, :p, :q]


def opt(x):
    return None if x is None else x.cuda()


@pytest.mark.parametrize("types", ADAPTER_TYPES, ids=lambda t: f"{t[0]}-{t[1]}-{int(t[2])}".replace("torch.", ""))
@pytest.mark.parametrize("shape", ADAPTER_SHAPES + WIDE_SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_adapter_matmul(shape, types):
    tokens, n, m, N, R, kind = shape
    ta, tw, columns = types
    ragged, pad = (tokens + n) % 2 == 1, n % 3
    gen, A, Bm, scales, ranks, index = make_adapters(shape, types, ragged)
    x, base = rand(gen, tokens, n).to(ta).double(), rand(gen, tokens, m).to(ta).double()
    y, hidden, size = adapters_oracle(A, Bm, scales, ranks, index, x, base)
    GA, GB = on_gpu(A, tw, pad, ranks, 1), on_gpu(Bm, tw, pad, ranks, 2)
    X, Bs = put(x, ta, columns, pad, 1), put(base, ta, columns, 1, pad)
    bound = stored(y, ta, (n + R + 8) * U * size)
    Y, H = room_for(tokens, m, ta, columns, pad, 1), torch.full((tokens, R), NAN, device="cuda")
    B.adapter_matmul(GA, GB, index.cuda(), X, Y, scales=opt(scales), ranks=opt(ranks), base=Bs, hidden=H)
    near(Y, y, bound, "y")
    in_size = torch.stack([A[int(a)].abs() @ x[t].abs() if 0 <= a < N else torch.zeros(R, dtype=torch.float64) for t, a in enumerate(index)])
    near(H, hidden, (n + 8) * U * in_size, "hidden")
    # without a base; in the base's own place, with the caller's workspace
    y0, _, size0 = adapters_oracle(A, Bm, scales, ranks, index, x, None)
    B.adapter_matmul(GA, GB, index.cuda(), X, Y, scales=opt(scales), ranks=opt(ranks))
    near(Y, y0, stored(y0, ta, (n + R + 8) * U * size0), "without base")
    work = torch.full((B.adapter_workspace_bytes(tokens, R, n, m) // 4,), NAN, device="cuda")
    B.adapter_matmul(GA, GB, index.cuda(), X, Bs, scales=opt(scales), ranks=opt(ranks), base=Bs, workspace=work)
    near(Bs, y, bound, "in place")


@pytest.mark.parametrize("types", ADAPTER_TYPES, ids=lambda t: f"{t[0]}-{t[1]}-{int(t[2])}".replace("torch.", ""))
@pytest.mark.parametrize("shape", ADAPTER_SHAPES + WIDE_SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_adapter_backward(shape, types):
    tokens, n, m, N, R, kind = shape
    ta, tw, columns = types
    ragged, pad = (tokens + n) % 2 == 0, m % 3
    gen, A, Bm, scales, ranks, index = make_adapters(shape, types, ragged)
    x, dy, base = rand(gen, tokens, n).to(ta).double(), rand(gen, tokens, m).to(ta).double(), rand(gen, tokens, n).to(ta).double() if tokens % 2 else None
    hidden = rand(gen, tokens, R).double()
    dx, sx, dA, sA, dB, sB = backward_oracle(A, Bm, scales, ranks, index, dy, x, hidden, base)
    GA, GB = on_gpu(A, tw, pad, ranks, 1), on_gpu(Bm, tw, pad, ranks, 2)
    H = hidden.float().cuda()
    for t, a in enumerate(index):  # what does not belong to the token's adapter is not looked at
        r = 0 if not 0 <= a < N else R if ranks is None else int(ranks[a])
        H[t, r:] = NAN
    DX = room_for(tokens, n, ta, columns, pad, 1)
    GdA, GdB = torch.full((N, R, n), NAN, device="cuda"), torch.full((N, m, R), NAN, device="cuda")
    B.adapter_backward(GA, GB, index.cuda(), put(dy, ta, columns, pad, 1), put(x, ta, columns, 1, pad), H, scales=opt(scales), ranks=opt(ranks),
                       base=None if base is None else put(base, ta, columns, pad, 0), dX=DX, dA=GdA, dB=GdB)
    near(DX, dx, stored(dx, ta, (m + R + 8) * U * sx), "dx")
    near(GdA, dA, (m + tokens + 8) * U * sA, "dA")
    near(GdB, dB, (tokens + 8) * U * sB, "dB")


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("types", [(F32, False), (F32, True), (BF16, False), (F16, False)], ids=lambda t: f"{t[0]}-{int(t[1])}".replace("torch.", ""))
def test_adapters_keep_requests_apart(types, wide):
    """A request of NaN and infinities between two others, one whose adapter is NaN, and an adapter of NaN that nobody has: nothing of them shows elsewhere."""
    ta, columns = types
    gen = torch.Generator().manual_seed(5)
    n, m, N, R = 100, 140, 5, 16
    tokens = 400 if wide else 97
    A, Bm = rand(gen, N, R, n).to(ta).double(), rand(gen, N, m, R).to(ta).double()
    x, dy, base = rand(gen, tokens, n).to(ta).double(), rand(gen, tokens, m).to(ta).double(), rand(gen, tokens, m).to(ta).double()
    index = torch.tensor([0] * 20 + [1] * 13 + [-1] * 7 + [2] * (tokens - 47) + [4] * 7, dtype=torch.int32)
    clean, hidden, size = adapters_oracle(A, Bm, None, None, index, x, base)
    dx, sx, dA, sA, dB, sB = backward_oracle(A, Bm, None, None, index, dy, x, hidden, None)
    A[3:], Bm[3:] = NAN, NAN
    x[20:40], dy[20:40], base[20:33] = NAN, float("inf"), NAN
    hidden[20:40] = NAN
    GA, GB, I = A.to(ta).cuda(), Bm.to(ta).cuda(), index.cuda()
    Y = room_for(tokens, m, ta, columns)
    B.adapter_matmul(GA, GB, I, put(x, ta, columns), Y, base=put(base, ta, columns))
    fine = [t for t in range(tokens - 7) if not 20 <= t < 33]
    near(Y[fine], clean[fine], stored(clean, ta, (n + R + 8) * U * size)[fine], "y")
    assert torch.isnan(host(Y)[20:33]).all() and torch.isnan(host(Y)[-7:]).all()
    DX, GdA, GdB = room_for(tokens, n, ta, columns), torch.empty((N, R, n), device="cuda"), torch.empty((N, m, R), device="cuda")
    B.adapter_backward(GA, GB, I, put(dy, ta, columns), put(x, ta, columns), hidden.float().cuda(), dX=DX, dA=GdA, dB=GdB)
    near(DX[fine], dx[fine], stored(dx, ta, (m + R + 8) * U * sx)[fine], "dx")
    for a in (0, 2, 3):
        near(GdA[a], dA[a], (m + tokens + 8) * U * sA[a], "dA")
        near(GdB[a], dB[a], (tokens + 8) * U * sB[a], "dB")
    assert (host(GdA)[3] == 0).all() and (host(GdB)[3] == 0).all()


def test_adapter_backward_against_differences():
    """The forward pass is linear in x, in A and in B, so that a central difference of any step is the derivative; both by the kernels."""
    gen = torch.Generator().manual_seed(9)
    tokens, n, m, N, R = 70, 60, 50, 3, 6
    A, Bm, x, c = (rand(gen, *s).cuda() for s in ((N, R, n), (N, m, R), (tokens, n), (tokens, m)))
    index, scales = index_of("runs", tokens, N, 1).cuda(), torch.tensor([0.5, 1.5, -2.0], device="cuda")
    Y, H = torch.empty((tokens, m), device="cuda"), torch.empty((tokens, R), device="cuda")

    def f(A, Bm, x):
        B.adapter_matmul(A, Bm, index, x, Y, scales=scales, hidden=H)
        return float((Y.double() * c.double()).sum())

    f(A, Bm, x)
    dX, dA, dB = torch.empty_like(x), torch.empty_like(A), torch.empty_like(Bm)
    B.adapter_backward(A, Bm, index, c, x, H, scales=scales, dX=dX, dA=dA, dB=dB)
    # each f is a sum of about tokens . m . R . n products in 32 bits of size 1: off by some 1e-6 of its magnitude sum (below 2e6)
    for k, (p, g) in enumerate(((A, dA), (Bm, dB), (x, dX))):
        e = torch.randn(p.shape, generator=torch.Generator().manual_seed(k)).cuda()
        args = [A, Bm, x]
        args[k] = p + e
        up = f(*args)
        args[k] = p - e
        down = f(*args)
        assert abs((up - down) / 2 - float((g.double() * e.double()).sum())) < 2.0


def test_adapter_empty_batch():
    A, Bm = torch.ones((2, 4, 8), device="cuda"), torch.ones((2, 6, 4), device="cuda")
    x, y, index = torch.empty((0, 8), device="cuda"), torch.empty((0, 6), device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    B.adapter_matmul(A, Bm, index, x, y)
    dA, dB = torch.full_like(A, 3), torch.full_like(Bm, 3)
    B.adapter_backward(A, Bm, index, y, x, torch.empty((0, 4), device="cuda"), dA=dA, dB=dB)
    assert (dA == 0).all() and (dB == 0).all()


def test_results_repeat_and_streams():
    """The same bits again, on another stream, and from a graph replayed between other work."""
    gen = torch.Generator().manual_seed(21)
    tokens, n, m, N, R = 40, 512, 256, 6, 16
    A, Bm = rand(gen, N, R, n).to(BF16).cuda(), rand(gen, N, m, R).to(BF16).cuda()
    index = index_of("any", tokens, N, 2).cuda()
    x, base = put(rand(gen, tokens, n), F32, True), put(rand(gen, tokens, m), F32, True)
    Y = room_for(tokens, m, F32, True)
    work = torch.empty(B.adapter_workspace_bytes(tokens, R, n, m) // 4, device="cuda")
    B.adapter_matmul(A, Bm, index, x, Y, base=base, workspace=work)
    first = Y.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.adapter_matmul(A, Bm, index, x, Y.zero_(), base=base)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(first, Y)
    B.adapter_matmul(A, Bm, index, x, Y.zero_(), base=base, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    out = torch.empty_like(base.t())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.adapter_matmul(A, Bm, index, x, Y, base=base, workspace=work)
        B.rms_norm(base.t(), out)
    for k in range(3):
        Y.zero_()
        x.mul_(2.0) if k else None
        graph.replay()
        torch.cuda.synchronize()
        want = room_for(tokens, m, F32, True)
        B.adapter_matmul(A, Bm, index, x, want, base=base)
        assert torch.equal(want, Y)
        other = torch.empty_like(out)
        B.rms_norm(base.t(), other)
        assert torch.equal(other, out)


# ---- clipping -------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("limit", [0.3, 5.0, 0.0])
@pytest.mark.parametrize("sizes", [[1], [0, 7, 0], [8192, 8193, 8191, 1], [100_000, 3], [5] * 400, []], ids=str)
def test_grad_clip(sizes, limit):
    if len(sizes) > 10:
        sizes = [1 + (i * 37) % 900 for i in range(len(sizes))]
    gen = torch.Generator().manual_seed(len(sizes))
    types = (F32, BF16, F16)
    grads = [rand(gen, k + 1).to(types[i % 3]) for i, k in enumerate(sizes)]
    grads = [g[i % 2:][:k] for i, (g, k) in enumerate(zip(grads, sizes))]  # some not at a multiple of 16 bytes
    count = max(1, sum(sizes))
    want = float(np.sqrt(sum(float((g.double() ** 2).sum()) for g in grads)))
    most = limit * count ** 0.5
    c = min(1.0, most / (want + 1e-6))
    G = []
    for i, g in enumerate(grads):
        room = torch.zeros(g.numel() + 1, dtype=g.dtype, device="cuda")
        G.append(room[i % 2:][:g.numel()])
        G[-1].copy_(g)
    outs, norm = [torch.full_like(g, 9.0) for g in G], torch.full((1,), NAN, device="cuda")
    B.grad_clip(G, most, norm, outs=outs)
    assert abs(float(norm) - want) <= 2 * U * want
    for g, o, s in zip(grads, outs, G):
        near(o, g.double() * c, stored(g.double() * c, o.dtype, 4 * U * g.double().abs() * c), "out")
        assert torch.equal(s.cpu(), g)
    alone = torch.full((1,), NAN, device="cuda")
    B.grad_norm(G, alone)
    assert torch.equal(alone, norm)
    B.grad_clip(G, most, norm)  # in place
    for s, o in zip(G, outs):
        assert torch.equal(s, o)


def test_grad_clip_large_values_and_nan():
    big = torch.full((1000,), 1e30, device="cuda")  # squares of which are past fp32
    norm = torch.empty(1, device="cuda")
    B.grad_clip([big], 1.0, norm)
    assert abs(float(norm) / (1e30 * 1000 ** 0.5) - 1) < 1e-6
    near(big, torch.full((1000,), 1000 ** -0.5), 1e-6 * 1000 ** -0.5)
    for bad, then in ((NAN, NAN), (float("inf"), 0.0)):
        g = [torch.ones(10, device="cuda"), torch.tensor([bad, 1.0], device="cuda")]
        B.grad_clip(g, 1.0, norm)
        assert not np.isfinite(float(norm))
        assert (host(g[0]) == then).all() if then == 0.0 else torch.isnan(g[0]).all()
        assert torch.isnan(g[1][0])


def test_refusals():
    x = torch.ones((4, 64), device="cuda")
    y, w, norm = torch.empty_like(x), torch.ones(64, device="cuda"), torch.empty(1, device="cuda")
    with pytest.raises(ValueError, match="device memory"):
        B.rms_norm(x.cpu(), y)
    with pytest.raises(ValueError, match="shape"):
        B.rms_norm(x, torch.empty((4, 63), device="cuda"))
    with pytest.raises(ValueError, match="dimensions"):
        B.rms_norm(x[0], y)
    with pytest.raises(ValueError, match="contiguous"):
        B.rms_norm(torch.ones((4, 128), device="cuda")[:, ::2], y)
    with pytest.raises(ValueError, match="float32"):
        B.rms_norm(x.double(), y)
    with pytest.raises(TypeError, match="required"):
        B.rms_norm(x)
    with pytest.raises(TypeError, match="unexpected"):
        B.rms_norm(x, y, bias=w)
    with pytest.raises(ValueError, match="number of elements"):
        B.rms_norm(x, y, w[:3])
    for bad in (lambda: B.rms_norm(x, y.to(BF16)),                      # not X's type
                lambda: B.rms_norm(x, y.to(F8)),                        # no scale
                lambda: B.rms_norm(x, y, scale=torch.empty(4, device="cuda")),
                lambda: B.rms_norm(x, y, eps=-1.0),
                lambda: B.rms_norm(x, y, residual=x.to(BF16)),
                lambda: B.rms_norm(x.to(BF16).t().contiguous().t(), y),   # columns of 16 bits
                lambda: B.rms_norm(x, y[:1].expand(4, 64)),               # an output that overlaps itself
                lambda: B.rms_norm(torch.ones((1, 70000), device="cuda"), torch.empty((1, 70000), device="cuda")),
                lambda: B.rms_norm_backward(x, x.t().contiguous().t(), torch.ones(4, device="cuda"), y.t().contiguous().t()),
                lambda: B.grad_clip([x], -1.0, norm), lambda: B.grad_clip([x], NAN, norm)):
        with pytest.raises(B.CerError):
            bad()
    A, Bm = torch.ones((2, 8, 64), device="cuda"), torch.ones((2, 32, 8), device="cuda")
    index, out = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.empty((4, 32), device="cuda")
    with pytest.raises(ValueError, match="A's type"):
        B.adapter_matmul(A, Bm.to(BF16), index, x, out)
    with pytest.raises(ValueError, match="rank"):
        B.adapter_matmul(A, Bm[:, :, :4], index, x, out)
    with pytest.raises(ValueError, match="int32"):
        B.adapter_matmul(A, Bm, index.long(), x, out)
    with pytest.raises(ValueError, match="number of elements"):
        B.adapter_matmul(A, Bm, index[:3], x, out)
    for bad in (lambda: B.adapter_matmul(A.to(F16), Bm.to(F16), index, x.to(BF16), out.to(BF16)),
                lambda: B.adapter_matmul(A, Bm, index, x.to(BF16), out.to(BF16)),
                lambda: B.adapter_matmul(A, Bm, index, x, out.t().contiguous().t()),
                lambda: B.adapter_matmul(A, Bm, index, x, out, workspace=torch.empty(1, device="cuda")),
                lambda: B.adapter_matmul(torch.ones((1, 257, 64), device="cuda"), torch.ones((1, 32, 257), device="cuda"), index, x, out)):
        with pytest.raises(B.CerError):
            bad()
    with pytest.raises(ValueError, match="as many"):
        B.grad_clip([x], 1.0, norm, outs=[])
    with pytest.raises(ValueError, match="contiguous"):
        B.grad_norm([x.t()], norm)
