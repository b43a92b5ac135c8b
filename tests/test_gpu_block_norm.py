"""block_norm and block_norm_backward against the formulas in 64 bits.

What a result may be off by: a sum of n squares or products formed in 32 bits by at most 64 steps a thread, wave and workgroup is within (n / 64 + 80) . 2^-24 of its terms'
sizes (here: 200 . 2^-24 up to 7680 features, 700 . 2^-24 up to 32768), half of which an inverse root passes on; every further operation adds 2^-24; a result is rounded once."""
import pytest
import torch

from block_reference import HALF, SMALLEST, near
from paper_1805_10692_amd import binding as B

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
EPS = 1e-5


def numbers(seed, *shape, dtype=F32, columns=False, scale=1.0):
    x = (torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * scale).to(dtype)
    return x.t().contiguous().t() if columns else x


def steps(n):
    return (200 if n <= 7680 else 700) * 2.0 ** -24


def make_gate(kind, tokens, n, dtype):
    return None if kind == "none" else numbers(3, n) if kind == "features" else numbers(3, tokens, n, dtype=dtype)


def forward(tokens, n, dtype, branch, gate="features", post=True, columns=(False, False), out=None, weights=True, scale=0.75):
    out = out or branch
    x, f, g = numbers(1, tokens, n, dtype=dtype), numbers(2, tokens, n, dtype=branch, columns=columns[0]), make_gate(gate, tokens, n, dtype)
    a, b = (numbers(4, n), numbers(5, n)) if weights else (None, None)
    h, y = torch.empty_like(x), numbers(6, tokens, n, dtype=out, columns=columns[1])
    q, r = torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda")
    B.block_norm(x, f, h, y, gate=g, post_weight=a if post else None, pre_weight=b, scale=scale, eps=EPS, post=post, rstd_post=q if post else None, rstd_pre=r)
    s = steps(n)
    u = f.double().contiguous()
    slack = torch.zeros_like(u)
    if post:
        root = torch.rsqrt((u * u).mean(1, keepdim=True) + EPS)
        near(q[:, None], root, s * root, HALF[F32])
        u = u * root * (1.0 if a is None else a.double())
        slack = (s + 4 * 2.0 ** -24) * u.abs()
    if g is not None:
        u, slack = u * g.double(), slack * g.double().abs() + 2.0 ** -24 * (u * g.double()).abs()
    want = scale * x.double() + u
    slack = slack + 2.0 ** -23 * ((scale * x.double()).abs() + u.abs())
    near(h, want, slack + SMALLEST[dtype], HALF[dtype])
    root = torch.rsqrt((want * want).mean(1, keepdim=True) + EPS)
    off = s + (slack * want.abs()).mean(1, keepdim=True) * root ** 2  # of the root, relative: from its sum, and from h
    near(r[:, None], root, off * root, HALF[F32])
    w = 1.0 if b is None else b.double()
    near(y, want * root * w, (slack + (off + 4 * 2.0 ** -24) * want.abs()) * root * (1.0 if b is None else w.abs()) + SMALLEST[out], HALF[out])


SIZES = [(1, 1), (1, 8), (3, 7), (5, 64), (2, 515), (130, 96), (7, 4096), (3, 7679), (600, 33)]


@pytest.mark.parametrize("tokens,n", SIZES + [(2, 8193), (3, 12001), (2, 20000), (2, 32768)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_forward(tokens, n, dtype):
    forward(tokens, n, dtype, dtype)


@pytest.mark.parametrize("gate", ["none", "features", "tokens"])
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("dtype,branch,out", [(BF16, F32, BF16), (F16, F16, F32), (BF16, F32, F32), (F32, F32, F32)])
def test_forward_forms(gate, post, dtype, branch, out):
    forward(9, 200, dtype, branch, gate, post, out=out, weights=gate != "none")


@pytest.mark.parametrize("tokens,n", [(1, 1), (1, 70), (70, 1), (65, 67), (130, 515), (3, 4100)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("columns", [(True, False), (False, True), (True, True)])
def test_forward_columns(tokens, n, dtype, columns):
    forward(tokens, n, dtype, F32, columns=columns)


def backward(tokens, n, dtype, branch, gate="features", post=True, columns=(False, False), dy_type=None, weights=True, through=True, scale=0.75):
    dy_type = dy_type or branch
    h, f, g = numbers(11, tokens, n, dtype=dtype), numbers(12, tokens, n, dtype=branch, columns=columns[1]), make_gate(gate, tokens, n, dtype)
    dy, dh = numbers(13, tokens, n, dtype=dy_type, columns=columns[0]), numbers(14, tokens, n, dtype=dtype) if through else None
    a, b = (numbers(4, n) if post else None, numbers(5, n)) if weights else (None, None)
    r, q = torch.rsqrt(h.float().square().mean(1) + EPS), torch.rsqrt(f.float().square().mean(1) + EPS) if post else None
    dx, df = torch.empty_like(h), numbers(15, tokens, n, dtype=branch, columns=columns[1])
    dg, da, db = None if g is None else torch.empty_like(g), numbers(16, n) if post else None, numbers(17, n)
    B.block_norm_backward(dy, h, f, r, dx, df, rstd_post=q, gate=g, post_weight=a, pre_weight=b, scale=scale, dsum=dh, dgate=dg, dpost_weight=da, dpre_weight=db)
    e, s = 2.0 ** -24, steps(n)
    H, F, Y = h.double(), f.double().contiguous(), dy.double().contiguous()
    R, Q = r.double()[:, None], q.double()[:, None] if post else torch.ones((tokens, 1), dtype=torch.float64, device="cuda")
    A, Bw, G = (torch.ones(n, dtype=torch.float64, device="cuda") if v is None else v.double() for v in (a, b, g))
    hat, fhat, k = H * R, F * Q, Y * Bw
    mean, size = (k * hat).mean(1, keepdim=True), (k * hat).abs().mean(1, keepdim=True)
    d = R * (k - hat * mean)
    slack = R * (6 * e * k.abs() + hat.abs() * ((s + 6 * e) * size))
    if dh is not None:
        d, slack = d + dh.double(), slack + 2 * e * (d.abs() + dh.double().abs())
    near(dx, scale * d, abs(scale) * (slack + e * d.abs()) + SMALLEST[dtype], HALF[dtype])
    many = (tokens + 40) * e
    near(db, (Y * hat).sum(0), many * (Y * hat).abs().sum(0), HALF[F32])
    u = fhat * A
    if gate != "none":
        off = slack * u.abs() + 4 * e * (d * u).abs()
        if gate == "features":
            near(dg, (d * u).sum(0), off.sum(0) + many * (d * u).abs().sum(0), HALF[F32])
        else:
            near(dg, d * u, off + SMALLEST[dtype], HALF[dtype])
    du, slack = d * G, slack * G.abs() + e * (d * G).abs()
    want, off = du, slack
    if post:
        near(da, (du * fhat).sum(0), (slack * fhat.abs()).sum(0) + (many + 4 * e) * (du * fhat).abs().sum(0), HALF[F32])
        E = du * A
        off = slack * A.abs() + e * E.abs()
        mean, size = (E * fhat).mean(1, keepdim=True), (E * fhat).abs().mean(1, keepdim=True)
        want = Q * (E - fhat * mean)
        off = Q * (off + 4 * e * E.abs() + fhat.abs() * ((s + 8 * e) * size + (off * fhat.abs()).mean(1, keepdim=True)))
    near(df, want, off + SMALLEST[branch], HALF[branch])


@pytest.mark.parametrize("tokens,n", SIZES + [(2, 8192), (2, 8193), (70, 12001), (2, 20000), (2, 32768), (300, 6144), (300, 6145), (1500, 130), (3100, 40), (700, 1000)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_backward(tokens, n, dtype):
    backward(tokens, n, dtype, dtype)


@pytest.mark.parametrize("gate", ["none", "features", "tokens"])
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("n", [200, 9000])
@pytest.mark.parametrize("dtype,branch,dy_type", [(BF16, F32, BF16), (F16, F16, F32), (BF16, F32, F32), (F32, F32, F32)])
def test_backward_forms(gate, post, dtype, branch, dy_type, n):
    backward(9, n, dtype, branch, gate, post, dy_type=dy_type, weights=gate != "none", through=post)


@pytest.mark.parametrize("tokens,n", [(1, 1), (1, 70), (70, 1), (65, 67), (130, 515), (600, 40)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("columns", [(True, False), (False, True), (True, True)])
def test_backward_columns(tokens, n, dtype, columns):
    backward(tokens, n, dtype, F32, "tokens", columns=columns)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strides_in_place_and_what_lies_around(dtype):
    tokens, n = 11, 77
    x, f, wide = numbers(21, tokens, n + 3, dtype=dtype)[:, 2:n + 2], numbers(22, tokens, n, dtype=dtype), numbers(23, tokens + 2, n + 5, dtype=dtype)
    h, y = torch.empty((tokens, n), dtype=dtype, device="cuda"), torch.empty((tokens, n), dtype=dtype, device="cuda")
    B.block_norm(x, f, h, y)
    kept, inner = wide.clone(), wide[1:-1, 3:n + 3]
    h2 = x.clone()
    B.block_norm(h2, f, h2, inner)  # the residual stream in its own place
    kept[1:-1, 3:n + 3] = y
    assert torch.equal(h, h2) and torch.equal(wide, kept)
    f2 = f.clone()
    B.block_norm(x, f2, h2, f2)
    assert torch.equal(f2, y) and torch.equal(h2, h)
    # a token's numbers for all tokens, also as the gate of each
    one = numbers(24, 1, n, dtype=dtype)
    B.block_norm(one.expand(tokens, n), f, h, y, gate=one.expand(tokens, n))
    B.block_norm(one.expand(tokens, n).contiguous(), f, h2, inner, gate=one.expand(tokens, n).contiguous())
    assert torch.equal(h, h2) and torch.equal(y, inner)


@pytest.mark.parametrize("n", [64, 9000])
def test_bad_tokens_stay_alone(n):
    x, f = numbers(31, 6, n, dtype=BF16), numbers(32, 6, n, dtype=BF16)
    h, y, h2, y2 = (torch.empty_like(x) for _ in range(4))
    B.block_norm(x, f, h, y)
    f[2, n - 1], x[4, 0] = float("nan"), float("inf")
    B.block_norm(x, f, h2, y2)
    good = torch.tensor([0, 1, 3, 5], device="cuda")
    assert torch.equal(h[good], h2[good]) and torch.equal(y[good], y2[good])
    assert bool(h2[2].isnan().all()) and bool(y2[2].isnan().all()) and h2[4, 0] == float("inf") and bool(y2[4, 0].isnan()) and bool((y2[4, 1:] == 0).all())


def test_tokens_of_zeros():
    x = torch.zeros((3, 100), dtype=BF16, device="cuda")
    h, y, r, q = torch.empty_like(x), torch.empty_like(x), torch.empty(3, device="cuda"), torch.empty(3, device="cuda")
    B.block_norm(x, x.clone(), h, y, eps=EPS, rstd_post=q, rstd_pre=r)
    assert not h.any() and not y.any() and torch.allclose(r, torch.full_like(r, EPS ** -0.5)) and torch.equal(r, q)


def test_no_tokens():
    x, v = torch.empty((0, 40), device="cuda"), torch.empty(0, device="cuda")
    B.block_norm(x, x, x, x)
    w, g = torch.ones(40, device="cuda"), [torch.ones(40, device="cuda") for _ in range(3)]
    B.block_norm_backward(x, x, x, v, x, x, rstd_post=v, gate=w, dgate=g[0], dpost_weight=g[1], dpre_weight=g[2])
    assert not any(bool(t.any()) for t in g)


@pytest.mark.parametrize("which", ["dgate", "dpost_weight", "dpre_weight"])
@pytest.mark.parametrize("n", [300, 9000])
def test_sums_that_are_not_wanted(which, n):
    h, f, dy, g = numbers(41, 20, n), numbers(42, 20, n), numbers(43, 20, n), numbers(44, n)
    r, q = torch.ones(20, device="cuda"), torch.ones(20, device="cuda")

    def call(**wanted):
        dx, df = torch.empty_like(h), torch.empty_like(h)
        B.block_norm_backward(dy, h, f, r, dx, df, rstd_post=q, gate=g, **wanted)
        return dx, df
    every = {k: torch.empty(n, device="cuda") for k in ("dgate", "dpost_weight", "dpre_weight")}
    want, one = call(**every), torch.empty(n, device="cuda")
    for got in (call(**{which: one}), call()):
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(one, every[which])


def test_gradients_against_differences():
    """Central differences with a step of 2^-6: off by h^2 / 6 of a third derivative (below 60 here: two norms of vectors of length sqrt(6) in a row) and rounding 2^-19 / h."""
    tokens, n, step = 3, 6, 2.0 ** -6
    x, f, g, a, b = numbers(51, tokens, n) + 1.5, numbers(52, tokens, n) + 1.0, numbers(53, n) * 0.2 + 0.5, numbers(54, n) * 0.2 + 1, numbers(55, n) * 0.2 + 1
    dy, dh = numbers(56, tokens, n), numbers(57, tokens, n)

    def run(x, f, g, a, b):
        h, y, r, q = torch.empty_like(x), torch.empty_like(x), torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda")
        B.block_norm(x, f, h, y, gate=g, post_weight=a, pre_weight=b, scale=0.5, eps=EPS, rstd_post=q, rstd_pre=r)
        return h, y, r, q, float((y.double() * dy.double()).sum() + (h.double() * dh.double()).sum())
    h, _, r, q, _ = run(x, f, g, a, b)
    dx, df, dg, da, db = (torch.empty_like(v) for v in (x, f, g, a, b))
    B.block_norm_backward(dy, h, f, r, dx, df, rstd_post=q, gate=g, post_weight=a, pre_weight=b, scale=0.5, dsum=dh, dgate=dg, dpost_weight=da, dpre_weight=db)
    slack = float(dy.abs().sum() + dh.abs().sum()) * (60 * step * step / 6 + 2.0 ** -19 / step)
    for which, got in enumerate((dx, df, dg, da, db)):
        for at in range(got.numel()):
            both = []
            for sign in (1, -1):
                moved = [v.clone() for v in (x, f, g, a, b)]
                moved[which].view(-1)[at] += sign * step
                both.append(run(*moved)[-1])
            assert abs((both[0] - both[1]) / (2 * step) - float(got.view(-1)[at])) <= slack


@pytest.mark.parametrize("vector", [BF16, F16])
@pytest.mark.parametrize("n", [70, 9000])
def test_types_of_weights_and_gate(vector, n):
    x, f, dy = numbers(61, 5, n, dtype=BF16), numbers(62, 5, n), numbers(63, 5, n)
    g, a, b = numbers(64, n, dtype=vector), numbers(65, n, dtype=vector), numbers(66, n, dtype=vector)
    r = torch.ones(5, device="cuda")

    def run(g, a, b):
        h, y, dx, df = torch.empty_like(x), torch.empty_like(f), torch.empty_like(x), torch.empty_like(f)
        sums = [torch.empty(n, device="cuda") for _ in range(3)]
        B.block_norm(x, f, h, y, gate=g, post_weight=a, pre_weight=b)
        B.block_norm_backward(dy, h, f, r, dx, df, rstd_post=r, gate=g, post_weight=a, pre_weight=b, dgate=sums[0], dpost_weight=sums[1], dpre_weight=sums[2])
        return [h, y, dx, df] + sums
    for got, want in zip(run(g, a, b), run(g.float(), a.float(), b.float())):
        assert torch.equal(got, want)


def test_arguments_are_checked():
    x, f, v, t = numbers(1, 3, 8), numbers(2, 3, 8), numbers(3, 8), numbers(4, 3)
    h, y = torch.empty_like(x), torch.empty_like(x)
    for bad in (lambda: B.block_norm(x, f, h, y, gate=numbers(5, 7)), lambda: B.block_norm(x, f, h, y, gate=numbers(5, 2, 8)), lambda: B.block_norm(x, f[:2], h, y),
                lambda: B.block_norm(x, f, h, y, post_weight=v[:4]), lambda: B.block_norm(x, f, h, y, post=False, post_weight=v), lambda: B.block_norm(x, f, h, y, rstd_pre=v),
                lambda: B.block_norm(x, f, h, y, gate=numbers(5, 3, 8, dtype=BF16)), lambda: B.block_norm(x, f, f, y),
                lambda: B.block_norm_backward(f, x, f, t, h, y, gate=v, dgate=numbers(6, 3, 8)), lambda: B.block_norm_backward(f, x, f, t, h, y, gate=v, dgate=v.to(BF16)),
                lambda: B.block_norm_backward(f, x, f, t, h, y, dpost_weight=v), lambda: B.block_norm_backward(f, x, f, t, x, y)):
        with pytest.raises((ValueError, B.CerError)):
            bad()
