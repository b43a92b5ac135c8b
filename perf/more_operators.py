"""Operators of a block around projections, as measurable cases: a dense product with its epilogue, the norms on both sides of a block with
its gate and residual scale, dropout.

A case is one of

  linear           z = x W^T + b, y = r + act(z).  `pre`: z is kept for the backward pass
  linear_backward  dz = dy act'(z); gradients of x (added to what other paths send back, where `through`), W and b
  block            u = f / rms(f) * w_post, h = s x + g u, y = h / rms(h) * w_pre for a block's output f and the residual stream x.
                   `gate`: none, one number per feature ("features") or per token and feature ("tokens"); `post`: with the norm behind the block
  block_backward   gradients of x, f, g and both weights; `through`: a gradient of h comes from the residual stream too
  dropout          y = r + keep x / (1 - p), keep from Philox 4x32-10: eight 16-bit numbers per counter, kept where they are not below
                   p 2^16.  Its backward pass is the same call on the gradient, without r

Fields: tokens, n (features in), m (features out), type, columns (fp32 activations feature after feature, as cer_matmul reads and writes
them; in `block` only f, y and their gradients, beside a residual stream of `type` in rows), activation, residual, p.
"""
import functools
import math

import numpy as np
import torch

own = False

_TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
_BYTES = {"float32": 4, "bfloat16": 2, "float16": 2}
_EPS = 1e-6
_LOW = 0xFFFFFFFF


def _linear(op, tokens, n, m, type, activation, residual, columns=False, pre=False):
    """`residual` in a backward case: dx is added to what other paths send back."""
    return {"op": op, "tokens": tokens, "n": n, "m": m, "type": type, "activation": activation, "residual": residual, "columns": columns, "pre": pre}


def _block(op, tokens, n, type, gate, post=True, columns=False, through=True):
    return {"op": op, "tokens": tokens, "n": n, "type": type, "gate": gate, "post": post, "columns": columns, "through": through}


def _dropout(tokens, n, type, p, residual, columns=False):
    return {"op": "dropout", "tokens": tokens, "n": n, "type": type, "p": p, "residual": residual, "columns": columns}


def listed():
    return [
        # one sequence's next token through a gate of a block: the weights have to come from memory, the rest is latency
        {"name": "linear_token", **_linear("linear", 1, 4096, 4096, "bfloat16", "silu", False)},
        # a decode step of 64 sequences through the last layer of a block, added to the residual stream
        {"name": "linear_decode_b64", **_linear("linear", 64, 9216, 4096, "float16", "none", True)},
        # an odd last batch in cer_matmul's order, in 32 bits
        {"name": "linear_columns_f32", **_linear("linear", 999, 2048, 4608, "float32", "relu", False, columns=True)},
        # prompts, or the forward pass of training: z is kept
        {"name": "linear_train", **_linear("linear", 4096, 4096, 9216, "bfloat16", "gelu_tanh", False, pre=True)},
        # its backward pass
        {"name": "linear_backward_train", **_linear("linear_backward", 4096, 4096, 9216, "bfloat16", "gelu_tanh", True)},
        # a small fine-tuning step in 32 bits, odd sizes
        {"name": "linear_backward_f32", **_linear("linear_backward", 257, 1001, 2049, "float32", "gelu", False)},
        # one token between two blocks: latency
        {"name": "block_token", **_block("block", 1, 4096, "bfloat16", "features")},
        # prompts, a gate per feature, everything in 16 bits
        {"name": "block_prompts", **_block("block", 8192, 4096, "bfloat16", "features")},
        # the backward pass of a training step
        {"name": "block_backward_train", **_block("block_backward", 4096, 4608, "bfloat16", "features")},
        # between two compressed projections, whose order is columns; a gate for every token
        {"name": "block_backward_columns", **_block("block_backward", 999, 2304, "float32", "tokens", columns=True)},
        # in front of an adapter of a small batch
        {"name": "dropout_small", **_dropout(99, 4096, "float32", 0.05, False, columns=True)},
        # behind a block in training, added to the residual stream
        {"name": "dropout_train", **_dropout(8192, 4608, "bfloat16", 0.1, True)},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(("linear", "linear", "linear_backward", "block", "block_backward", "dropout"))
        type = rng.choice(("float32", "bfloat16", "float16"))
        tokens, n, m = _log(rng, 1, 8192), _log(rng, 256, 25088), _log(rng, 256, 9216)
        if rng.random() < 0.6:  # sizes of layers are round, or here of the awkward kind
            n, m = -(-n // 640) * 640, -(-m // 640) * 640
        else:
            n, m = n | 1, m | 1
        tokens = tokens | 1 if tokens > 1024 else tokens
        columns = type == "float32" and rng.random() < 0.4
        if op == "dropout":
            case = _dropout(tokens, n, type, round(rng.uniform(0.02, 0.6), 3), rng.random() < 0.5, columns)
        elif op in ("block", "block_backward"):
            case = _block(op, tokens, n, type, rng.choice(("none", "features", "tokens")), rng.random() < 0.8, rng.random() < 0.3, rng.random() < 0.7)
        else:
            if op == "linear" and rng.random() < 0.3:  # a decode step
                tokens = rng.randint(1, 128)
            case = _linear(op, tokens, min(n, 12800), m, type, rng.choice(("none", "relu", "gelu", "gelu_tanh", "silu")), rng.random() < 0.5, columns,
                           op == "linear" and rng.random() < 0.4)
        w = work(case)
        if w["bytes"] <= 4e8 and w["flops"] <= (3e10 if type == "float32" else 3e11):
            return case


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _activations(tokens, n, type, gen, columns=False, scale=1.0):
    """Normal, a few features eight times as large; `columns`: feature after feature in memory, seen as (tokens, n)."""
    x = torch.randn((tokens, n), generator=gen, device="cuda") * scale
    x[:, torch.randint(0, n, (max(1, n // 500),), generator=gen, device="cuda")] *= 8.0
    x = x.to(_TYPES[type])
    return x.t().contiguous().t() if columns else x


def _buffer(tokens, n, type, columns=False):
    return torch.empty((n, tokens), dtype=_TYPES[type], device="cuda").t() if columns else torch.empty((tokens, n), dtype=_TYPES[type], device="cuda")


def prepare(case, seed):
    gen = _generator(seed)
    s = dict(case)
    tokens, n, type, columns = case["tokens"], case["n"], case["type"], case["columns"]
    if case["op"] == "dropout":
        s["x"] = _activations(tokens, n, type, gen, columns)
        s["r"] = _activations(tokens, n, type, gen, columns) if case["residual"] else None
        s["key"] = torch.randint(-(1 << 62), 1 << 62, (2,), generator=gen, device="cuda")  # seed and offset
        s["y"] = _buffer(tokens, n, type, columns)
        return s
    if case["op"] in ("linear", "linear_backward"):
        m = case["m"]
        s["W"] = (torch.randn((m, n), generator=gen, device="cuda") / math.sqrt(n)).to(_TYPES[type])
        s["x"] = _activations(tokens, n, type, gen, columns)
        if case["op"] == "linear":
            s["b"] = 0.3 * torch.randn(m, generator=gen, device="cuda")
            s["r"] = _activations(tokens, m, type, gen, columns) if case["residual"] else None
            s["z"] = _buffer(tokens, m, type, columns) if case["pre"] else None
            s["y"] = _buffer(tokens, m, type, columns)
            return s
        s["dy"] = _activations(tokens, m, type, gen, columns, 0.1)
        s["z"] = _activations(tokens, m, type, gen, columns) if case["activation"] != "none" else None
        s["r"] = _activations(tokens, n, type, gen, columns, 0.1) if case["residual"] else None
        s["dx"] = _buffer(tokens, n, type, columns)
        s["dW"] = torch.empty((m, n), dtype=_TYPES[type], device="cuda")
        s["db"] = torch.empty(m, dtype=torch.float32, device="cuda")
        return s
    branch = "float32" if columns else type
    s["f"] = _activations(tokens, n, branch, gen, columns, 0.5)
    s["w_post"] = 1.0 + 0.1 * torch.randn(n, generator=gen, device="cuda") if case["post"] else None
    s["w_pre"] = 1.0 + 0.1 * torch.randn(n, generator=gen, device="cuda")
    s["g"] = None if case["gate"] == "none" else 0.5 + 0.1 * torch.randn(n, generator=gen, device="cuda") if case["gate"] == "features" else _activations(tokens, n, type, gen)
    s["scale"] = 0.8
    if case["op"] == "block":
        s["x"] = _activations(tokens, n, type, gen)
        s["h"], s["y"] = _buffer(tokens, n, type), _buffer(tokens, n, branch, columns)
        s["rstd_pre"] = torch.empty(tokens, device="cuda")
        s["rstd_post"] = torch.empty(tokens, device="cuda") if case["post"] else None
        return s
    s["h"] = _activations(tokens, n, type, gen)
    s["dy"] = _activations(tokens, n, branch, gen, columns)
    s["dh"] = _activations(tokens, n, type, gen) if case["through"] else None
    s["rstd_pre"] = torch.rsqrt(s["h"].float().square().mean(1) + _EPS)
    s["rstd_post"] = torch.rsqrt(s["f"].float().square().mean(1) + _EPS) if case["post"] else None
    s["dx"], s["df"] = _buffer(tokens, n, type), _buffer(tokens, n, branch, columns)
    s["dg"] = None if s["g"] is None else torch.empty_like(s["g"])
    s["dw_post"] = torch.empty(n, device="cuda") if case["post"] else None
    s["dw_pre"] = torch.empty(n, device="cuda")
    return s


def _act(z, name):
    if name == "none":
        return z
    if name == "relu":
        return z.clamp(min=0.0)
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))


def _act_slope(z, name):
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0.0).float()
    if name == "silu":
        q = 1.0 / (1.0 + torch.exp(-z))
        return q * (1.0 + z * (1.0 - q))
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    t = torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z))
    return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * math.sqrt(2.0 / math.pi) * (1.0 + 3.0 * 0.044715 * z * z)


def _laid(x, s, type):
    return (x.t().contiguous().t() if s["columns"] else x).to(_TYPES[type])


def _plain_linear(s):
    z = s["x"].float() @ s["W"].float().t() + s["b"]
    y = _act(z, s["activation"])
    if s["r"] is not None:
        y = y + s["r"].float()
    got = {"y": _laid(y, s, s["type"])}
    if s["z"] is not None:
        got["z"] = _laid(z, s, s["type"])
    return got


def _plain_linear_backward(s):
    dz = s["dy"].float()
    if s["z"] is not None:
        dz = dz * _act_slope(s["z"].float(), s["activation"])
    dx = dz @ s["W"].float()
    if s["r"] is not None:
        dx = dx + s["r"].float()
    return {"dx": _laid(dx, s, s["type"]), "dW": (dz.t() @ s["x"].float()).to(_TYPES[s["type"]]), "db": dz.sum(0)}


def _plain_block(s):
    f = s["f"].float()
    got, u = {}, f
    if s["post"]:
        got["rstd_post"] = torch.rsqrt(f.square().mean(1) + _EPS)
        u = f * got["rstd_post"][:, None] * s["w_post"]
    h = s["scale"] * s["x"].float() + (u if s["g"] is None else s["g"].float() * u)
    got["rstd_pre"] = torch.rsqrt(h.square().mean(1) + _EPS)
    got["h"] = h.to(s["h"].dtype)
    got["y"] = _laid(h * got["rstd_pre"][:, None] * s["w_pre"], s, "float32" if s["columns"] else s["type"])
    return got


def _plain_block_backward(s):
    f, dy = s["f"].float(), s["dy"].float()
    hat, k = s["h"].float() * s["rstd_pre"][:, None], dy * s["w_pre"]
    d = s["rstd_pre"][:, None] * (k - hat * (k * hat).mean(1, keepdim=True))
    if s["dh"] is not None:
        d = d + s["dh"].float()
    got = {"dx": (s["scale"] * d).to(s["h"].dtype), "dw_pre": (dy * hat).sum(0)}
    u = fhat = f * s["rstd_post"][:, None] if s["post"] else f
    if s["post"]:
        u = fhat * s["w_post"]
    du = d
    if s["g"] is not None:
        dg = d * u
        got["dg"] = dg.sum(0) if s["gate"] == "features" else dg.to(s["g"].dtype)
        du = d * s["g"].float()
    df = du
    if s["post"]:
        got["dw_post"] = (du * fhat).sum(0)
        e = du * s["w_post"]
        df = s["rstd_post"][:, None] * (e - fhat * (e * fhat).mean(1, keepdim=True))
    got["df"] = _laid(df, s, "float32" if s["columns"] else s["type"])
    return got


def _philox_round(words, _):
    a, b, c, d, k, l = words
    p, q = a * 0xD2511F53, c * 0xCD9E8D57  # 64 bits, whose lower and upper halves are right whatever the sign
    return ((q >> 32) & _LOW) ^ b ^ k, q & _LOW, ((p >> 32) & _LOW) ^ d ^ l, p & _LOW, (k + 0x9E3779B9) & _LOW, (l + 0xBB67AE85) & _LOW


def _keep(tokens, n, key, p):
    """(tokens, n) truth values.  Philox 4x32-10 of Salmon, Moraes, Dror and Shaw (2011)."""
    blocks = -(-n // 8)
    at = torch.arange(tokens * blocks, device=key.device)
    seed, offset = key[0], key[1]
    every = torch.zeros_like(at)
    words = functools.reduce(_philox_round, range(10), (at & _LOW, at >> 32, every + (offset & _LOW), every + ((offset >> 32) & _LOW), seed & _LOW, (seed >> 32) & _LOW))
    halves = torch.stack([words[k // 2] >> (16 * (k % 2)) & 0xFFFF for k in range(8)], 1)
    return (halves >= round(p * 65536)).reshape(tokens, blocks * 8)[:, :n]


def _plain_dropout(s):
    dropped = round(s["p"] * 65536)
    y = torch.where(_keep(s["tokens"], s["n"], s["key"], s["p"]), s["x"].float() * (65536 / (65536 - dropped)), torch.zeros((), device="cuda"))
    if s["r"] is not None:
        y = y + s["r"].float()
    return {"y": _laid(y, s, s["type"])}


_PLAIN = {"linear": _plain_linear, "linear_backward": _plain_linear_backward, "block": _plain_block, "block_backward": _plain_block_backward,
          "dropout": _plain_dropout}


def run(state):
    s = state
    if not own:
        return _PLAIN[s["op"]](s)
    from paper_1805_10692_amd import binding as F
    if s["op"] == "linear":
        F.linear_matmul(s["W"], s["x"], s["y"], bias=s["b"], residual=s["r"], activation=s["activation"], pre=s["z"])
        return {"y": s["y"]} if s["z"] is None else {"y": s["y"], "z": s["z"]}
    if s["op"] == "linear_backward":
        F.linear_backward(s["W"], s["dy"], X=s["x"], activation=s["activation"], pre=s["z"], base=s["r"], dX=s["dx"], dW=s["dW"], dbias=s["db"])
        return {"dx": s["dx"], "dW": s["dW"], "db": s["db"]}
    if s["op"] == "block":
        F.block_norm(s["x"], s["f"], s["h"], s["y"], gate=s["g"], post_weight=s["w_post"], pre_weight=s["w_pre"], scale=s["scale"], eps=_EPS, post=s["post"],
                     rstd_post=s["rstd_post"], rstd_pre=s["rstd_pre"])
        got = {"rstd_post": s["rstd_post"]} if s["post"] else {}
        return {**got, "rstd_pre": s["rstd_pre"], "h": s["h"], "y": s["y"]}
    if s["op"] == "block_backward":
        F.block_norm_backward(s["dy"], s["h"], s["f"], s["rstd_pre"], s["dx"], s["df"], rstd_post=s["rstd_post"], gate=s["g"], post_weight=s["w_post"],
                              pre_weight=s["w_pre"], scale=s["scale"], dsum=s["dh"], dgate=s["dg"], dpost_weight=s["dw_post"], dpre_weight=s["dw_pre"])
        got = {"dx": s["dx"], "dw_pre": s["dw_pre"]}
        if s["g"] is not None:
            got["dg"] = s["dg"]
        if s["post"]:
            got["dw_post"] = s["dw_post"]
        return {**got, "df": s["df"]}
    F.dropout_add(s["x"], s["y"], s["key"], s["p"], residual=s["r"])
    return {"y": s["y"]}


def work(case):
    tokens, n, item = case["tokens"], case["n"], _BYTES[case["type"]]
    if case["op"] == "dropout":  # the generator's whole numbers are not counted: a product, a comparison, a sum
        return {"bytes": item * (3.0 if case["residual"] else 2.0) * tokens * n + 16, "flops": 3.0 * tokens * n}
    if case["op"] in ("linear", "linear_backward"):
        m, more = case["m"], 1.0 if case["residual"] else 0.0
        if case["op"] == "linear":
            return {"bytes": item * (tokens * (n + m * (1 + more + (1 if case["pre"] else 0))) + m * n) + 4.0 * m, "flops": 2.0 * tokens * n * m}
        z = 0.0 if case["activation"] == "none" else 1.0
        return {"bytes": item * (tokens * (n * (2 + more) + m * (1 + z)) + 2.0 * m * n) + 4.0 * m, "flops": 4.0 * tokens * n * m}
    branch = 4 if case["columns"] else item
    gate, features = {"none": (0, 0), "features": (0, 1), "tokens": (1, 0)}[case["gate"]]
    if case["op"] == "block":  # x, h and a gate for every token; f and y
        return {"bytes": tokens * n * (item * (2.0 + gate) + 2.0 * branch) + 4.0 * n * (1 + case["post"] + features) + 8.0 * tokens, "flops": 10.0 * tokens * n}
    streams = item * (2.0 + case["through"] + 2 * gate) + 3.0 * branch  # h, dx, dh, the gate and its gradient; dy, f, df
    return {"bytes": tokens * n * streams + 8.0 * n * (1 + case["post"] + features) + 8.0 * tokens, "flops": 25.0 * tokens * n}


def _exact_act(z, name):
    """(act(z), its slope) in 64 bits."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        return torch.where(z > 0, z, 0.0 * z), torch.where(z > 0, 1.0, 0.0).to(z.dtype)
    if name == "silu":
        q = torch.special.expit(z)
        return z * q, q + z * q * torch.special.expit(-z)
    if name == "gelu":
        q = torch.special.ndtr(z)
        return z * q, q + z * torch.exp(-z * z / 2) * (0.5 / math.pi) ** 0.5
    c = (2 / math.pi) ** 0.5
    q = torch.special.expit(2 * c * z * (1 + 0.044715 * z ** 2))  # (1 + tanh a) / 2 = 1 / (1 + exp(-2 a))
    return z * q, q + z * q * (1 - q) * 2 * c * (1 + 0.134145 * z ** 2)


def _exact_keep(tokens, n, key, p):
    """The generator again, on the host, 32-bit words in numpy's unsigned 64-bit numbers."""
    low, wide = np.uint64(_LOW), np.uint64(32)
    seed, offset = (int(v) % (1 << 64) for v in key.tolist())
    blocks = (n + 7) // 8
    x = np.empty((4, tokens * blocks), dtype=np.uint64)
    x[0] = np.arange(tokens * blocks, dtype=np.uint64)
    x[1] = x[0] >> wide
    x[0] &= low
    x[2], x[3] = np.uint64(offset % (1 << 32)), np.uint64(offset >> 32)
    for r in range(10):
        k = [(half + r * w) % (1 << 32) for half, w in ((seed % (1 << 32), 0x9E3779B9), (seed >> 32, 0xBB67AE85))]
        first, second = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = np.stack([(second >> wide) ^ x[1] ^ np.uint64(k[0]), second & low, (first >> wide) ^ x[3] ^ np.uint64(k[1]), first & low])
    numbers = np.ascontiguousarray(x.T).astype("<u4").view("<u2").reshape(tokens, blocks * 8)
    return torch.from_numpy(numbers[:, :n] >= int(np.rint(p * 65536))).cuda()


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "dropout":
        dropped = int(np.rint(case["p"] * 65536))
        y = s["x"].double() * (65536.0 / (65536 - dropped)) * _exact_keep(case["tokens"], case["n"], s["key"], case["p"])
        return {"y": y if s["r"] is None else y + s["r"].double()}
    if case["op"] == "linear":
        z = torch.addmm(s["b"].double(), s["x"].double().contiguous(), s["W"].double().t().contiguous())
        y, _ = _exact_act(z, case["activation"])
        if s["r"] is not None:
            y = y + s["r"].double()
        return {"y": y} if s["z"] is None else {"y": y, "z": z}
    if case["op"] == "linear_backward":
        dz = s["dy"].double().contiguous()
        if s["z"] is not None:
            dz = dz * _exact_act(s["z"].double().contiguous(), case["activation"])[1]
        dx = torch.mm(dz, s["W"].double())
        dW = torch.mm(dz.t().contiguous(), s["x"].double().contiguous())
        return {"dx": dx if s["r"] is None else dx + s["r"].double(), "dW": dW, "db": torch.mv(dz.t().contiguous(), torch.ones_like(dz[:, 0]))}
    n, f = case["n"], s["f"].double()
    gate = torch.ones((), dtype=torch.float64, device="cuda") if s["g"] is None else s["g"].double()
    w_pre, w_post = s["w_pre"].double(), s["w_post"].double() if case["post"] else torch.ones(n, dtype=torch.float64, device="cuda")
    if case["op"] == "block":
        got = {}
        r = torch.ones(case["tokens"], dtype=torch.float64, device="cuda")
        if case["post"]:
            r = got["rstd_post"] = ((f ** 2).sum(1) / n + _EPS) ** -0.5
        h = 0.8 * s["x"].double() + gate * (f * w_post) * r.unsqueeze(1)
        got["rstd_pre"] = ((h ** 2).sum(1) / n + _EPS) ** -0.5
        got["h"] = h
        got["y"] = h * w_pre * got["rstd_pre"].unsqueeze(1)
        return got
    h, dy, r = s["h"].double(), s["dy"].double(), s["rstd_pre"].double()
    along = (dy * w_pre * h).sum(1) * r ** 3 / n
    d = dy * w_pre * r.unsqueeze(1) - h * along.unsqueeze(1)
    if s["dh"] is not None:
        d = d + s["dh"].double()
    got = {"dx": 0.8 * d, "dw_pre": torch.mv((dy * h).t().contiguous(), r)}
    q = s["rstd_post"].double() if case["post"] else torch.ones_like(r)
    if s["g"] is not None:
        each = d * f * w_post * q.unsqueeze(1)
        got["dg"] = each.sum(0) if case["gate"] == "features" else each
    through_gate = d * gate
    df = through_gate
    if case["post"]:
        got["dw_post"] = torch.mv((through_gate * f).t().contiguous(), q)
        across = (through_gate * w_post * f).sum(1) * q ** 3 / n
        df = through_gate * w_post * q.unsqueeze(1) - f * across.unsqueeze(1)
    got["df"] = df
    return got
