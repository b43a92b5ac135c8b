"""Operators beside a compressed projection, as measurable cases: the norm in front of it, low-rank adapters next to it, the clipping
of the adapters' gradients.

A case is one of

  norm              h = x + residual, y = h / rms(h) * w.  `out`: the type of y ("float8": e4m3 with a scale per token); `columns`: y
                    in the order in which cer_matmul reads its input (feature after feature)
  norm_backward     gradients of x and w; `through`: a gradient of h comes from the residual stream too
  adapters          y = base + scale_a B_a A_a x for tokens of many requests, each with an adapter of its own or none
  adapters_backward gradients of x, A and B for the same
  clip              the global norm over many gradient tensors, and the gradients scaled down to it

Fields: tokens, n (features in), m (features out), type of the activations, weights (type of the adapters), adapters (in memory),
requests (each a run of tokens with one adapter; every eighth has none), rank, tensors and numbers (of gradients, in total), columns
(activations in cer_matmul's order), limit (the norm to clip to, as a share of the norm that the gradients have).
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16, "float8": torch.float8_e4m3fn}
_BYTES = {"float32": 4, "bfloat16": 2, "float16": 2, "float8": 1}
_LARGEST8 = 448.0
_EPS = 1e-6
_CLIP_EPS = 1e-6


def _norm(tokens, n, type, out, columns=False, residual=True):
    return {"op": "norm", "tokens": tokens, "n": n, "type": type, "out": out, "columns": columns, "residual": residual}


def _norm_backward(tokens, n, type, through=True):
    return {"op": "norm_backward", "tokens": tokens, "n": n, "type": type, "through": through}


def _adapters(op, tokens, n, m, type, weights, adapters, requests, rank, columns):
    return {"op": op, "tokens": tokens, "n": n, "m": m, "type": type, "weights": weights, "adapters": adapters, "requests": requests,
            "rank": rank, "columns": columns}


def _clip(tensors, numbers, type, limit):
    return {"op": "clip", "tensors": tensors, "numbers": numbers, "type": type, "limit": limit}


def listed():
    return [
        # one sequence's next token in front of a layer of 4096 inputs: nothing but the latency of a call
        {"name": "norm_token", **_norm(1, 4096, "float32", "float32")},
        # the odd last batch of an evaluation, from a 16-bit residual stream into the order that cer_matmul reads
        {"name": "norm_columns_b99", **_norm(99, 9216, "bfloat16", "float32", columns=True)},
        # a prompt batch, 8-bit outputs with a scale per token
        {"name": "norm_prompts_8bit", **_norm(8192, 4096, "bfloat16", "float8")},
        # the same layer's backward pass while adapters are trained
        {"name": "norm_backward", **_norm_backward(4096, 4608, "bfloat16")},
        # one request with an adapter beside a middling projection: latency
        {"name": "adapter_token", **_adapters("adapters", 1, 2048, 2048, "float32", "bfloat16", 4, 1, 16, True)},
        # a decode step of 64 requests with 48 adapters beside the AlexNet fc6 shape, in cer_matmul's order
        {"name": "adapters_decode_b64", **_adapters("adapters", 64, 9216, 4096, "float32", "bfloat16", 48, 64, 16, True)},
        # prompts of 16 requests, activations in cer_matmul's order, as many tokens as the convolution has positions
        {"name": "adapters_prompts_columns", **_adapters("adapters", 3136, 4096, 4096, "float32", "bfloat16", 8, 16, 16, True)},
        # prompts of 40 requests in 16 bits, token after token, a large rank
        {"name": "adapters_prompts_rows", **_adapters("adapters", 8192, 4096, 4096, "bfloat16", "bfloat16", 16, 40, 64, False)},
        # a small fine-tuning step in 32 bits, odd number of tokens, a small rank
        {"name": "adapters_backward_f32", **_adapters("adapters_backward", 999, 2048, 4608, "float32", "float32", 4, 6, 8, True)},
        # a large one in 16 bits
        {"name": "adapters_backward_bf16", **_adapters("adapters_backward", 4096, 9216, 4096, "bfloat16", "bfloat16", 8, 24, 32, False)},
        # one projection's two adapter gradients and a few norms' weights
        {"name": "clip_few", **_clip(6, 70_000, "float32", 0.5)},
        # all gradients of a network of some dozen tensors
        {"name": "clip_many", **_clip(56, 48_000_000, "float32", 0.1)},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(("norm", "norm", "norm_backward", "adapters", "adapters", "adapters_backward", "clip"))
        type = rng.choice(("float32", "bfloat16", "float16"))
        tokens, n, m = _log(rng, 1, 8192), _log(rng, 256, 25088), _log(rng, 256, 9216)
        if rng.random() < 0.5:  # sizes of layers are round, or here of the awkward kind
            n, m = -(-n // 640) * 640, -(-m // 640) * 640
        else:
            n, m = n | 1, m | 1
        tokens = tokens | 1 if tokens > 1024 else tokens
        if op == "norm":
            out = rng.choice(("float32", type, "float8"))
            case = _norm(tokens, n, type, out, out == "float32" and rng.random() < 0.6, rng.random() < 0.8)
        elif op == "norm_backward":
            case = _norm_backward(tokens, n, type, rng.random() < 0.7)
        elif op == "clip":
            tensors = rng.randint(1, 62)
            case = _clip(tensors, tensors * _log(rng, 64, 1_000_000), type, round(rng.uniform(0.05, 1.5), 3))
        else:
            if op == "adapters_backward":
                tokens = max(tokens, 16)
            requests = rng.randint(1, max(1, min(tokens, 64)))
            if op == "adapters" and rng.random() < 0.4:  # a decode step: a token for each request
                tokens = requests = rng.randint(1, 256)
            weights = type if type != "float32" else rng.choice(("float32", "bfloat16", "float16"))
            case = _adapters(op, tokens, n, m, type, weights, _log(rng, 1, 64), requests, rng.choice((4, 8, 16, 24, 32, 64, 128)),
                             type == "float32" and rng.random() < 0.6)
        w = work(case)
        if w["bytes"] <= 3.5e8 and w["flops"] <= 8.6e9:
            return case


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _activations(tokens, n, type, gen, columns=False):
    """Normal, a few features sixteen times as large; `columns`: feature after feature in memory, seen as (tokens, n)."""
    x = torch.randn((tokens, n), generator=gen, device="cuda")
    x[:, torch.randint(0, n, (max(1, n // 500),), generator=gen, device="cuda")] *= 16.0
    x = x.to(_TYPES[type])
    return x.t().contiguous().t() if columns else x


def _buffer(tokens, n, type, columns=False):
    return torch.empty((n, tokens), dtype=_TYPES[type], device="cuda").t() if columns else torch.empty((tokens, n), dtype=_TYPES[type], device="cuda")


def _with_adapter(case):
    """(requests with an adapter, adapters that occur)"""
    some = case["requests"] - case["requests"] // 8
    return some, min(some, case["adapters"])


def _index(case, seed):
    """The adapter of each token: requests one after the other, each at least a token long, -1 for every eighth."""
    rng = np.random.RandomState(seed % (1 << 32))
    requests, tokens = case["requests"], case["tokens"]
    share = rng.lognormal(0.0, 0.7, requests)
    ends = np.floor(np.cumsum(share) / share.sum() * (tokens - requests) + 1e-9).astype(np.int64)
    ends[-1] = tokens - requests
    lengths = np.diff(ends, prepend=0) + 1
    some, _ = _with_adapter(case)
    which = np.concatenate([np.arange(some) % case["adapters"], np.full(requests - some, -1)])
    which[:some] = rng.permutation(case["adapters"])[which[:some]]
    return torch.tensor(np.repeat(rng.permutation(which), lengths), dtype=torch.int32, device="cuda")


def _sizes(case):
    """Numbers per gradient tensor: ragged, at least one each, `numbers` in all."""
    tensors, numbers = case["tensors"], case["numbers"]
    rng = np.random.RandomState(numbers % (1 << 32))
    share = rng.lognormal(0.0, 1.0, tensors)
    ends = np.floor(np.cumsum(share) / share.sum() * (numbers - tensors) + 1e-9).astype(np.int64)
    ends[-1] = numbers - tensors
    return (np.diff(ends, prepend=0) + 1).tolist()


def prepare(case, seed):
    gen = _generator(seed)
    state = dict(case)
    if case["op"] == "clip":
        state["grads"] = [torch.randn(k, generator=gen, device="cuda").to(_TYPES[case["type"]]) for k in _sizes(case)]
        state["outs"] = [torch.empty_like(g) for g in state["grads"]]
        state["norm"] = torch.empty(1, dtype=torch.float32, device="cuda")
        state["max_norm"] = case["limit"] * math.sqrt(case["numbers"])
        return state
    tokens, n, type = case["tokens"], case["n"], case["type"]
    if case["op"] == "norm":
        state["x"] = _activations(tokens, n, type, gen)
        state["r"] = _activations(tokens, n, type, gen) if case["residual"] else None
        state["w"] = 1.0 + 0.1 * torch.randn(n, generator=gen, device="cuda")
        state["sum"] = _buffer(tokens, n, type) if case["residual"] else None
        state["y"] = _buffer(tokens, n, case["out"], case["columns"])
        state["s"] = torch.empty(tokens, dtype=torch.float32, device="cuda") if case["out"] == "float8" else None
        state["rstd"] = torch.empty(tokens, dtype=torch.float32, device="cuda")
        return state
    if case["op"] == "norm_backward":
        state["dy"] = _activations(tokens, n, type, gen)
        state["h"] = _activations(tokens, n, type, gen)
        state["dh"] = _activations(tokens, n, type, gen) if case["through"] else None
        state["w"] = 1.0 + 0.1 * torch.randn(n, generator=gen, device="cuda")
        state["rstd"] = torch.rsqrt(state["h"].float().square().mean(1) + _EPS)
        state["dx"] = _buffer(tokens, n, type)
        state["dw"] = torch.empty(n, dtype=torch.float32, device="cuda")
        return state
    m, adapters, rank, weights = case["m"], case["adapters"], case["rank"], _TYPES[case["weights"]]
    state["index"] = _index(case, seed)
    state["A"] = (torch.randn((adapters, rank, n), generator=gen, device="cuda") / math.sqrt(n)).to(weights)
    state["B"] = (torch.randn((adapters, m, rank), generator=gen, device="cuda") / math.sqrt(rank)).to(weights)
    state["scales"] = torch.rand(adapters, generator=gen, device="cuda") + 0.5
    state["x"] = _activations(tokens, n, type, gen, case["columns"])
    if case["op"] == "adapters":
        state["base"] = _activations(tokens, m, type, gen, case["columns"])
        state["y"] = _buffer(tokens, m, type, case["columns"])
        return state
    state["dy"] = _activations(tokens, m, type, gen, case["columns"])
    state["base"] = _activations(tokens, n, type, gen, case["columns"])  # what the projection itself has sent back to x
    state["hidden"] = _hidden(state["A"], state["index"], state["x"])    # the forward pass kept it
    state["dx"] = _buffer(tokens, n, type, case["columns"])
    state["dA"] = torch.empty((adapters, rank, n), dtype=torch.float32, device="cuda")
    state["dB"] = torch.empty((adapters, m, rank), dtype=torch.float32, device="cuda")
    return state


def _membership(index, adapters):
    """(tokens, adapters): 1 where the token has that adapter."""
    return (index[:, None] == torch.arange(adapters, device=index.device)[None, :]).float()


def _hidden(A, index, x):
    """A_a x for every token's own a, 0 without an adapter.  Few tokens: each one's own A; many: all adapters' A at once, the others' products dropped."""
    adapters, rank, n = A.shape
    if index.numel() <= 256:
        return (A[index.clamp(min=0).long()].float() @ x.float()[:, :, None])[:, :, 0] * (index >= 0).float()[:, None]
    every = (x.float() @ A.reshape(-1, n).float().t()).reshape(-1, adapters, rank)
    return (every * _membership(index, adapters)[:, :, None]).sum(1)


def _spread(per_token, index, adapters):
    """(tokens, adapters * rank): each token's numbers at its adapter's place, 0 elsewhere."""
    return (per_token[:, None, :] * _membership(index, adapters)[:, :, None]).reshape(per_token.shape[0], -1)


def _scale_of(scales, index):
    return torch.where(index >= 0, scales[index.clamp(min=0).long()], torch.zeros((), device=scales.device))[:, None]


def _plain_norm(s):
    h = s["x"].float() if s["r"] is None else s["x"].float() + s["r"].float()
    rstd = torch.rsqrt(h.square().mean(1) + _EPS)
    y = h * rstd[:, None] * s["w"]
    got = {"rstd": rstd}
    if s["r"] is not None:
        got["sum"] = h.to(s["x"].dtype)
    if s["out"] == "float8":
        most = y.abs().amax(1)
        got["scale"] = torch.where(most > 0, most / _LARGEST8, torch.ones_like(most))
        got["y"] = (y / got["scale"][:, None]).to(torch.float8_e4m3fn)
    else:
        got["y"] = (y.t().contiguous().t() if s["columns"] else y).to(_TYPES[s["out"]])
    return got


def _plain_norm_backward(s):
    h, dy, rstd = s["h"].float(), s["dy"].float(), s["rstd"][:, None]
    hat, g = h * rstd, dy * s["w"]
    dx = rstd * (g - hat * (g * hat).mean(1, keepdim=True))
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    return {"dx": dx.to(s["dy"].dtype), "dw": (dy * hat).sum(0)}


def _plain_adapters(s):
    adapters, m, rank = s["B"].shape
    hidden = _hidden(s["A"], s["index"], s["x"]) * _scale_of(s["scales"], s["index"])
    if s["index"].numel() <= 256:
        more = (s["B"][s["index"].clamp(min=0).long()].float() @ hidden[:, :, None])[:, :, 0]
    else:
        more = _spread(hidden, s["index"], adapters) @ s["B"].transpose(1, 2).reshape(-1, m).float()
    y = s["base"].float() + more
    return {"y": (y.t().contiguous().t() if s["columns"] else y).to(s["base"].dtype)}


def _plain_adapters_backward(s):
    adapters, m, rank = s["B"].shape
    n, index = s["x"].shape[1], s["index"]
    dy, x = s["dy"].float(), s["x"].float()
    scale = _scale_of(s["scales"], index)
    d = _hidden(s["B"].transpose(1, 2).contiguous(), index, dy) * scale
    wide = _spread(d, index, adapters)
    dx = s["base"].float() + wide @ s["A"].reshape(-1, n).float()
    dA = (wide.t() @ x).reshape(adapters, rank, n)
    dB = (dy.t() @ _spread(s["hidden"] * scale, index, adapters)).reshape(m, adapters, rank).transpose(0, 1).contiguous()
    return {"dx": (dx.t().contiguous().t() if s["columns"] else dx).to(s["x"].dtype), "dA": dA, "dB": dB}


def _plain_clip(s):
    flat = torch.cat([g.reshape(-1) for g in s["grads"]]).float()
    norm = flat.square().sum().sqrt()
    clipped = (flat * (s["max_norm"] / (norm + _CLIP_EPS)).clamp(max=1.0)).to(s["grads"][0].dtype)
    return {"norm": norm.reshape(1), "grads": list(clipped.split([g.numel() for g in s["grads"]]))}


_PLAIN = {"norm": _plain_norm, "norm_backward": _plain_norm_backward, "adapters": _plain_adapters,
          "adapters_backward": _plain_adapters_backward, "clip": _plain_clip}


def run(state):
    s = state
    if not own:
        return _PLAIN[s["op"]](s)
    from paper_1805_10692_amd import binding as F
    if s["op"] == "norm":
        F.rms_norm(s["x"], s["y"], s["w"], residual=s["r"], sum=s["sum"], eps=_EPS, scale=s["s"], rstd=s["rstd"])
        got = {"rstd": s["rstd"], "y": s["y"]}
        if s["r"] is not None:
            got["sum"] = s["sum"]
        if s["s"] is not None:
            got["scale"] = s["s"]
        return got
    if s["op"] == "norm_backward":
        F.rms_norm_backward(s["dy"], s["h"], s["rstd"], s["dx"], s["w"], dsum=s["dh"], dweight=s["dw"])
        return {"dx": s["dx"], "dw": s["dw"]}
    if s["op"] == "adapters":
        F.adapter_matmul(s["A"], s["B"], s["index"], s["x"], s["y"], scales=s["scales"], base=s["base"])
        return {"y": s["y"]}
    if s["op"] == "adapters_backward":
        F.adapter_backward(s["A"], s["B"], s["index"], s["dy"], s["x"], s["hidden"], scales=s["scales"], base=s["base"], dX=s["dx"],
                           dA=s["dA"], dB=s["dB"])
        return {"dx": s["dx"], "dA": s["dA"], "dB": s["dB"]}
    F.grad_clip(s["grads"], s["max_norm"], s["norm"], outs=s["outs"])
    return {"norm": s["norm"], "grads": s["outs"]}


def work(case):
    if case["op"] == "clip":  # the gradients in, the clipped ones out; a square, a sum and a product each
        return {"bytes": 2.0 * _BYTES[case["type"]] * case["numbers"] + 4, "flops": 3.0 * case["numbers"]}
    tokens, n, item = case["tokens"], case["n"], _BYTES[case["type"]]
    if case["op"] == "norm":
        many = item * (3 if case["residual"] else 1) + _BYTES[case["out"]]
        return {"bytes": many * tokens * n + 4.0 * n + (8.0 if case["out"] == "float8" else 4.0) * tokens, "flops": 5.0 * tokens * n}
    if case["op"] == "norm_backward":
        return {"bytes": item * (4 if case["through"] else 3) * tokens * n + 8.0 * n + 4.0 * tokens, "flops": 10.0 * tokens * n}
    m, rank = case["m"], case["rank"]
    some, present = _with_adapter(case)
    busy = tokens * some / case["requests"]  # tokens with an adapter, to expect
    weights = present * rank * (n + m) * _BYTES[case["weights"]]
    if case["op"] == "adapters":  # x of those tokens, base and y of all of them
        return {"bytes": item * (busy * n + 2.0 * tokens * m) + weights + 8.0 * tokens, "flops": 2.0 * busy * rank * (n + m)}
    grads = 4.0 * case["adapters"] * rank * (n + m)
    return {"bytes": item * (busy * (n + m) + 2.0 * tokens * n) + weights + grads + 4.0 * tokens * (rank + 2), "flops": 4.0 * busy * rank * (n + m)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "clip":
        squares = sum(float((g.double() ** 2).sum()) for g in s["grads"])
        norm = math.sqrt(squares)
        c = min(1.0, s["max_norm"] / (norm + _CLIP_EPS))
        return {"norm": torch.tensor([norm], dtype=torch.float64), "grads": [g.double() * c for g in s["grads"]]}
    if case["op"] == "norm":
        h = s["x"].double() + (0.0 if s["r"] is None else s["r"].double())
        rstd = ((h * h).sum(1) / case["n"] + _EPS) ** -0.5
        y = torch.einsum("tn,t,n->tn", h, rstd, s["w"].double())
        got = {"rstd": rstd, "y": y}
        if s["r"] is not None:
            got["sum"] = h
        if case["out"] == "float8":
            got["scale"] = y.abs().max(1).values / _LARGEST8
            got["y"] = y / got["scale"][:, None]
        return got
    if case["op"] == "norm_backward":
        h, dy, rstd, w = s["h"].double(), s["dy"].double(), s["rstd"].double(), s["w"].double()
        along = (dy * w * h).sum(1) * rstd ** 3 / case["n"]
        dx = dy * w * rstd[:, None] - h * along[:, None]
        return {"dx": dx if s["dh"] is None else dx + s["dh"].double(), "dw": torch.mv((dy * h).t().contiguous(), rstd)}
    index, scales = s["index"].cpu(), s["scales"].double()
    base = s["base"].double()
    if case["op"] == "adapters":
        y = base.clone()
        for a in range(case["adapters"]):
            at = torch.nonzero(index == a)[:, 0].cuda()
            if len(at):
                y[at] += scales[a] * ((s["x"][at].double() @ s["A"][a].double().t().contiguous()) @ s["B"][a].double().t().contiguous())
        return {"y": y}
    dx = base.clone()
    dA = torch.zeros((case["adapters"], case["rank"], case["n"]), dtype=torch.float64, device="cuda")
    dB = torch.zeros((case["adapters"], case["m"], case["rank"]), dtype=torch.float64, device="cuda")
    for a in range(case["adapters"]):
        at = torch.nonzero(index == a)[:, 0].cuda()
        if not len(at):
            continue
        dy, x = s["dy"][at].double() * scales[a], s["x"][at].double()
        d = dy @ s["B"][a].double()
        dx[at] += d @ s["A"][a].double()
        dA[a] = d.t().contiguous() @ x
        dB[a] = dy.t().contiguous() @ s["hidden"][at].double()
    return {"dx": dx, "dA": dA, "dB": dB}
