"""Plain 64-bit forms of the operators of a block around projections, for their tests; the dropout's generator in whole numbers."""
import math

import numpy as np
import torch

HALF = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}
SMALLEST = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}  # half of the step below the normal numbers


def act(z, name):
    """(value, slope)"""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        return z.clamp(min=0), (z > 0).double()
    if name == "silu":
        q = torch.sigmoid(z)
        return z * q, q + z * q * torch.sigmoid(-z)
    if name == "gelu":
        q = torch.special.erfc(-z * math.sqrt(0.5)) / 2  # keeps its digits in the lower tail, where 1 + erf loses them
        return z * q, q + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    u = 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
    q = torch.sigmoid(u)
    return z * q, q + z * q * torch.sigmoid(-u) * 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)


def philox(counters, key, rounds=10):
    """Philox 4x32 (Salmon, Moraes, Dror, Shaw 2011) on Python integers: a list of four-word counters, a two-word key."""
    out = []
    for c in counters:
        a, b, d, e = c
        k, l = key
        for _ in range(rounds):
            p, q = a * 0xD2511F53, d * 0xCD9E8D57
            a, b, d, e = (q >> 32) ^ b ^ k, q % 2 ** 32, (p >> 32) ^ e ^ l, p % 2 ** 32
            k, l = (k + 0x9E3779B9) % 2 ** 32, (l + 0xBB67AE85) % 2 ** 32
        out.append((a, b, d, e))
    return out


def numbers16(tokens, n, seed, offset):
    """(tokens, n) 16-bit numbers of dropout_add."""
    blocks = (n + 7) // 8
    seed, offset = seed % 2 ** 64, offset % 2 ** 64
    counters = [(at % 2 ** 32, at >> 32, offset % 2 ** 32, offset >> 32) for at in range(tokens * blocks)]
    words = np.array(philox(counters, (seed % 2 ** 32, seed >> 32)), dtype=np.uint64)
    halves = np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], axis=2)  # lower half first
    return halves.reshape(tokens, blocks * 8)[:, :n].astype(np.int64)


def near(got, want, slack, half):
    """got, of a type with that half step, may be `slack` off before it is rounded."""
    got = got.double()
    ok = (got - want).abs() <= half * want.abs() + (1 + half) * slack
    assert bool(ok.all()), f"{int((~ok).sum())} of {ok.numel()} off, the furthest by {float(((got - want).abs() / (half * want.abs() + (1 + half) * slack + 1e-300)).max()):.3g} times what it may"
