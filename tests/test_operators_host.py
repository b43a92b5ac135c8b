"""Operators beside a projection, on the CPU: declared and exported names, call signatures, and what the C entry points refuse before they launch
anything (nothing here reaches a device: every call is refused, or has nothing to do)."""
import ctypes
import inspect
import os
import re

import pytest
import torch

from paper_1805_10692_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Tokens(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("ld", ctypes.c_int64), ("type", ctypes.c_int32), ("order", ctypes.c_int32)]


class Adapters(ctypes.Structure):
    _fields_ = [(k, ctypes.c_void_p) for k in ("A", "B", "scales", "ranks")] + [
        (k, ctypes.c_int64) for k in ("adapters", "rank", "n", "m", "stride_a", "ld_a", "stride_b", "ld_b")] + [("type", ctypes.c_int32)]


class Gradient(ctypes.Structure):
    _fields_ = [("grad", ctypes.c_void_p), ("out", ctypes.c_void_p), ("numbers", ctypes.c_int64), ("type", ctypes.c_int32)]


F32, BF16, F16, F8 = range(4)
ROWS, COLUMNS = range(2)
AT = 1 << 12  # an address that nothing reads


def test_declared_and_exported():
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "cer.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b((?:rms|adapter|grad)_[a-z_]+)\s*\(", header))
    assert declared == set(B.OPERATOR_EXPORTS)
    for name in declared:
        assert hasattr(B.lib(), name), name


@pytest.mark.parametrize("call,names", [
    (B.rms_norm, "X Y weight residual sum eps scale rstd stream"), (B.rms_norm_backward, "dY H rstd dX weight dsum dweight stream"),
    (B.adapter_matmul, "A B index X Y scales ranks base hidden workspace stream"),
    (B.adapter_backward, "A B index dY X hidden scales ranks base dX dA dB stream"), (B.grad_norm, "grads norm stream"),
    (B.grad_clip, "grads max_norm norm outs stream")])
def test_signatures(call, names):
    assert list(inspect.signature(call).parameters) == names.split()
    with pytest.raises(TypeError, match="required"):
        call(stream=0)
    with pytest.raises(TypeError, match="unexpected"):
        call(nothing=1)
    with pytest.raises(TypeError, match="positional"):
        call(*range(20))


def test_host_tensors_are_refused():
    x, w, i = torch.zeros((2, 4)), torch.zeros((1, 4, 4)), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: B.rms_norm(x, x, stream=0), lambda: B.rms_norm_backward(x, x, x, x, stream=0), lambda: B.adapter_matmul(w, w, i, x, x, stream=0),
                 lambda: B.adapter_backward(w, w, i, x, x, x, stream=0), lambda: B.grad_norm([x], x, stream=0), lambda: B.grad_clip([x], 1.0, x, stream=0)):
        with pytest.raises(ValueError, match="device memory"):
            call()


def tokens(type=F32, order=ROWS, ld=8, at=AT):
    return Tokens(at, ld, type, order)


def test_norm_refusals():
    L = B.lib()

    def call(x=tokens(), r=None, s=None, y=tokens(at=2 * AT), n_tokens=4, n=8, w=0, wt=F32, eps=1e-6, scale=0, rstd=0):
        ref = lambda m: ctypes.byref(m) if m is not None else None  # noqa: E731
        return L.rms_norm(ref(x), ref(r), ref(s), ref(y), ctypes.c_int64(n_tokens), ctypes.c_int64(n), ctypes.c_void_p(w), ctypes.c_int32(wt), ctypes.c_float(eps),
                          ctypes.c_void_p(scale), ctypes.c_void_p(rstd), None)

    assert call(n_tokens=0) == B.CER_OK
    for bad in ({"x": None}, {"y": None}, {"n": 0}, {"n_tokens": -1}, {"eps": -1.0}, {"eps": float("nan")}, {"eps": float("inf")}, {"x": tokens(F8)}, {"x": tokens(7)},
                {"x": tokens(order=2)}, {"x": tokens(BF16, COLUMNS), "y": tokens(F32, COLUMNS)}, {"x": tokens(ld=-8)}, {"y": tokens(ld=7, at=2 * AT)},
                {"y": tokens(order=COLUMNS, ld=3, at=2 * AT)}, {"x": tokens(at=AT + 2)}, {"x": tokens(BF16, at=AT + 1)}, {"r": tokens(BF16)}, {"r": tokens(order=COLUMNS)},
                {"s": tokens(ld=0, at=3 * AT)}, {"s": tokens(ld=9)}, {"y": tokens(F16)}, {"y": tokens(F8)}, {"scale": AT}, {"x": tokens(order=COLUMNS), "y": tokens(F8), "scale": AT},
                {"w": AT, "wt": F8}, {"x": tokens(ld=1 << 62)}):
        assert call(**bad) == B.CER_E_INVALID, bad
    assert call(n=65537, x=tokens(ld=70000), y=tokens(ld=70000)) == B.CER_E_TOO_LARGE
    assert call(n_tokens=(1 << 28) + 1) == B.CER_E_TOO_LARGE


def test_norm_backward_refusals():
    L = B.lib()

    def call(dy=tokens(), h=tokens(at=2 * AT), s=None, dx=tokens(at=3 * AT), n_tokens=4, n=8, rstd=AT, w=0, wt=F32):
        ref = lambda m: ctypes.byref(m) if m is not None else None  # noqa: E731
        return L.rms_norm_backward(ref(dy), ref(h), ref(s), ref(dx), ctypes.c_int64(n_tokens), ctypes.c_int64(n), ctypes.c_void_p(rstd), ctypes.c_void_p(w), ctypes.c_int32(wt),
                                   None, None)

    assert call(n_tokens=0) == B.CER_OK
    for bad in ({"dy": None}, {"h": None}, {"dx": None}, {"rstd": 0}, {"n": 0}, {"dy": tokens(BF16)}, {"dx": tokens(BF16)}, {"s": tokens(F16)}, {"dx": tokens(order=COLUMNS)},
                {"h": tokens(order=COLUMNS), "dx": tokens(order=COLUMNS)}, {"dx": tokens(ld=9)}, {"dx": tokens(ld=4, at=3 * AT)}, {"w": AT, "wt": F8}):
        assert call(**bad) == B.CER_E_INVALID, bad


def adapters(**more):
    f = dict(A=AT, B=2 * AT, scales=0, ranks=0, adapters=2, rank=4, n=8, m=6, stride_a=32, ld_a=8, stride_b=24, ld_b=4, type=F32)
    f.update(more)
    return Adapters(*(f[k] for k, _ in Adapters._fields_))


def test_adapter_refusals():
    L = B.lib()
    ref = lambda m: ctypes.byref(m) if m is not None else None  # noqa: E731

    def call(w=adapters(), index=AT, n_tokens=3, x=tokens(), base=None, y=tokens(ld=6, at=4 * AT), hidden=0, work=0, work_bytes=0):
        return L.adapter_matmul(ref(w), ctypes.c_void_p(index), ctypes.c_int64(n_tokens), ref(x), ref(base), ref(y), ctypes.c_void_p(hidden), ctypes.c_void_p(work),
                                ctypes.c_int64(work_bytes), None)

    def back(w=adapters(), index=AT, n_tokens=3, dy=tokens(ld=6), x=tokens(at=3 * AT), hidden=AT, base=None, dx=tokens(at=4 * AT), dA=AT, dB=AT):
        return L.adapter_backward(ref(w), ctypes.c_void_p(index), ctypes.c_int64(n_tokens), ref(dy), ref(x), ctypes.c_void_p(hidden), ref(base), ref(dx), ctypes.c_void_p(dA),
                                  ctypes.c_void_p(dB), None)

    assert call(n_tokens=0) == B.CER_OK and back(n_tokens=0, dA=0, dB=0) == B.CER_OK
    wrong = [adapters(A=0), adapters(B=0), adapters(adapters=0), adapters(rank=0), adapters(n=0), adapters(m=0), adapters(type=F8), adapters(A=AT + 2), adapters(ld_a=-1),
             adapters(type=BF16, B=AT + 1)]
    for w in [None] + wrong:
        assert call(w=w) == back(w=w) == B.CER_E_INVALID
    for w in (adapters(rank=257), adapters(adapters=65536), adapters(n=(1 << 22) + 1), adapters(m=(1 << 22) + 1), adapters(stride_b=(1 << 40) + 1),
              adapters(adapters=60000, rank=256, n=1 << 20)):
        assert call(w=w) == back(w=w) == B.CER_E_TOO_LARGE
    for bad in ({"index": 0}, {"x": None}, {"y": None}, {"x": tokens(BF16), "y": tokens(BF16, ld=6)}, {"y": tokens(ld=5)}, {"y": tokens(order=COLUMNS, ld=3)}, {"base": tokens(F16)},
                {"base": tokens(ld=7, at=4 * AT)}, {"work": AT, "work_bytes": 8}, {"work": AT + 2, "work_bytes": 1 << 20}, {"n_tokens": -1}):
        assert call(**bad) == B.CER_E_INVALID, bad
    for bad in ({"index": 0}, {"dy": None}, {"x": None}, {"hidden": 0}, {"dx": tokens(BF16)}, {"dx": tokens(order=COLUMNS)}, {"dx": tokens(ld=7)}, {"base": tokens(ld=9, at=4 * AT)},
                {"x": tokens(order=COLUMNS)}, {"n_tokens": -1}):
        assert back(**bad) == B.CER_E_INVALID, bad
    assert call(n_tokens=(1 << 28) + 1) == B.CER_E_TOO_LARGE
    with pytest.raises(B.CerError):
        B.adapter_workspace_bytes(4, 0, 8, 8)
    assert B.adapter_workspace_bytes(0, 4, 8, 8) == 0
    assert B.adapter_workspace_bytes(64, 16, 9216, 4096) % (64 * 16 * 4) == 0


def test_clip_refusals():
    L = B.lib()

    def call(grads, max_norm=1.0, norm=AT):
        a = (Gradient * max(1, len(grads)))(*grads)
        return L.grad_clip(a, ctypes.c_int64(len(grads)), ctypes.c_float(max_norm), ctypes.c_void_p(norm), None)

    good = Gradient(AT, AT, 4, F32)
    for bad in ([Gradient(0, AT, 4, F32)], [good, Gradient(AT, 0, 4, F32)], [Gradient(AT, AT, -1, F32)], [Gradient(AT, AT, 4, F8)], [Gradient(AT + 2, AT, 4, F32)],
                [Gradient(AT, AT + 1, 4, BF16)]):
        assert call(bad) == B.CER_E_INVALID
    for most in (-1.0, float("nan"), float("inf")):
        assert call([good], max_norm=most) == B.CER_E_INVALID
    assert call([good], norm=0) == B.CER_E_INVALID
    assert call([Gradient(AT, AT, 1 << 50, F32)]) == B.CER_E_TOO_LARGE


@pytest.mark.parametrize("where", ["tokens", "ld_a", "ld_b", "x", "y", "base"])
def test_adapter_sizes_past_the_kernels_offsets(where):
    """Offsets inside a tile of 64 tokens have 32 bits, and so has a grid: what could pass them is refused before a launch."""
    L, most = B.lib(), 1 << 22

    def call(n_tokens=3, ld_a=8, ld_b=4, x=8, y=6, base=6):
        X, Y, base = tokens(ld=x), tokens(ld=y, at=4 * AT), tokens(ld=base, at=8 * AT)
        w = adapters(ld_a=ld_a, ld_b=ld_b, stride_a=max(32, 4 * ld_a), stride_b=max(24, 6 * ld_b))
        return L.adapter_matmul(ctypes.byref(w), ctypes.c_void_p(AT), ctypes.c_int64(n_tokens), ctypes.byref(X), ctypes.byref(base), ctypes.byref(Y), None, None, ctypes.c_int64(0), None)

    assert call(**{"n_tokens" if where == "tokens" else where: (1 << 24) + 1 if where == "tokens" else most + 1}) == B.CER_E_TOO_LARGE
