"""Operators of a block around projections, on the CPU: declared and exported names, call signatures, and what the C entry points refuse before they launch
anything (nothing here reaches a device: every call is refused, or has nothing to do)."""
import ctypes
import inspect
import os
import re

import pytest
import torch

from paper_1805_10692_amd import binding as B
from test_operators_host import AT, BF16, COLUMNS, F8, F16, F32, ROOT, tokens

I64, I32, F, D, P = ctypes.c_int64, ctypes.c_int32, ctypes.c_float, ctypes.c_double, ctypes.c_void_p


def ref(m):
    return ctypes.byref(m) if m is not None else None


def test_declared_and_exported():
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "cer.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b((?:linear|block|dropout)_[a-z_]+)\s*\(", header))
    assert declared == set(B.BLOCK_EXPORTS)
    for name in declared:
        assert hasattr(B.lib(), name), name


@pytest.mark.parametrize("call,names", [
    (B.linear_matmul, "W X Y bias residual activation pre workspace stream"), (B.linear_backward, "W dY X activation pre base dX dW dbias workspace stream"),
    (B.block_norm, "X F H Y gate post_weight pre_weight scale eps post rstd_post rstd_pre workspace stream"),
    (B.block_norm_backward, "dY H F rstd_pre dX dF rstd_post gate post_weight pre_weight scale dsum dgate dpost_weight dpre_weight workspace stream"),
    (B.dropout_add, "X Y key p residual call stream")])
def test_signatures(call, names):
    assert list(inspect.signature(call).parameters) == names.split()
    with pytest.raises(TypeError, match="required"):
        call(stream=0)
    with pytest.raises(TypeError, match="unexpected"):
        call(nothing=1)
    with pytest.raises(TypeError, match="positional"):
        call(*range(20))


def test_host_tensors_are_refused():
    x, v, k = torch.zeros((2, 4)), torch.zeros(2), torch.zeros(2, dtype=torch.int64)
    for call in (lambda: B.linear_matmul(x, x, x, stream=0), lambda: B.linear_backward(x, x, stream=0), lambda: B.block_norm(x, x, x, x, stream=0),
                 lambda: B.block_norm_backward(x, x, x, v, x, x, stream=0), lambda: B.dropout_add(x, x, k, 0.5, stream=0)):
        with pytest.raises(ValueError, match="device memory"):
            call()


def linear(W=AT, ldw=8, type=F32, n_tokens=4, n=8, m=6, x=tokens(at=2 * AT), y=tokens(at=3 * AT), bias=0, bias_type=F32, r=None, act=0, pre=None, work=0,
           room=0):
    return B.lib().linear_matmul(P(W), I64(ldw), I32(type), I64(n_tokens), I64(n), I64(m), ref(x), ref(y), P(bias), I32(bias_type), ref(r), I32(act), ref(pre), P(work), I64(room), None)


def test_linear_refusals():
    assert linear(n_tokens=0) == B.CER_OK
    columns = {"x": tokens(order=COLUMNS, at=2 * AT), "y": tokens(order=COLUMNS, at=3 * AT)}
    for bad in ({"W": 0}, {"W": AT + 2}, {"ldw": -1}, {"ldw": 1 << 61}, {"type": F8}, {"type": 9}, {"n_tokens": -1}, {"n": 0}, {"m": 0}, {"act": -1}, {"act": 5}, {"x": None}, {"y": None},
                {"type": BF16}, {"x": tokens(BF16, at=2 * AT)}, {"y": tokens(F16, at=3 * AT)}, {"y": tokens(ld=5, at=3 * AT)}, {"y": columns["y"]}, {"x": columns["x"]},
                {**columns, "r": tokens(at=4 * AT)}, {**columns, "y": tokens(order=COLUMNS, ld=3, at=3 * AT)}, {"bias": AT + 2}, {"bias": AT, "bias_type": F8}, {"r": tokens(BF16, at=4 * AT)},
                {"r": tokens(ld=9, at=3 * AT)}, {"pre": tokens(ld=4, at=4 * AT)}, {"pre": tokens(at=3 * AT)}, {"pre": tokens(at=2 * AT)}, {"y": tokens(at=2 * AT)}, {"y": tokens(at=AT)},
                {"pre": tokens(at=AT)}, {"pre": tokens(at=4 * AT), "r": tokens(at=4 * AT)}, {"type": BF16, "x": tokens(BF16, COLUMNS, at=2 * AT), "y": tokens(BF16, COLUMNS, at=3 * AT)}):
        assert linear(**bad) == B.CER_E_INVALID, bad
    for bad in ({"n_tokens": (1 << 24) + 1}, {"n": (1 << 22) + 1}, {"m": (1 << 22) + 1}, {"n_tokens": 1 << 24, "m": (1 << 16) + 1}, {"n": 1 << 21, "m": (1 << 19) + 1}):
        assert linear(**bad) == B.CER_E_TOO_LARGE, bad


def linear_back(W=AT, ldw=8, type=F32, n_tokens=4, n=8, m=6, dy=tokens(at=2 * AT), x=tokens(at=3 * AT), act=0, pre=None, base=None, dx=tokens(at=4 * AT), dw=5 * AT, lddw=8, db=6 * AT, work=0,
                room=0):
    return B.lib().linear_backward(P(W), I64(ldw), I32(type), I64(n_tokens), I64(n), I64(m), ref(dy), ref(x), I32(act), ref(pre), ref(base), ref(dx), P(dw), I64(lddw), P(db), P(work), I64(room),
                                   None)


def test_linear_backward_refusals():
    assert linear_back(n_tokens=0, dw=0, db=0) == B.CER_OK
    for bad in ({"W": 0}, {"type": F8}, {"dy": None}, {"dy": tokens(BF16, at=2 * AT)}, {"x": None}, {"x": tokens(F16, at=3 * AT)}, {"x": tokens(order=COLUMNS, at=3 * AT)}, {"act": 1}, {"act": 7},
                {"act": 2, "pre": tokens(BF16, at=7 * AT)}, {"dx": tokens(BF16, at=4 * AT)}, {"dx": tokens(ld=7, at=4 * AT)}, {"base": tokens(ld=9, at=4 * AT)}, {"base": tokens(F16, at=7 * AT)},
                {"lddw": 7}, {"dw": AT}, {"dw": 5 * AT + 2}, {"db": 6 * AT + 2}, {"dx": tokens(at=2 * AT)}, {"dx": tokens(at=3 * AT)}, {"dx": tokens(at=AT)}, {"dx": tokens(at=5 * AT)},
                {"dw": 3 * AT}, {"db": 2 * AT}, {"act": 1, "pre": tokens(at=4 * AT)}):
        assert linear_back(**bad) == B.CER_E_INVALID, bad
    for bad in ({"n_tokens": (1 << 24) + 1}, {"n": (1 << 22) + 1}):
        assert linear_back(**bad) == B.CER_E_TOO_LARGE, bad


def block(x=tokens(), f=tokens(at=2 * AT), h=tokens(at=3 * AT), y=tokens(at=4 * AT), n_tokens=4, n=8, gate=None, vector=0, gate_type=F32, post_w=0, post_t=F32, pre_w=0, pre_t=F32, scale=1.0,
          eps=1e-6, post=1, rstd_post=0, rstd_pre=0, work=0, room=0):
    return B.lib().block_norm(ref(x), ref(f), ref(h), ref(y), I64(n_tokens), I64(n), ref(gate), P(vector), I32(gate_type), P(post_w), I32(post_t), P(pre_w), I32(pre_t), F(scale), F(eps),
                              I32(post), P(rstd_post), P(rstd_pre), P(work), I64(room), None)


def test_block_refusals():
    assert block(n_tokens=0) == B.CER_OK
    nan, inf = float("nan"), float("inf")
    for bad in ({"x": None}, {"f": None}, {"h": None}, {"y": None}, {"n": 0}, {"n_tokens": -1}, {"eps": -1.0}, {"eps": nan}, {"eps": inf}, {"scale": nan}, {"scale": inf},
                {"x": tokens(order=COLUMNS)}, {"h": tokens(BF16, at=3 * AT)}, {"h": tokens(ld=7, at=3 * AT)}, {"h": tokens(ld=9)}, {"f": tokens(BF16, at=2 * AT)}, {"y": tokens(F16, at=4 * AT)},
                {"y": tokens(F8, at=4 * AT)}, {"y": tokens(order=COLUMNS, ld=3, at=4 * AT)}, {"x": tokens(BF16), "h": tokens(BF16, at=3 * AT), "f": tokens(BF16, COLUMNS, at=2 * AT)},
                {"x": tokens(BF16), "h": tokens(BF16, at=3 * AT), "f": tokens(F16, at=2 * AT)}, {"gate": tokens(BF16, at=5 * AT)}, {"gate": tokens(order=COLUMNS, at=5 * AT)},
                {"gate": tokens(at=5 * AT), "vector": AT}, {"vector": AT, "gate_type": F8}, {"post_w": AT + 1}, {"pre_w": AT, "pre_t": 5}, {"post": 0, "post_w": AT}, {"post": 0, "rstd_post": AT},
                {"h": tokens(at=2 * AT)}, {"h": tokens(at=4 * AT)}, {"y": tokens(ld=9, at=2 * AT)}, {"f": tokens(order=COLUMNS, at=4 * AT), "y": tokens(order=COLUMNS, at=4 * AT)},
                {"y": tokens()}, {"gate": tokens(at=4 * AT)}):
        assert block(**bad) == B.CER_E_INVALID, bad
    for bad in ({"n": 32769}, {"n_tokens": (1 << 28) + 1}, {"n_tokens": 1 << 28, "n": 4097}):
        assert block(**bad) == B.CER_E_TOO_LARGE, bad


def block_back(dy=tokens(), h=tokens(at=2 * AT), f=tokens(at=3 * AT), rstd_pre=AT, rstd_post=AT, dx=tokens(at=4 * AT), df=tokens(at=5 * AT), n_tokens=4, n=8, gate=None, vector=0, gate_type=F32,
               post_w=0, post_t=F32, pre_w=0, pre_t=F32, scale=1.0, dsum=None, dgate=None, dvector=0, dpost=0, dpre=0, work=0, room=0):
    return B.lib().block_norm_backward(ref(dy), ref(h), ref(f), P(rstd_pre), P(rstd_post), ref(dx), ref(df), I64(n_tokens), I64(n), ref(gate), P(vector), I32(gate_type), P(post_w), I32(post_t),
                                       P(pre_w), I32(pre_t), F(scale), ref(dsum), ref(dgate), P(dvector), P(dpost), P(dpre), P(work), I64(room), None)


def test_block_backward_refusals():
    assert block_back(n_tokens=0) == B.CER_OK
    gate = tokens(at=6 * AT)
    for bad in ({"dy": None}, {"h": None}, {"f": None}, {"dx": None}, {"df": None}, {"rstd_pre": 0}, {"rstd_post": 0, "post_w": AT}, {"rstd_post": 0, "dpost": AT}, {"n": 0},
                {"scale": float("inf")}, {"dy": tokens(BF16)}, {"h": tokens(order=COLUMNS, at=2 * AT), "dx": tokens(order=COLUMNS, at=4 * AT)}, {"dx": tokens(BF16, at=4 * AT)},
                {"df": tokens(order=COLUMNS, at=5 * AT)}, {"df": tokens(ld=7, at=5 * AT)}, {"dsum": tokens(F16, at=6 * AT)}, {"gate": gate, "vector": AT}, {"dvector": AT},
                {"dgate": tokens(at=7 * AT)}, {"gate": gate, "dgate": tokens(ld=7, at=7 * AT)}, {"gate": gate, "dgate": gate}, {"dx": tokens(at=2 * AT)}, {"dx": tokens()},
                {"df": tokens(at=3 * AT)}, {"df": tokens(at=4 * AT)}, {"dsum": tokens(at=4 * AT)}, {"vector": AT + 2}):
        assert block_back(**bad) == B.CER_E_INVALID, bad
    assert block_back(n=32769) == B.CER_E_TOO_LARGE


def test_dropout_refusals():
    def call(x=tokens(), r=None, y=tokens(at=2 * AT), n_tokens=4, n=8, key=AT, p=0.1, which=0):
        return B.lib().dropout_add(ref(x), ref(r), ref(y), I64(n_tokens), I64(n), P(key), D(p), I64(which), None)

    assert call(n_tokens=0) == B.CER_OK
    for bad in ({"x": None}, {"y": None}, {"key": 0}, {"key": AT + 4}, {"p": -0.1}, {"p": 1.5}, {"p": float("nan")}, {"n": 0}, {"n_tokens": -1}, {"x": tokens(BF16)}, {"x": tokens(F8), "y": tokens(F8)},
                {"y": tokens(order=COLUMNS, at=2 * AT)}, {"y": tokens(ld=9)}, {"y": tokens(ld=7, at=2 * AT)}, {"r": tokens(F16, at=3 * AT)}, {"r": tokens(ld=9, at=2 * AT)}):
        assert call(**bad) == B.CER_E_INVALID, bad
    for bad in ({"n": (1 << 22) + 1}, {"n_tokens": (1 << 28) + 1}, {"n_tokens": 1 << 28, "n": 4097}):
        assert call(**bad) == B.CER_E_TOO_LARGE, bad


def test_workspaces():
    f32, bf16 = torch.float32, torch.bfloat16
    assert B.linear_workspace_bytes(1, 4096, 4096, bf16) == 0 and B.linear_workspace_bytes(0, 8, 8, f32) == 0
    need = B.linear_workspace_bytes(64, 9216, 4096, bf16)
    assert need > 0 and need % 256 == 0
    x, y = tokens(BF16, ld=9216, at=2 * AT), tokens(BF16, ld=4096, at=3 * AT)
    sizes = dict(type=BF16, n_tokens=64, n=9216, m=4096, ldw=9216, x=x, y=y)
    for work, room in ((AT, need - 1), (AT + 4, need), (AT, 0)):
        assert linear(work=work, room=room, **sizes) == B.CER_E_INVALID
    back = B.linear_workspace_bytes(300, 1000, 2000, f32, backward=True)
    assert back >= 300 * 2000 * 4
    wide = dict(n_tokens=300, n=1000, m=2000, ldw=1000, lddw=1000, dy=tokens(ld=2000, at=2 * AT), x=tokens(ld=1000, at=3 * AT), act=4, pre=tokens(ld=2000, at=7 * AT), dx=tokens(ld=1000, at=4 * AT))
    assert linear_back(work=AT, room=300 * 2000 * 4 - 256, **wide) == B.CER_E_INVALID
    assert B.block_workspace_bytes(100, 64, bf16) == 0 and B.block_workspace_bytes(100, 64, bf16, columns=True) == 2 * 100 * 64 * 4
    assert B.block_workspace_bytes(100, 64, bf16, backward=True) > 0
    assert block(f=tokens(order=COLUMNS, at=2 * AT), work=AT, room=127) == B.CER_E_INVALID
    assert block_back(dpre=AT, work=AT, room=31) == B.CER_E_INVALID
    for bad in (lambda: B.linear_workspace_bytes(-1, 8, 8, f32), lambda: B.linear_workspace_bytes(4, 0, 8, f32), lambda: B.linear_workspace_bytes(4, 8, 8, torch.int32),
                lambda: B.linear_workspace_bytes(4, 8, 8, bf16, columns=True), lambda: B.block_workspace_bytes(4, 0, f32), lambda: B.block_workspace_bytes(4, 40000, f32),
                lambda: B.block_workspace_bytes(4, 8, torch.float8_e4m3fn)):
        with pytest.raises(B.CerError):
            bad()
