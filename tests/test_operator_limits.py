"""Limits of the operators beside a projection that include/cer.h names, at their edges, on the CPU (every call is refused before anything is launched)."""
import ctypes

import pytest

from paper_1805_10692_amd import binding as B
from test_operators_host import AT, COLUMNS, Gradient, adapters, tokens


def matmul(n_tokens, w, x, y, base=None):
    return B.lib().adapter_matmul(ctypes.byref(w), ctypes.c_void_p(AT), ctypes.c_int64(n_tokens), ctypes.byref(x), None if base is None else ctypes.byref(base), ctypes.byref(y), None, None,
                                  ctypes.c_int64(0), None)


def backward(n_tokens, w, dy, x):
    return B.lib().adapter_backward(ctypes.byref(w), ctypes.c_void_p(AT), ctypes.c_int64(n_tokens), ctypes.byref(dy), ctypes.byref(x), ctypes.c_void_p(AT), None, None, ctypes.c_void_p(AT),
                                    ctypes.c_void_p(AT), None)


@pytest.mark.parametrize("where", ["x", "y", "base"])
def test_columns_further_apart_than_the_most_tokens(where):
    ld = {k: (1 << 24) + (k == where) for k in ("x", "y", "base")}
    x, y, base = (tokens(order=COLUMNS, ld=ld[k], at=i * AT) for i, k in ((1, "x"), (2, "y"), (3, "base")))
    assert matmul(3, adapters(), x, y, base) == B.CER_E_TOO_LARGE


def test_tokens_times_rank():
    w = adapters(rank=128, ld_b=128, stride_a=8 * 128, stride_b=6 * 128)
    assert matmul(1 << 24, w, tokens(), tokens(ld=6, at=4 * AT)) == B.CER_E_TOO_LARGE
    assert backward(1 << 24, w, tokens(ld=6), tokens()) == B.CER_E_TOO_LARGE


def test_gradients_of_all_adapters():
    w = adapters(adapters=1 << 15, rank=1, n=(1 << 18) + 1, ld_a=(1 << 18) + 1, stride_a=(1 << 18) + 1, stride_b=6, ld_b=1)
    assert matmul(3, w, tokens(ld=(1 << 18) + 1), tokens(ld=6, at=4 * AT)) == B.CER_E_TOO_LARGE
    assert matmul(3, adapters(stride_a=(1 << 40) + 1), tokens(), tokens(ld=6, at=4 * AT)) == B.CER_E_TOO_LARGE


def test_numbers_of_a_gradient():
    g = (Gradient * 1)(Gradient(AT, AT, (1 << 48) + 1, 0))
    assert B.lib().grad_clip(g, ctypes.c_int64(1), ctypes.c_float(1.0), ctypes.c_void_p(AT), None) == B.CER_E_TOO_LARGE
