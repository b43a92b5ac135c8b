"""Operators of a block around projections on streams other than the null one: a call that needs memory brings its workspace there, and is refused before it launches or
allocates anything without one.  On the CPU, with the HIP runtime of tests/fake_hip.cpp in the place of the real one (a process of its own)."""
import json
import os
import subprocess
import sys

import pytest

from paper_1805_10692_amd import binding as B
from test_prepare_errors import HERE, fake  # noqa: F401  (the library of that runtime)

# Every call on the null stream and on another one, without a workspace and with one: the code, the HIP error, the launches' last kernel and the device memory in use.
CHILD = """
import ctypes, json
import torch
import test_block_operators_host as H
from test_operators_host import AT, BF16, COLUMNS, F32, tokens
from paper_1805_10692_amd import binding as B
fake = ctypes.CDLL(None)
fake.fake_hip_launch.restype = ctypes.c_char_p
fake.fake_hip_bytes.restype = ctypes.c_size_t
P, I64, I32, F = H.P, H.I64, H.I32, H.F


def linear(t, n, m, order, stream, work, room):
    x, y = tokens(order=order, ld=t if order else n, at=2 * AT), tokens(order=order, ld=t if order else m, at=3 * AT)
    return B.lib().linear_matmul(P(AT), I64(n), I32(F32), I64(t), I64(n), I64(m), H.ref(x), H.ref(y), None, I32(F32), None, I32(0), None, P(work), I64(room), P(stream))


def linear_back(t, n, m, act, stream, work, room):
    dy, x, pre, dx = (tokens(ld=k, at=at * AT) for k, at in ((m, 2), (n, 3), (m, 4), (n, 5)))
    return B.lib().linear_backward(P(AT), I64(n), I32(F32), I64(t), I64(n), I64(m), H.ref(dy), H.ref(x), I32(act), H.ref(pre), None, H.ref(dx), None, I64(0), None, P(work), I64(room), P(stream))


def block(t, n, order, stream, work, room):
    x, f, h, y = tokens(ld=n), tokens(order=order, ld=t if order else n, at=2 * AT), tokens(ld=n, at=3 * AT), tokens(ld=n, at=4 * AT)
    return B.lib().block_norm(H.ref(x), H.ref(f), H.ref(h), H.ref(y), I64(t), I64(n), None, None, I32(F32), None, I32(F32), None, I32(F32), F(1.0), F(1e-6), I32(1), None, None, P(work),
                              I64(room), P(stream))


def block_back(t, n, sums, stream, work, room):
    dy, h, f, dx, df = (tokens(ld=n, at=k * AT) for k in (1, 2, 3, 4, 5))
    return B.lib().block_norm_backward(H.ref(dy), H.ref(h), H.ref(f), P(AT), P(AT), H.ref(dx), H.ref(df), I64(t), I64(n), None, None, I32(F32), None, I32(F32), None, I32(F32), F(1.0), None,
                                       None, None, None, P(6 * AT if sums else 0), P(work), I64(room), P(stream))


CALLS = {"few tokens": (linear, 4, 64, 2048, 0), "parts": (linear, 130, 4100, 300, 0), "parts, columns": (linear, 130, 4100, 300, COLUMNS), "dz": (linear_back, 300, 64, 64, 4),
         "no dz": (linear_back, 300, 64, 64, 0), "block": (block, 130, 515, 0), "block, columns": (block, 130, 515, COLUMNS), "block's gradient": (block_back, 130, 515, False),
         "block's gradient, sums": (block_back, 130, 515, True), "wide block's gradient": (block_back, 130, 9000, False)}
got = {}
for name, (f, *a) in CALLS.items():
    got[name] = []
    for stream, work in ((0, 0), (AT, 0), (AT, 64 * AT)):
        fake.fake_hip_forget()
        B.lib().cer_trim()
        before = fake.fake_hip_bytes()
        rc = f(*a, stream, work, 1 << 30 if work else 0)
        shape = (ctypes.c_uint * 7)()
        got[name].append([rc, B.lib().cer_last_hip_error() if rc else 0, fake.fake_hip_launch(b"", shape) is not None, fake.fake_hip_bytes() > before])
print(json.dumps(got))
"""


@pytest.fixture(scope="module")
def got(fake):  # noqa: F811
    env = dict(os.environ, LD_PRELOAD=fake, PYTHONPATH=os.pathsep.join((os.path.dirname(HERE), HERE)))
    out = subprocess.run([sys.executable, "-c", CHILD], env=env, capture_output=True, text=True, timeout=600)
    assert out.returncode == 0, out.stderr
    return json.loads(out.stdout.splitlines()[-1])


REFUSED = [B.CER_E_HIP, 801, False, False]  # hipErrorNotSupported; nothing launched, nothing allocated


@pytest.mark.parametrize("name", ["parts", "parts, columns", "dz", "block, columns", "block's gradient, sums", "wide block's gradient"])
def test_a_call_that_needs_memory(got, name):
    null, other, with_workspace = got[name]
    assert null == [0, 0, True, True]  # its temporary is kept for the next call
    assert other == REFUSED
    assert with_workspace == [0, 0, True, False]


@pytest.mark.parametrize("name", ["few tokens", "no dz", "block", "block's gradient"])
def test_a_call_that_needs_none(got, name):
    for k in range(3):
        assert got[name][k] == [0, 0, True, False]
