"""Which way block_norm_backward takes and the workspace that it needs for it, on both sides of each border: on the CPU, with the HIP runtime of tests/fake_hip.cpp in the place
of the real one (a process of its own)."""
import json
import os
import subprocess
import sys

import pytest

from paper_1805_10692_amd import binding as B
from test_prepare_errors import HERE, fake  # noqa: F401  (the library of that runtime)

TOKENS = 1000
CHILD = """
import ctypes, json, sys
import test_block_operators_host as H
from test_operators_host import AT, tokens
fake = ctypes.CDLL(None)
fake.fake_hip_launch.restype = ctypes.c_char_p
for type, n in json.load(sys.stdin):
    dy, h, f, dx, df = (tokens(type, ld=n, at=k * AT) for k in (1, 2, 3, 4, 5))
    fake.fake_hip_forget()
    assert H.block_back(dy=dy, h=h, f=f, dx=dx, df=df, n_tokens=1000, n=n, vector=AT, dvector=6 * AT, dpre=7 * AT) == 0
    shape = (ctypes.c_uint * 7)()
    print(json.dumps([fake.fake_hip_launch(k, shape) is not None for k in (b"block_back_rows_kernel", b"block_back_means_kernel", b"block_back_strips_kernel", b"block_back_totals_kernel")]))
"""
F32, BF16, F16 = range(3)
# in one launch, and over that in two, which read the inputs twice
BORDERS = {F32: ([4, 4092, 4096, 4097, 4608, 5000, 5120, 6144, 6145, 8192], [8193, 9000, 32768]), BF16: ([8, 4608, 6144], [6145, 8192, 8193, 32768]), F16: ([6144], [6145])}
WAYS = [(type, n, once) for type, both in BORDERS.items() for once, sizes in zip((True, False), both) for n in sizes]


def test_launches(fake):  # noqa: F811
    env = dict(os.environ, LD_PRELOAD=fake, PYTHONPATH=os.pathsep.join((os.path.dirname(HERE), HERE)))
    out = subprocess.run([sys.executable, "-c", CHILD], input=json.dumps([(type, n) for type, n, _ in WAYS]), env=env, capture_output=True, text=True, timeout=600)
    assert out.returncode == 0, out.stderr
    for (type, n, once), line in zip(WAYS, out.stdout.splitlines(), strict=True):
        assert json.loads(line) == ([True, False, False, True] if once else [False, True, True, True]), (type, n)


@pytest.mark.parametrize("type,n,once", [w for w in WAYS if w[1] > 3000])
def test_workspace(type, n, once):
    """One launch: two sums of 256 workgroups.  Two: those of 63 parts of 16 tokens, and two means a token."""
    rounded = lambda b: -(-b // 256) * 256  # noqa: E731
    want = rounded(2 * 256 * n * 4) if once else rounded(2 * 63 * n * 4) + rounded(TOKENS * 8)
    assert B.block_workspace_bytes(TOKENS, n, {F32: "float32", BF16: "bfloat16", F16: "float16"}[type], backward=True) == want
