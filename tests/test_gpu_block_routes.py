"""block_norm_backward of fp32 where a thread of its one launch has two vectors: 4097 to 8192 features.  Tolerances: those of tests/test_gpu_block_norm.py."""
import pytest

from test_gpu_block_norm import BF16, F32, backward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,n", [(1, 4097), (7, 4608), (300, 5000), (513, 5120), (257, 6143), (600, 6144), (2, 6145), (300, 7680)])
@pytest.mark.parametrize("gate", ["none", "features", "tokens"])
def test_backward(tokens, n, gate):
    backward(tokens, n, F32, F32, gate)


@pytest.mark.parametrize("n", [4097, 6144])
@pytest.mark.parametrize("columns", [(True, False), (False, True), (True, True)])
def test_backward_columns(n, columns):
    backward(130, n, F32, F32, columns=columns)
    backward(130, n, BF16, F32, columns=columns)


@pytest.mark.parametrize("n", [4100, 6144])
def test_without_the_norm_behind(n):
    backward(40, n, F32, F32, "features", post=False)
    backward(40, n, F32, F32, "none", post=False, weights=False, through=False)
