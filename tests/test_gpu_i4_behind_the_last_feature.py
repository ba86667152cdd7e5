"""Products with 4-bit matrices whose features end inside a block of 128, at sizes that go through the LDS ring: nothing stands behind the last feature."""
import numpy as np
import pytest
import torch

from oracle import rows4
from tests.test_gpu_i4_ops import DEV, TD, Matrix, _dev, _np, _rng, _tolerance, linear, swiglu

pytestmark = pytest.mark.gpu

# rows, columns, features: 8 of them in the last block
SHAPES = [(20, 16, 8), (64, 8208, 136), (200, 8208, 392)]
KINDS = [(dtype, group, zeros) for dtype in ("bf16", "fp16") for group in (32, 64, 128) for zeros in (False, True)]


@pytest.mark.parametrize("rows,n,k", SHAPES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
def test_large_values_in_the_last_features(group, zeros, rows, n, k):
    """32 times the sum of a group's |x| is 2.6e38, within fp32's range as the products ask for: 8 features of 1e36, in a group of their own."""
    rng = _rng(rows, n, k, group, 3)
    m = Matrix(rng, n, k, group, zeros, "bf16")
    x = rng.standard_normal((rows, k))
    x[:, -8:] = 1e36 * rng.choice([-1.0, 1.0], (rows, 8))
    x = _dev(x.astype(np.float32), "bf16")
    assert k % group == 8 and 32 * np.abs(_np(x)[:, -8:]).sum(1).max() < 3.4e38
    off = np.abs(_np(linear(x, m, group, n, "fp32")) - rows4.linear(_np(x), m.values))
    assert (off <= _tolerance(_np(x), m, group, k)).all(), off.max()  # (not a number is not within it)


@pytest.mark.parametrize("rows,n,k", SHAPES + [(1024, 4096, 136), (520, 8208, 392)])
@pytest.mark.parametrize("dtype,group,zeros", KINDS)
def test_the_same_from_any_address(dtype, group, zeros, rows, n, k):
    """Rows that start off 16 bytes are copied and padded with zeros; rows that do not need it are to have the same products, bit for bit."""
    rng = _rng(rows, n, k, group, 4)
    gate, up = Matrix(rng, n, k, group, zeros, dtype), Matrix(rng, n, k, group, zeros, dtype)
    x = rng.standard_normal((rows, k))
    x[:, -8:] *= 64
    x = _dev(x.astype(np.float32), dtype)
    assert x.data_ptr() % 16 == 0
    moved = torch.empty(rows * k + 1, dtype=TD[dtype], device=DEV)[1:].view(rows, k).copy_(x)
    assert torch.equal(linear(moved, gate, group, n, "fp32"), linear(x, gate, group, n, "fp32"))
    assert torch.equal(swiglu(moved, gate, up, group, n), swiglu(x, gate, up, group, n))
