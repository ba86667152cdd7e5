"""Gated products with 4-bit matrices in every cut, where all that is wanted has to be there; and rows that are not finite, in the cuts for more than 16 rows."""
import pytest
import torch

import paper_2603_03383_amd as P
from tests.close import settled
from tests.test_gpu_i4_cuts import COLUMNS, DEV, HALF, ROWS, TD, _matrix

pytestmark = pytest.mark.gpu


def _swiglu(x, gate, up, n, group, zeros):
    rows, k = x.shape
    y = torch.full((rows, n), 7.5, dtype=x.dtype, device=DEV)
    P.medusa_swiglu_i4(x, gate, up, group, zeros, y, torch.empty(P.medusa_swiglu_i4_workspace_bytes(rows, n, k), dtype=torch.uint8, device=DEV))
    return y


def _linear(x, packed, n, group, zeros):
    rows, k = x.shape
    y = torch.full((rows, n), 7.5, device=DEV)
    P.medusa_linear_i4(x, packed, group, zeros, y, torch.empty(P.medusa_linear_i4_workspace_bytes(rows, n, k), dtype=torch.uint8, device=DEV))
    return y


@pytest.mark.parametrize("n", COLUMNS)
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_every_gated_output_is_there(dtype, group, zeros, n):
    """Both sums are exact (small integers times powers of two); the activation has 8 roundings of fp32 at most, its exponential is of an exponent that is
    exact, and the output one."""
    k = 392
    gen = torch.Generator(DEV).manual_seed(n + group)
    (gate, g64), (up, u64) = (_matrix(gen, n, k, group, zeros, dtype) for _ in range(2))
    whole = torch.randint(-4, 5, (max(ROWS), k), device=DEV, generator=gen).to(TD[dtype]) / 64
    g, u = torch.mm(whole.double(), g64.t().contiguous()), torch.mm(whole.double(), u64.t().contiguous())
    want = g * torch.sigmoid(g) * u
    # (2^-25 is half of binary16's smallest step; 2^-100: where exp(-g) leaves fp32's range the factor is zero)
    bound = (HALF[dtype] + 9 * 2.0 ** -24) * want.abs() + 2.0 ** -25 + 2.0 ** -100
    for rows in ROWS:
        ok = settled(_swiglu(whole[:rows].contiguous(), gate, up, n, group, zeros), want[:rows], bound[:rows], dtype)
        assert bool(ok.all()), (rows, int((~ok).sum()))


@pytest.mark.parametrize("rows,n,k", [(20, 16, 8), (20, 40, 261), (64, 8208, 136), (200, 8208, 392), (90, 8208, 261)])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_rows_that_are_not_finite_stay_alone(dtype, group, zeros, rows, n, k):
    gen = torch.Generator(DEV).manual_seed(rows * n + k)
    (gate, g64), (up, u64) = (_matrix(gen, n, k, group, zeros, dtype) for _ in range(2))
    clean = torch.randn(rows, k, device=DEV, generator=gen).to(TD[dtype])
    x = clean.clone()
    bad = {3: (min(17, k - 1), float("nan")), 5: (k - 1, float("inf")), rows - 1: (0, float("-inf"))}
    for r, (at, v) in bad.items():
        x[r, at] = v
    others = torch.tensor([r not in bad for r in range(rows)], device=DEV)
    y, was = _linear(x, gate, n, group, zeros), _linear(clean, gate, n, group, zeros)
    assert torch.equal(y[others], was[others]) and bool(torch.isfinite(was).all())
    z, was = _swiglu(x, gate, up, n, group, zeros), _swiglu(clean / 16, gate, up, n, group, zeros)
    assert torch.equal(_swiglu(torch.where(others[:, None], clean, x), gate, up, n, group, zeros)[others], z[others]) and bool(torch.isfinite(was).all())
    for r, (at, _) in bad.items():
        assert not bool(torch.isfinite(y[r])[g64[:, at] != 0].any())
        assert not bool(torch.isfinite(z[r])[(g64[:, at] != 0) & (u64[:, at] != 0)].any())
