"""Every way in which a product with a 4-bit matrix is cut (by rows, columns, group size, type and zero points), on matrices of many columns."""
import numpy as np
import pytest
import torch

import paper_2603_03383_amd as P

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TD = {"bf16": torch.bfloat16, "fp16": torch.float16}
HALF = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
ROWS = [1, 4, 5, 16, 17, 32, 33, 64, 90, 200, 520]
COLUMNS = [2000, 4112, 8208, 16421]  # 125, 257, 513 and 1027 tiles of 16


def _matrix(gen, n, k, group, zeros, dtype):
    groups = -(-k // group)
    codes = torch.randint(0, 16, (n, k), device=DEV, dtype=torch.uint8, generator=gen)
    scales = torch.pow(2.0, -torch.randint(0, 4, (n, groups), device=DEV, generator=gen).float()).to(TD[dtype])
    points = torch.randint(0, 16, (n, groups), device=DEV, dtype=torch.uint8, generator=gen) if zeros else None
    packed = torch.empty(P.medusa_packed_i4_bytes(n, k, group, zeros), dtype=torch.uint8, device=DEV)
    P.medusa_pack_codes_i4(codes, scales, points, group, packed, n)
    spread = lambda t: t.double().repeat_interleave(group, dim=1)[:, :k]  # noqa: E731
    return packed, (codes.double() - (8.0 if points is None else spread(points))) * spread(scales)


@pytest.mark.parametrize("k", [392, 131])
@pytest.mark.parametrize("n", COLUMNS)
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_products_of_integers(dtype, group, zeros, n, k):
    """Small integers times powers of two: sums are multiples of 1 / 8 below 2^21, which fp32 holds in any order, so a product is exact and the gated
    product is off by its activation alone (exponential, sum, quotient, product: 8 roundings at most) and by its rounding."""
    gen = torch.Generator(DEV).manual_seed(n * k + group)
    (gate, g64), (up, u64) = (_matrix(gen, n, k, group, zeros, dtype) for _ in range(2))
    whole = torch.randint(-4, 5, (max(ROWS), k), device=DEV, generator=gen).to(TD[dtype])
    small = whole / 64  # (the activation is then neither flat nor a step)
    for rows in ROWS:
        x = whole[:rows].contiguous()
        y = torch.full((rows + 3, n), 7.5, device=DEV)
        P.medusa_linear_i4(x, gate, group, zeros, y[:rows], torch.empty(P.medusa_linear_i4_workspace_bytes(rows, n, k), dtype=torch.uint8, device=DEV))
        assert torch.equal(y[:rows].double(), torch.mm(x.double(), g64.t().contiguous())), rows
        assert bool((y[rows:] == 7.5).all())
        x = small[:rows].contiguous()
        z = torch.full((rows + 3, n), 7.5, dtype=TD[dtype], device=DEV)
        P.medusa_swiglu_i4(x, gate, up, group, zeros, z[:rows], torch.empty(P.medusa_swiglu_i4_workspace_bytes(rows, n, k), dtype=torch.uint8, device=DEV))
        g, u = torch.mm(x.double(), g64.t().contiguous()), torch.mm(x.double(), u64.t().contiguous())
        want = g * torch.sigmoid(g) * u
        # (beside the relative errors: where exp(-g) leaves fp32's range the factor is zero, and binary16 has a smallest step)
        bound = (HALF[dtype] + 9 * 2.0 ** -24) * want.abs() + 2.0 ** -25 + 2.0 ** -100
        if dtype == "fp16":
            inside = want.abs() < 65000
            bound = torch.where(inside, bound, torch.full_like(bound, np.inf))
        assert bool(((z[:rows].double() - want).abs() <= bound)[torch.isfinite(z[:rows])].all()), rows
        assert bool((z[rows:] == 7.5).all())
