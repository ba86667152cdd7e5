"""A product with a 4-bit matrix of one column tile and more rows than the kernel of few columns has places for in its grid (64 x 65535)."""
import numpy as np
import pytest
import torch

import paper_2603_03383_amd as P

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("rows", [64 * 65535, 64 * 65536 + 5])
def test_a_narrow_product_of_millions_of_rows(rows):
    """Integers times a power of two: exact."""
    rng = np.random.default_rng(rows)
    k, n = 3, 2
    codes = rng.integers(0, 16, (n, k), dtype=np.uint8)
    packed = torch.empty(P.medusa_packed_i4_bytes(n, k, 128), dtype=torch.uint8, device=DEV)
    P.medusa_pack_codes_i4(torch.from_numpy(codes).to(DEV), torch.full((n, 1), 0.25, dtype=torch.bfloat16, device=DEV), None, 128, packed, n)
    x = torch.randint(-4, 5, (rows, k), device=DEV, generator=torch.Generator(DEV).manual_seed(1)).to(torch.bfloat16)
    y = torch.full((rows + 3, n), 7.5, device=DEV)
    ws = torch.empty(P.medusa_linear_i4_workspace_bytes(rows, n, k), dtype=torch.uint8, device=DEV)
    P.medusa_linear_i4(x, packed, 128, False, y[:rows], ws)
    w = torch.from_numpy((codes.astype(np.float32) - 8) * 0.25).to(DEV)
    want = sum(x[:, i:i + 1].float() * w[:, i] for i in range(k))
    assert torch.equal(y[:rows], want) and bool((y[rows:] == 7.5).all())
