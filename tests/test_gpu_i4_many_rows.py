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


@pytest.mark.parametrize("gated", [False, True])
def test_outputs_beyond_32_bits_of_offset(gated):
    rng = np.random.default_rng(3)
    rows, n, k = 17000, 128003, 24
    codes = torch.from_numpy(rng.integers(0, 16, (n, k), dtype=np.uint8)).to(DEV)
    packed = torch.empty(P.medusa_packed_i4_bytes(n, k, 32), dtype=torch.uint8, device=DEV)
    P.medusa_pack_codes_i4(codes, torch.full((n, 1), 2.0 ** -6, dtype=torch.bfloat16, device=DEV), None, 32, packed, n)
    x = torch.randint(-4, 5, (rows, k), device=DEV, generator=torch.Generator(DEV).manual_seed(2)).to(torch.bfloat16)
    y = torch.empty(rows, n, dtype=torch.bfloat16, device=DEV)
    assert y.numel() > 2 ** 31
    if gated:
        P.medusa_swiglu_i4(x, packed, packed, 32, False, y, torch.empty(P.medusa_swiglu_i4_workspace_bytes(rows, n, k), dtype=torch.uint8, device=DEV))
    else:
        P.medusa_linear_i4(x, packed, 32, False, y, torch.empty(P.medusa_linear_i4_workspace_bytes(rows, n, k), dtype=torch.uint8, device=DEV))
    w = ((codes.double() - 8) * 2.0 ** -6).t().contiguous()
    for r in (0, 16776, 16777, rows - 1):  # about 2^31 elements in, and the last
        s = torch.mm(x[r:r + 1].double(), w)[0]
        if not gated:
            assert torch.equal(y[r], s.float().to(torch.bfloat16)), r  # (the sums are exact, and rounded once)
        else:
            want = s * torch.sigmoid(s) * s
            # half a step of bf16; the exponent, up to 12 * 1.45, is rounded in fp32, which the exponential makes 12 * 2^-24 of; 8 more roundings at most
            assert bool(((y[r].double() - want).abs() <= (2.0 ** -8 + 20 * 2.0 ** -24) * want.abs()).all()), r
