"""Rows of the norm that hold nothing: the scale is 1 and they stand for zeros, whatever eps is, in every kernel that makes such rows."""
import numpy as np
import pytest
import torch

import paper_2603_03383_amd as P
from oracle import rows8

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def empty(rows, d, dtype=torch.bfloat16):
    return (torch.full((rows, d), 77, dtype=torch.int8, device=DEV), torch.full((rows,), 7.5, device=DEV),
            torch.full((rows, d), 7.5, dtype=dtype, device=DEV))


@pytest.mark.parametrize("eps", [1e-5, 0.0])
@pytest.mark.parametrize("d", [1, 4, 5, 64, 1387, 4096, 16384, 16388, 40001])  # one, two and four pieces per thread, tails, rows read twice
def test_rows_of_zeros(d, eps):
    x = torch.empty(6, d, device=DEV).normal_(generator=torch.Generator(DEV).manual_seed(d)) + 3
    delta = torch.zeros_like(x)
    x[1], x[2] = 0, -0.0
    delta[3] = -x[3]                 # a sum of zeros
    x[4] = 1e-44                     # the maximum over 127 is zero in fp32
    gain = torch.ones(d, dtype=torch.bfloat16, device=DEV)
    for dl in (None, delta):
        codes, scales, values = empty(6, d)
        P.medusa_residual_rmsnorm_i8(x, dl, gain, eps, None, codes, scales, values)
        zero = [1, 2, 4] if dl is None else [1, 2, 3, 4]
        assert scales[zero].tolist() == [1.0] * len(zero)
        assert not bool(codes[zero].any()) and bool((values[zero] == 0).all())
        with np.errstate(divide="ignore"):
            want = rows8.rmsnorm_rows(x.cpu().numpy(), None if dl is None else dl.cpu().numpy(), gain.float().cpu().numpy(), eps)[2]
        assert np.array_equal(want[zero], np.ones(len(zero)))
        # ... and a product of them is zero, not NaN
        if d <= 4096:
            w = torch.full((16, d), 3, dtype=torch.int8, device=DEV)
            packed = torch.empty(P.medusa_packed_i8_bytes(16, d), dtype=torch.uint8, device=DEV)
            P.medusa_pack_codes_i8(w, torch.full((16,), 0.5, device=DEV), packed, 16)
            y = torch.empty(6, 16, device=DEV)
            P.medusa_linear_i8(codes, scales, packed, y, torch.empty(P.medusa_linear_i8_workspace_bytes(6, 16, d), dtype=torch.uint8, device=DEV))
            assert bool((y[zero] == 0).all()) and bool(torch.isfinite(y).all())


@pytest.mark.parametrize("eps", [1e-5, 0.0])
@pytest.mark.parametrize("m,d,k,parts", [(64, 4096, 11008, 4), (64, 512, 1408, 2), (5, 256, 512, 1)])
def test_rows_of_zeros_over_a_products_parts(m, d, k, parts, eps):
    plan = P.medusa_linear_i8_parts_plan(m, d, k)
    assert plan["k_splits"] == parts
    codes, sx = torch.zeros(m, k, dtype=torch.int8, device=DEV), torch.ones(m, device=DEV)
    packed = torch.empty(P.medusa_packed_i8_bytes(d, k), dtype=torch.uint8, device=DEV)
    P.medusa_pack_codes_i8(torch.ones(d, k, dtype=torch.int8, device=DEV), torch.ones(d, device=DEV), packed, d)
    x = torch.zeros(m, d, device=DEV)
    x[2] = 1.0
    out_codes, scales, _ = empty(m, d)
    ws = torch.empty(plan["workspace_bytes"], dtype=torch.uint8, device=DEV)
    P.medusa_test_i8_update_norm(codes, sx, packed, x, torch.ones(d, dtype=torch.bfloat16, device=DEV), eps, out_codes, scales,
                                 torch.empty(m, d, device=DEV), ws)
    zero = [r for r in range(m) if r != 2]
    assert bool((scales[zero] == 1).all()) and not bool(out_codes[zero].any()) and bool((out_codes[2] == 127).all())
