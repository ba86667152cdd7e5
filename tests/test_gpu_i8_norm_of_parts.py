"""The residual update of an 8-bit layer whose product leaves its sums in parts for the norm that follows, against the same product and norm as two calls
and against the definition."""
import numpy as np
import pytest
import torch

import paper_2603_03383_amd as P
from oracle import rows8

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TD = {"bf16": torch.bfloat16, "fp16": torch.float16}
EPS = 1e-5

# (parts, (rows, width, features)): whole products and two, three and four parts, each with one, two and four pieces of a row per thread of the norm
CASES = [(1, (5, 256, 512)), (1, (64, 4096, 4096)),
         (2, (33, 32, 1024)), (2, (64, 512, 1408)), (2, (33, 5120, 1024)), (2, (300, 2048, 4096)), (2, (33, 12288, 5001)), (2, (300, 4096, 11008)),
         (2, (65, 16384, 11008)),
         (3, (257, 256, 2000)), (3, (200, 4096, 5001)), (3, (64, 5120, 4096)), (3, (300, 1376, 4096)), (3, (98, 8192, 5001)), (3, (19, 10240, 8192)),
         (4, (17, 256, 11008)), (4, (40, 4096, 4096)), (4, (90, 4096, 4096)), (4, (64, 4096, 11008)), (4, (65, 6144, 4096)), (4, (300, 2048, 11008)),
         (4, (257, 6144, 11008)), (4, (129, 11008, 8192))]


def _np(t):
    return t.detach().float().cpu().numpy()


def make(m, d, k, dtype, seed):
    g = torch.Generator(DEV).manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.empty(*shape, device=DEV).normal_(0.0, std, generator=g)
    codes, w = (normal(r, k, std=40).round().clamp(-127, 127).to(torch.int8) for r in (m, d))
    sx, sw = ((0.5 + torch.rand(r, device=DEV, generator=g)) / 64 for r in (m, d))
    x, gain = normal(m, d, std=3.0), (1 + normal(d, std=0.3)).to(TD[dtype])
    sx[1] = float("nan")           # a row without a scale
    codes[2], x[3] = 0, 0          # a row that gets nothing, and one that had nothing
    packed = torch.empty(P.medusa_packed_i8_bytes(d, k), dtype=torch.uint8, device=DEV)
    P.medusa_pack_codes_i8(w, sw, packed, d)
    return codes, sx, w, sw, packed, x, gain


@pytest.mark.parametrize("parts,shape", CASES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_norm_of_parts_is_the_product_and_the_norm(dtype, parts, shape):
    m, d, k = shape
    plan = P.medusa_linear_i8_parts_plan(m, d, k)
    assert plan["k_splits"] == parts
    codes, sx, w, sw, packed, x0, gain = make(m, d, k, dtype, m + d + k)
    # as two calls
    y = torch.empty(m, d, device=DEV)
    ws = torch.full((P.medusa_linear_i8_workspace_bytes(m, d, k),), 255, dtype=torch.uint8, device=DEV)
    P.medusa_linear_i8(codes, sx, packed, y, ws)
    want_x, want_codes, want_scales = torch.empty_like(x0), torch.empty(m, d, dtype=torch.int8, device=DEV), torch.empty(m, device=DEV)
    P.medusa_residual_rmsnorm_i8(x0, y, gain, EPS, want_x, want_codes, want_scales)
    # as a layer does it: in place, the new row scales over the old ones
    guard = 3
    x_all = torch.full((m + guard, d), 7.5, device=DEV)
    codes_all = torch.full((m + guard, d), 77, dtype=torch.int8, device=DEV)
    scales_all = torch.full((m + guard,), 7.5, device=DEV)
    x_all[:m], scales_all[:m] = x0, sx
    ws = torch.full((plan["workspace_bytes"],), 255, dtype=torch.uint8, device=DEV)
    P.medusa_test_i8_update_norm(codes, scales_all[:m], packed, x_all[:m], gain, EPS, codes_all[:m], scales_all[:m], torch.empty(m, d, device=DEV), ws)
    assert np.array_equal(_np(x_all[:m]), _np(want_x), equal_nan=True)
    assert torch.equal(codes_all[:m], want_codes)
    assert bool((x_all[m:] == 7.5).all()) and bool((codes_all[m:] == 77).all()) and bool((scales_all[m:] == 7.5).all())
    # the definition: exact sums, every rounding of fp32 by itself
    sums = (codes.double() @ w.double().t().contiguous()).cpu().numpy()
    with np.errstate(invalid="ignore"):
        update = sums.astype(np.float32) * (_np(sx)[:, None] * _np(sw)[None, :])
        x_ref, codes_ref, scales_ref = rows8.rmsnorm_rows(_np(x0), update, _np(gain), EPS)
    assert np.array_equal(_np(want_x), x_ref, equal_nan=True)
    assert np.array_equal(want_codes.cpu().numpy(), codes_ref)
    fine = np.isfinite(scales_ref)
    assert not fine[1] and fine.sum() == m - 1
    # d squares, each rounded and summed in chains of at most d / 64 + 16 additions, halved by the root; six more roundings.  (The two norms may differ in
    # that sum's last bits, so scales are each held to the definition.)
    for scales in (want_scales, scales_all[:m]):
        got = _np(scales).astype(np.float64)
        assert np.isnan(got[1]) and (np.abs(got - scales_ref)[fine] <= (d / 128 + 16) * 2.0 ** -24 * scales_ref[fine]).all()
