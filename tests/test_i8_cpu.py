"""Rows in 8 bits without a GPU: the oracle's quantiser against the definition, and the refusals of the entry points (status codes,
nothing enqueued)."""
import os

import numpy as np
import pytest
import torch

import paper_2603_03383_amd as P
from oracle import rows8


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(P.LIB_PATH):
        import __graft_entry__ as g
        g.build()


def test_oracle_codes_are_the_nearest_and_ties_go_to_even():
    # max 127 puts the scale at 1, so the row's own halves are ties
    codes, scale = rows8.quantize_rows(np.array([[127, 0.5, 1.5, -2.5, 3.4999, -0.5, 126.5, -126.5]], np.float32))
    assert scale.tolist() == [1.0]
    assert codes.tolist() == [[127, 0, 2, -2, 3, 0, 126, -126]]
    rng = np.random.default_rng(1)
    t = rng.standard_normal((50, 33)).astype(np.float32)
    codes, scale = rows8.quantize_rows(t)
    every = np.arange(-127, 128)
    best = every[np.argmin(np.abs(t[..., None].astype(np.float64) - every * scale[:, None, None].astype(np.float64)), axis=-1)]
    assert np.array_equal(codes, best) and (np.abs(codes).max(axis=1) == 127).all()
    # half a step is the furthest a value can be from its row; the scale and the quotient are rounded (2^-24 each, of up to 127 steps)
    assert (np.abs(rows8.roundtrip_rows(t) - t) <= scale[:, None] * (0.5 + 127 * 2.0 ** -22)).all()


def test_oracle_rows_without_a_scale():
    t = np.array([[0, -0.0, 0], [1, np.nan, 2], [np.inf, 1, 0], [-np.inf, np.nan, 0], [1e-44, 0, -1e-44]], np.float32)
    codes, scale = rows8.quantize_rows(t)
    assert scale[0] == 1 and not codes[0].any()
    assert np.isnan(scale[1:4]).all() and not codes[1:4].any()
    assert scale[4] == 1 and not codes[4].any()  # max / 127 is zero in fp32


def test_packed_bytes():
    assert P.medusa_packed_i8_bytes(4096, 4096) == 4096 * 4096 + 4 * 4096
    assert P.medusa_packed_i8_bytes(17, 129) == 32 * 256 + 4 * 32  # rows padded to 16, features to 128
    for bad in [(0, 16), (16, 0), (-1, 8), (16, 131072), (2 ** 31, 16)]:
        with pytest.raises(P.MedusaError):
            P.medusa_packed_i8_bytes(*bad)
    assert P.medusa_linear_i8_workspace_bytes(0, 5, 7) >= 0
    for bad in [(-1, 16, 16), (1, 0, 16), (1, 16, 0), (1, 16, 131072), (2 ** 30 + 1, 16, 16), (1, 2 ** 30 + 1, 16), (2 ** 25, 2 ** 15, 16)]:
        with pytest.raises(P.MedusaError):
            P.medusa_linear_i8_workspace_bytes(*bad)


def test_refusals_are_status_codes():
    """Pointers are never followed here: 16-byte aligned numbers stand for buffers."""
    lib, A = P.lib(), 4096
    B = P.MDZ_BF16
    rows = [
        lib.medusa_quantize_rows_i8(7, A, 1, 8, A, A, None, None),
        lib.medusa_quantize_rows_i8(B, None, 1, 8, A, A, None, None),
        lib.medusa_quantize_rows_i8(B, A, 1, 8, None, A, None, None),
        lib.medusa_quantize_rows_i8(B, A, 1, 8, A, None, None, None),
        lib.medusa_quantize_rows_i8(B, A, -1, 8, A, A, None, None),
        lib.medusa_quantize_rows_i8(B, A, 1, 0, A, A, None, None),
        lib.medusa_quantize_rows_i8(B, A + 1, 1, 8, A, A, None, None),   # a 16-bit element on an odd address
        lib.medusa_quantize_rows_i8(B, A, 1, 8, A, A + 2, None, None),   # a scale off 4 bytes
        lib.medusa_quantize_rows_i8(B, A, 1, 8, A, A, A + 1, None),
        lib.medusa_swiglu_i8(-1, A, 1, 8, A, A, None, None),
        lib.medusa_swiglu_i8(B, None, 1, 8, A, A, None, None),
        lib.medusa_swiglu_i8(B, A, 1, -8, A, A, None, None),
        lib.medusa_swiglu_i8(B, A, 1, 2 ** 30, A, A, None, None),
        lib.medusa_residual_rmsnorm_i8(B, A, None, 0, None, 1e-5, 1, 8, None, A, A, None, None),
        lib.medusa_residual_rmsnorm_i8(B, None, None, 0, A, 1e-5, 1, 8, None, A, A, None, None),
        lib.medusa_residual_rmsnorm_i8(B, A, A, P.MDZ_FP16, A, 1e-5, 1, 8, None, A, A, None, None),  # neither fp32 nor the gains' type
        lib.medusa_residual_rmsnorm_i8(B, A, A, 9, A, 1e-5, 1, 8, None, A, A, None, None),
        lib.medusa_residual_rmsnorm_i8(B, A, None, 0, A, -1e-5, 1, 8, None, A, A, None, None),
        lib.medusa_residual_rmsnorm_i8(B, A, None, 0, A, float("nan"), 1, 8, None, A, A, None, None),
        lib.medusa_residual_rmsnorm_i8(B, A, None, 0, A, 1e-5, 1, 8, A + 2, A, A, None, None),
        lib.medusa_pack_weight_i8(B, None, 16, 64, A, 16, 0, None),
        lib.medusa_pack_weight_i8(B, A, 16, 64, None, 16, 0, None),
        lib.medusa_pack_weight_i8(5, A, 16, 64, A, 16, 0, None),
        lib.medusa_pack_weight_i8(B, A, 0, 64, A, 16, 0, None),
        lib.medusa_pack_weight_i8(B, A, 16, 64, A + 8, 16, 0, None),     # packed matrices start on 16 bytes
        lib.medusa_pack_codes_i8(A, None, 16, 64, A, 16, 0, None),
        lib.medusa_pack_codes_i8(None, A, 16, 64, A, 16, 0, None),
        lib.medusa_linear_i8(A, A, A, 1, 16, 64, 9, A, None, 0, None),
        lib.medusa_linear_i8(None, A, A, 1, 16, 64, B, A, None, 0, None),
        lib.medusa_linear_i8(A, None, A, 1, 16, 64, B, A, None, 0, None),
        lib.medusa_linear_i8(A, A, None, 1, 16, 64, B, A, None, 0, None),
        lib.medusa_linear_i8(A, A, A, 1, 16, 64, B, None, None, 0, None),
        lib.medusa_linear_i8(A, A, A + 4, 1, 16, 64, B, A, None, 0, None),
        lib.medusa_linear_i8(A, A, A, 1, 16, 64, B, A + 1, None, 0, None),
        lib.medusa_linear_i8(A, A + 2, A, 1, 16, 64, B, A, None, 0, None),
        lib.medusa_linear_i8(A, A, A, 64, 16, 64, B, A, A + 4, 1 << 40, None),
        lib.medusa_linear_i8(A, A, A, -1, 16, 64, B, A, None, 0, None),
    ]
    assert rows == [-1] * len(rows)
    assert lib.medusa_pack_weight_i8(B, A, 20, 64, A, 40, 0, None) == -2   # ends inside a tile, more to come
    assert lib.medusa_pack_weight_i8(B, A, 16, 64, A, 32, 2, None) == -2   # past the end
    assert lib.medusa_pack_weight_i8(B, A, 16, 64, A, 32, 2 ** 62, None) == -2
    assert lib.medusa_pack_weight_i8(B, A, 16, 131072, A, 16, 0, None) == -3
    assert lib.medusa_linear_i8(A, A, A, 1, 16, 131072, B, A, None, 0, None) == -3
    assert b"131071" in lib.medusa_last_error()
    need = P.medusa_linear_i8_workspace_bytes(64, 16, 64)
    assert lib.medusa_linear_i8(A, A, A, 64, 16, 64, B, A, A, need - 1, None) == -4
    assert lib.medusa_linear_i8(A, A, A, 64, 16, 64, B, A, None, need, None) == -4
    # no rows: nothing to do, and nothing is read
    assert lib.medusa_quantize_rows_i8(B, None, 0, 8, None, None, None, None) == 0
    assert lib.medusa_swiglu_i8(B, None, 0, 8, None, None, None, None) == 0
    assert lib.medusa_residual_rmsnorm_i8(B, None, None, 0, None, 1e-5, 0, 8, None, None, None, None, None) == 0
    assert lib.medusa_linear_i8(None, None, None, 0, 16, 64, B, None, None, 0, None) == 0


def test_more_than_a_launch_takes_is_refused():
    """A launch has fewer than 2^32 threads, at least 64 of them per row and 256 per 48 columns (few rows), 1024 outputs (tiles) or packed row."""
    lib, A, B = P.lib(), 4096, P.MDZ_BF16
    assert [
        lib.medusa_quantize_rows_i8(B, A, 2 ** 26, 16, A, A, None, None),
        lib.medusa_swiglu_i8(B, A, 2 ** 30, 16, A, A, None, None),
        lib.medusa_residual_rmsnorm_i8(B, A, None, 0, A, 1e-5, 2 ** 30, 16, None, A, A, None, None),
        lib.medusa_pack_weight_i8(B, A, 2 ** 24, 16, A, 2 ** 24, 0, None),
        lib.medusa_pack_codes_i8(A, A, 2 ** 24, 16, A, 2 ** 24, 0, None),
        lib.medusa_linear_i8(A, A, A, 1, 2 ** 30, 16, B, A, None, 0, None),
        lib.medusa_linear_i8(A, A, A, 2 ** 20, 64, 65537, B, A, A, 1 << 60, None),  # rows that have to be aligned first
        lib.medusa_linear_i8(A, A, A, 40, 2 ** 30, 16, B, A, A, 1 << 60, None),
    ] == [-3] * 8
    assert b"launch" in lib.medusa_last_error()


def test_binding_refuses_shapes_and_types():
    i8 = lambda *s: torch.zeros(*s, dtype=torch.int8)  # noqa: E731
    f = lambda *s: torch.zeros(*s)  # noqa: E731
    h = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    packed = torch.zeros(P.medusa_packed_i8_bytes(32, 64), dtype=torch.uint8)
    bad = [
        lambda: P.medusa_quantize_rows_i8(h(2, 8), i8(2, 7), f(2), stream=0),
        lambda: P.medusa_quantize_rows_i8(h(2, 8), f(2, 8), f(2), stream=0),
        lambda: P.medusa_quantize_rows_i8(h(2, 8), i8(2, 8), f(3), stream=0),
        lambda: P.medusa_quantize_rows_i8(h(2, 8), i8(2, 8), h(2), stream=0),
        lambda: P.medusa_quantize_rows_i8(h(2, 8), i8(2, 8), f(2), f(2, 8), stream=0),
        lambda: P.medusa_quantize_rows_i8(h(8), i8(8), f(1), stream=0),
        lambda: P.medusa_quantize_rows_i8(torch.zeros(2, 8, dtype=torch.float64), i8(2, 8), f(2), stream=0),
        lambda: P.medusa_quantize_rows_i8(h(8, 2).t(), i8(2, 8), f(2), stream=0),
        lambda: P.medusa_residual_rmsnorm_i8(h(2, 8), None, h(8), 1e-5, None, i8(2, 8), f(2), stream=0),
        lambda: P.medusa_residual_rmsnorm_i8(f(2, 8), f(2, 7), h(8), 1e-5, None, i8(2, 8), f(2), stream=0),
        lambda: P.medusa_residual_rmsnorm_i8(f(2, 8), f(2, 8).half(), h(8), 1e-5, None, i8(2, 8), f(2), stream=0),
        lambda: P.medusa_residual_rmsnorm_i8(f(2, 8), None, h(7), 1e-5, None, i8(2, 8), f(2), stream=0),
        lambda: P.medusa_residual_rmsnorm_i8(f(2, 8), None, h(8), 1e-5, h(2, 8), i8(2, 8), f(2), stream=0),
        lambda: P.medusa_swiglu_i8(h(2, 15), i8(2, 8), f(2), stream=0),
        lambda: P.medusa_swiglu_i8(h(2, 16), i8(16), f(2), stream=0),
        lambda: P.medusa_linear_i8(i8(2, 64), f(2), packed, f(3, 32), stream=0),
        lambda: P.medusa_linear_i8(i8(2, 64), f(2), packed, f(2, 33), stream=0),       # more columns than the packed bytes hold
        lambda: P.medusa_linear_i8(i8(2, 64), f(1), packed, f(2, 32), stream=0),
        lambda: P.medusa_linear_i8(f(2, 64), f(2), packed, f(2, 32), stream=0),
        lambda: P.medusa_linear_i8(i8(2, 64), f(2), packed, i8(2, 32), stream=0),
        lambda: P.medusa_pack_codes_i8(i8(32, 64), f(31), packed, 32, stream=0),
        lambda: P.medusa_pack_codes_i8(i8(32, 129), f(32), packed, 32, stream=0),
        lambda: P.medusa_pack_codes_i8(i8(64), f(1), packed, 32, stream=0),
        lambda: P.medusa_pack_weight_i8(i8(32, 64), packed, 32, stream=0),
        # right in shape and type, but not on a GPU
        lambda: P.medusa_quantize_rows_i8(h(2, 8), i8(2, 8), f(2), stream=0),
        lambda: P.medusa_linear_i8(i8(2, 64), f(2), packed, f(2, 32), stream=0),
    ]
    for k, call in enumerate(bad):
        try:
            call()
        except P.MedusaError as e:
            assert e.status in (-1, -2), (k, e)
        else:
            pytest.fail(f"call {k} was not refused")


def test_model_option():
    ok = P.ModelDesc(256, 4, 64, 704, 1024, 2, P.MDZ_BF16, P.MDZ_TREE_15, 1e-5, 1e4, 0, 0, 1)
    plain = P.ModelDesc(256, 4, 64, 704, 1024, 2, P.MDZ_BF16, P.MDZ_TREE_15, 1e-5, 1e4)
    assert P.medusa_workspace_bytes(ok, 1, 64) > 0 and plain.weights_i8 == 0
    for dtype, f16, i8 in [(P.MDZ_FP32, 0, 1), (P.MDZ_BF16, 1, 1), (P.MDZ_FP16, 0, 2), (P.MDZ_BF16, 0, -1)]:
        with pytest.raises(P.MedusaError) as e:
            P.medusa_workspace_bytes(P.ModelDesc(256, 4, 64, 704, 1024, 2, dtype, P.MDZ_TREE_15, 1e-5, 1e4, 0, f16, i8), 1, 64)
        assert e.value.status == -1
    with pytest.raises(P.MedusaError) as e:  # sums over so many features could overflow
        P.medusa_workspace_bytes(P.ModelDesc(256, 4, 64, 131072, 1024, 2, P.MDZ_BF16, P.MDZ_TREE_15, 1e-5, 1e4, 0, 0, 1), 1, 64)
    assert e.value.status == -3
