"""Refusals of the 8-bit operators, each by the check that it names (no GPU work: pointers are never followed)."""
import os

import pytest
import torch

import paper_2603_03383_amd as P


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(P.LIB_PATH):
        import __graft_entry__ as g
        g.build()


@pytest.mark.parametrize("codes", [4096, 4097])
@pytest.mark.parametrize("K", [16, 17])
def test_a_product_too_large_for_a_launch_is_refused_before_its_rows_are_aligned(codes, K):
    """Rows that do not start on 16 bytes are copied first; without a GPU that launch would fail with another status."""
    lib, A = P.lib(), 4096
    assert lib.medusa_linear_i8(codes, A, A, 40, 2 ** 30, K, P.MDZ_BF16, A, A, 1 << 60, None) == -3
    assert b"outputs are more than one launch takes" in lib.medusa_last_error()


def _i8(*s):
    return torch.zeros(*s, dtype=torch.int8)


def _bf(*s):
    return torch.zeros(*s, dtype=torch.bfloat16)


@pytest.mark.parametrize("n,k", [(16, 64), (32, 128 + 64), (48, 64), (1, 64), (16, 128)])
def test_a_matrix_packed_for_other_sizes_is_refused(n, k):
    """A packed matrix ends with its scales: with fewer columns than it has, codes would be read as scales."""
    packed = torch.zeros(P.medusa_packed_i8_bytes(32, 64), dtype=torch.uint8)
    with pytest.raises(P.MedusaError) as e:
        P.medusa_linear_i8(_i8(2, k), torch.zeros(2), packed, torch.zeros(2, n), stream=0)
    assert e.value.status == -2 and "packed" in str(e.value)


@pytest.mark.parametrize("n,k", [(32, 64), (17, 64), (32, 1), (32, 128)])
def test_a_matrix_of_the_same_padded_sizes_passes_the_check(n, k):
    packed = torch.zeros(P.medusa_packed_i8_bytes(32, 64), dtype=torch.uint8)
    with pytest.raises(P.MedusaError) as e:
        P.medusa_linear_i8(_i8(2, k), torch.zeros(2), packed, torch.zeros(2, n), stream=0)
    assert e.value.status == -1 and "GPU" in str(e.value)  # what is left to refuse here


def test_sizes_beyond_32_bits_are_refused():
    """The library takes sizes as 32-bit integers; 2^32 + 16 handed on as they are would arrive as 16."""
    big = 2 ** 32 + 16
    for sizes in [(big, 16, 16), (1, big, 16), (1, 16, big)]:
        for query in (P.medusa_linear_i8_workspace_bytes, P.medusa_linear_i8_plan, P.medusa_linear_i8_parts_plan):
            with pytest.raises(P.MedusaError) as e:
                query(*sizes)
            assert e.value.status == -3
    calls = [  # (no row, or no column, of such a size: nothing has to be allocated)
        lambda: P.medusa_quantize_rows_i8(_bf(0, big), _i8(0, big), torch.zeros(0), stream=0),
        lambda: P.medusa_swiglu_i8(_bf(0, big), _i8(0, big // 2), torch.zeros(0), stream=0),
        lambda: P.medusa_residual_rmsnorm_i8(torch.zeros(0, big), None, _bf(1).expand(big), 1e-5, None, _i8(0, big), torch.zeros(0), stream=0),
        lambda: P.medusa_linear_i8(_i8(0, 16), torch.zeros(0), _i8(16), torch.zeros(0, big), stream=0),
    ]
    for k, call in enumerate(calls):
        with pytest.raises(P.MedusaError) as e:
            call()
        assert e.value.status == -3, (k, e.value)
