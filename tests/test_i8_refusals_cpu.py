"""Refusals of the 8-bit operators, each by the check that it names (no GPU work: pointers are never followed)."""
import os

import pytest
import torch

import paper_2603_03383_amd as P
from paper_2603_03383_amd import binding


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


def _f(*s):
    return torch.zeros(*s)


def _packed():
    return torch.zeros(P.medusa_packed_i8_bytes(32, 64), dtype=torch.uint8)


# Calls whose operands are right but for one; they lie in host memory, which is refused last and with another status, so a check that is missing shows.
WRONG = {
    "rows: codes narrower": lambda: P.medusa_quantize_rows_i8(_bf(2, 8), _i8(2, 7), _f(2), stream=0),
    "rows: codes of fp32": lambda: P.medusa_quantize_rows_i8(_bf(2, 8), _f(2, 8), _f(2), stream=0),
    "rows: a scale too many": lambda: P.medusa_quantize_rows_i8(_bf(2, 8), _i8(2, 8), _f(3), stream=0),
    "rows: scales of bf16": lambda: P.medusa_quantize_rows_i8(_bf(2, 8), _i8(2, 8), _bf(2), stream=0),
    "rows: values of another type": lambda: P.medusa_quantize_rows_i8(_bf(2, 8), _i8(2, 8), _f(2), _f(2, 8), stream=0),
    "rows: values of another shape": lambda: P.medusa_quantize_rows_i8(_bf(2, 8), _i8(2, 8), _f(2), _bf(2, 9), stream=0),
    "rows: one axis": lambda: P.medusa_quantize_rows_i8(_bf(8), _i8(8), _f(1), stream=0),
    "rows: float64": lambda: P.medusa_quantize_rows_i8(torch.zeros(2, 8, dtype=torch.float64), _i8(2, 8), _f(2), stream=0),
    "rows: transposed": lambda: P.medusa_quantize_rows_i8(_bf(8, 2).t(), _i8(2, 8), _f(2), stream=0),
    "rows: codes transposed": lambda: P.medusa_quantize_rows_i8(_bf(2, 8), _i8(8, 2).t(), _f(2), stream=0),
    "rows: every other scale": lambda: P.medusa_quantize_rows_i8(_bf(2, 8), _i8(2, 8), _f(4)[::2], stream=0),
    "norm: x of bf16": lambda: P.medusa_residual_rmsnorm_i8(_bf(2, 8), None, _bf(8), 1e-5, None, _i8(2, 8), _f(2), stream=0),
    "norm: delta narrower": lambda: P.medusa_residual_rmsnorm_i8(_f(2, 8), _f(2, 7), _bf(8), 1e-5, None, _i8(2, 8), _f(2), stream=0),
    "norm: delta of a third type": lambda: P.medusa_residual_rmsnorm_i8(_f(2, 8), _f(2, 8).half(), _bf(8), 1e-5, None, _i8(2, 8), _f(2), stream=0),
    "norm: gain shorter": lambda: P.medusa_residual_rmsnorm_i8(_f(2, 8), None, _bf(7), 1e-5, None, _i8(2, 8), _f(2), stream=0),
    "norm: gain of integers": lambda: P.medusa_residual_rmsnorm_i8(_f(2, 8), None, _i8(8), 1e-5, None, _i8(2, 8), _f(2), stream=0),
    "norm: x_out of bf16": lambda: P.medusa_residual_rmsnorm_i8(_f(2, 8), None, _bf(8), 1e-5, _bf(2, 8), _i8(2, 8), _f(2), stream=0),
    "norm: x_out shorter": lambda: P.medusa_residual_rmsnorm_i8(_f(2, 8), None, _bf(8), 1e-5, _f(1, 8), _i8(2, 8), _f(2), stream=0),
    "norm: codes wider": lambda: P.medusa_residual_rmsnorm_i8(_f(2, 8), None, _bf(8), 1e-5, None, _i8(2, 9), _f(2), stream=0),
    "norm: a scale too few": lambda: P.medusa_residual_rmsnorm_i8(_f(2, 8), None, _bf(8), 1e-5, None, _i8(2, 8), _f(1), stream=0),
    "norm: values of fp32": lambda: P.medusa_residual_rmsnorm_i8(_f(2, 8), None, _bf(8), 1e-5, None, _i8(2, 8), _f(2), _f(2, 8), stream=0),
    "swiglu: odd width": lambda: P.medusa_swiglu_i8(_bf(2, 15), _i8(2, 7), _f(2), stream=0),
    "swiglu: codes as wide as gate and up": lambda: P.medusa_swiglu_i8(_bf(2, 16), _i8(2, 16), _f(2), stream=0),
    "swiglu: codes in one axis": lambda: P.medusa_swiglu_i8(_bf(2, 16), _i8(16), _f(2), stream=0),
    "swiglu: scales of fp16": lambda: P.medusa_swiglu_i8(_bf(2, 16), _i8(2, 8), _f(2).half(), stream=0),
    "swiglu: values of another type": lambda: P.medusa_swiglu_i8(_bf(2, 16), _i8(2, 8), _f(2), _f(2, 8), stream=0),
    "product: another number of rows": lambda: P.medusa_linear_i8(_i8(2, 64), _f(2), _packed(), _f(3, 32), stream=0),
    "product: more columns": lambda: P.medusa_linear_i8(_i8(2, 64), _f(2), _packed(), _f(2, 33), stream=0),
    "product: a scale too few": lambda: P.medusa_linear_i8(_i8(2, 64), _f(1), _packed(), _f(2, 32), stream=0),
    "product: codes of fp32": lambda: P.medusa_linear_i8(_f(2, 64), _f(2), _packed(), _f(2, 32), stream=0),
    "product: codes in one axis": lambda: P.medusa_linear_i8(_i8(64), _f(1), _packed(), _f(1, 32), stream=0),
    "product: y of integers": lambda: P.medusa_linear_i8(_i8(2, 64), _f(2), _packed(), _i8(2, 32), stream=0),
    "product: y transposed": lambda: P.medusa_linear_i8(_i8(2, 64), _f(2), _packed(), _f(32, 2).t(), stream=0),
    "product: every other byte of ws": lambda: P.medusa_linear_i8(_i8(2, 64), _f(2), _packed(), _f(2, 32), _i8(64)[::2], stream=0),
    "pack codes: a scale too few": lambda: P.medusa_pack_codes_i8(_i8(32, 64), _f(31), _packed(), 32, stream=0),
    "pack codes: more features": lambda: P.medusa_pack_codes_i8(_i8(32, 129), _f(32), _packed(), 32, stream=0),
    "pack codes: one axis": lambda: P.medusa_pack_codes_i8(_i8(64), _f(1), _packed(), 32, stream=0),
    "pack codes: codes of uint8": lambda: P.medusa_pack_codes_i8(_packed()[:2048].view(32, 64), _f(32), _packed(), 32, stream=0),
    "pack weight: integers": lambda: P.medusa_pack_weight_i8(_i8(32, 64), _packed(), 32, stream=0),
    "pack weight: transposed": lambda: P.medusa_pack_weight_i8(_bf(64, 32).t(), _packed(), 32, stream=0),
}


@pytest.mark.parametrize("what", WRONG)
def test_a_wrong_operand_is_refused_for_itself(what):
    with pytest.raises(P.MedusaError) as e:
        WRONG[what]()
    assert e.value.status == -2


def test_without_the_check_of_operands_these_calls_would_pass(monkeypatch):
    """What the test above relies on: with a check that looks at nothing (and no GPU to ask for), wrong calls end as right ones do here."""
    monkeypatch.setattr(binding, "_operand", lambda name, t, *rest: 4096)
    passed = set()
    for what, call in WRONG.items():
        with pytest.raises(P.MedusaError) as e:
            call()
        if e.value.status == -1:
            passed.add(what)
    kept = {"rows: one axis", "rows: float64", "norm: gain of integers", "product: more columns", "product: codes in one axis", "product: y of integers",
            "pack codes: more features", "pack codes: one axis", "pack weight: integers"}  # refused before their operands are looked at one by one
    assert passed == set(WRONG) - kept


def test_operands_in_host_memory_are_refused():
    for call in [lambda: P.medusa_quantize_rows_i8(_bf(2, 8), _i8(2, 8), _f(2), _bf(2, 8), stream=0),
                 lambda: P.medusa_residual_rmsnorm_i8(_f(2, 8), _f(2, 8), _bf(8), 1e-5, _f(2, 8), _i8(2, 8), _f(2), _bf(2, 8), stream=0),
                 lambda: P.medusa_swiglu_i8(_bf(2, 16), _i8(2, 8), _f(2), _bf(2, 8), stream=0),
                 lambda: P.medusa_linear_i8(_i8(2, 64), _f(2), _packed(), _f(2, 32), _i8(64), stream=0),
                 lambda: P.medusa_pack_codes_i8(_i8(32, 64), _f(32), _packed(), 32, stream=0),
                 lambda: P.medusa_pack_weight_i8(_bf(32, 64), _packed(), 32, stream=0)]:
        with pytest.raises(P.MedusaError) as e:
            call()
        assert e.value.status == -1 and "GPU" in str(e.value)
