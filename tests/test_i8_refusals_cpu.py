"""Refusals of the 8-bit operators, each by the check that it names (no GPU work: pointers are never followed)."""
import os

import pytest

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
