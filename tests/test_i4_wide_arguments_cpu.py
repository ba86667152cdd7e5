"""Numbers that do not fit the library's integers: handed on as they are they would arrive as their low bits."""
import os

import pytest
import torch

import paper_2603_03383_amd as P

EUNSUPPORTED = -3
WIDE = 2 ** 32 + 32  # arrives as 32


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(P.LIB_PATH):
        import __graft_entry__ as g
        g.build()


def _bf(*s):
    return torch.zeros(*s, dtype=torch.bfloat16)


def _u8(*s):
    return torch.zeros(*s, dtype=torch.uint8)


def _packed(zeros=False):
    return _u8(P.medusa_packed_i4_bytes(32, 64, 32, zeros))


# (operands in host memory: a call that is not refused for its numbers is refused for that, with another status)
CALLS = {
    "bytes: group": lambda: P.medusa_packed_i4_bytes(32, 64, WIDE),
    "bytes: group below zero": lambda: P.medusa_packed_i4_bytes(32, 64, 32 - 2 ** 32),
    "bytes: zeros": lambda: P.medusa_packed_i4_bytes(32, 64, 32, 2 ** 32),
    "bytes: rows": lambda: P.medusa_packed_i4_bytes(2 ** 64 + 32, 64, 32),
    "bytes: features": lambda: P.medusa_packed_i4_bytes(32, 2 ** 64 + 64, 32),
    # its one scale per row would be read as two
    "pack codes: group": lambda: P.medusa_pack_codes_i4(_u8(32, 64), _bf(32, 1), None, WIDE, _packed(), 32, stream=0),
    "pack codes: group, zero points": lambda: P.medusa_pack_codes_i4(_u8(32, 64), _bf(32, 1), _u8(32, 1), WIDE, _packed(True), 32, stream=0),
    "pack codes: tile": lambda: P.medusa_pack_codes_i4(_u8(32, 64), _bf(32, 2), None, 32, _packed(), 32, 2 ** 64, stream=0),
    "pack: group": lambda: P.medusa_pack_weight_i4(_bf(32, 64), WIDE, _packed(), 32, stream=0),
    "pack: rows": lambda: P.medusa_pack_weight_i4(_bf(32, 64), 32, _packed(), 2 ** 64 + 32, stream=0),
    "pack: tile": lambda: P.medusa_pack_weight_i4(_bf(32, 64), 32, _packed(), 32, 2 ** 64, stream=0),
    "pack: zeros": lambda: P.medusa_pack_weight_i4(_bf(32, 64), 32, _packed(True), 32, zeros=2 ** 32, stream=0),
    "product: group": lambda: P.medusa_linear_i4(_bf(2, 64), _packed(), WIDE, False, _bf(2, 32), stream=0),
    "product: zeros": lambda: P.medusa_linear_i4(_bf(2, 64), _packed(True), 32, 2 ** 32, _bf(2, 32), stream=0),
    "gated product: group": lambda: P.medusa_swiglu_i4(_bf(2, 64), _packed(), _packed(), WIDE, False, _bf(2, 32), stream=0),
}


@pytest.mark.parametrize("what", CALLS)
def test_a_number_that_does_not_fit_is_refused(what):
    with pytest.raises(P.MedusaError) as e:
        CALLS[what]()
    assert e.value.status == EUNSUPPORTED, e.value
