"""The comparison of tests/close.py refuses what a kernel must not return."""
import math

import pytest
import torch

from tests.close import settled


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_what_is_not_finite_is_refused(dtype):
    want = torch.tensor([0.0, 1.0, -3.0, 64000.0, -64000.0], dtype=torch.float64)
    bound = want.abs() * 2.0 ** -8 + 2.0 ** -25
    assert settled(want.clone(), want, bound, dtype).all()
    for bad in (math.nan, math.inf, -math.inf):
        for i in range(want.numel()):
            got = want.clone()
            got[i] = bad
            assert settled(got, want, bound, dtype).tolist() == [j != i for j in range(want.numel())]
    got = want + 1.01 * bound
    assert not settled(got, want, bound, dtype).any()


def test_binary16_may_overflow_where_the_wanted_value_does():
    want = torch.tensor([1e5, -1e5, 65510.0, 1e5, -1e5, 1e5], dtype=torch.float64)
    got = torch.tensor([math.inf, -math.inf, 65504.0, -math.inf, math.inf, math.nan], dtype=torch.float64)
    assert settled(got, want, want.abs() * 2.0 ** -11, "fp16").tolist() == [True, True, True, False, False, False]
    assert not settled(got[:2], want[:2], want[:2].abs() * 2.0 ** -8, "bf16").any()
