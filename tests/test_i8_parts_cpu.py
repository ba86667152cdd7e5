"""Products in parts without a GPU: how many parts the 7B layer's products take, and the refusals of the plan and of the test hook."""
import os

import pytest

import paper_2603_03383_amd as P


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(P.LIB_PATH):
        import __graft_entry__ as g
        g.build()


def test_parts_of_a_7b_layer():
    parts = lambda *s: P.medusa_linear_i8_parts_plan(*s)["k_splits"]  # noqa: E731
    assert parts(64, 4096, 11008) == 4 and parts(256, 4096, 11008) == 3      # down of one tree, of four
    assert parts(64, 4096, 4096) == 1 and parts(90, 4096, 4096) == 4         # O of one tree, of six small ones
    assert parts(1, 4096, 11008) == 1                                        # one row: whole sums
    for shape in [(64, 4096, 11008), (64, 4096, 4096), (90, 4096, 4096)]:    # scratch for either way
        need = P.medusa_linear_i8_parts_plan(*shape)["workspace_bytes"]
        assert need >= P.medusa_linear_i8_workspace_bytes(*shape) and need >= 4 * parts(*shape) * shape[0] * shape[1] * (parts(*shape) > 1)


def test_refusals():
    """Pointers are never followed here: 16-byte aligned numbers stand for buffers."""
    for bad in [(-1, 32, 32), (64, 0, 32), (64, 32, 0), (64, 32, 131072)]:
        with pytest.raises(P.MedusaError):
            P.medusa_linear_i8_parts_plan(*bad)
    A, B, f = 4096, P.MDZ_BF16, P.lib().medusa_test_i8_update_norm
    need = P.medusa_linear_i8_parts_plan(64, 512, 1408)["workspace_bytes"]

    def call(dtype=B, codes=A, M=64, d=512, K=1408, x=A, eps=1e-5, part=A, ws=A, ws_bytes=need):
        return f(dtype, codes, A, A, M, d, K, x, A, eps, A, A, part, ws, ws_bytes, None)
    assert [call(dtype=P.MDZ_FP32), call(codes=None), call(x=None), call(part=None), call(M=0), call(d=33), call(d=16416), call(ws=A + 4)] == [-1] * 8
    assert call(K=131072) == -3
    assert call(ws_bytes=need - 1) == -4 and call(ws=None) == -4
