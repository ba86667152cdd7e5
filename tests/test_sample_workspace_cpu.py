"""The size of sampling's workspace: one that serves a call serves every smaller one."""
import os

import pytest

import paper_2603_03383_amd as P


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(P.LIB_PATH):
        import __graft_entry__ as g
        g.build()


ROWS = [0, 1, 2, 15, 64, 128, 255, 256, 257, 300, 1024, 5000]
VOCABS = [1, 500, 8192, 8193, 32003, 128000, 1 << 24]


@pytest.mark.parametrize("vocab", VOCABS)
def test_fewer_rows_need_no_more(vocab):
    """Rows of a large vocabulary are split over workgroups only where there are few, so calls of many rows use none of it."""
    sizes = [P.medusa_sample_workspace_bytes(r, vocab) for r in ROWS]
    assert sizes == sorted(sizes), dict(zip(ROWS, sizes))
    assert sizes[1] > 0 or vocab <= 8192


@pytest.mark.parametrize("rows", ROWS)
def test_a_smaller_vocabulary_needs_no_more(rows):
    sizes = [P.medusa_sample_workspace_bytes(rows, v) for v in VOCABS]
    assert sizes == sorted(sizes), dict(zip(VOCABS, sizes))
