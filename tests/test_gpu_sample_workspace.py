"""One workspace, sized once for the largest batch, serves the draws of smaller ones; a batch that splits no rows takes none."""
import pytest
import torch

import paper_2603_03383_amd as P
from tests.test_gpu_sample import DEV, _rows, call

pytestmark = pytest.mark.gpu


def _draw(logits, u, ws):
    rows = logits.shape[0]
    token, prob = torch.empty(rows, dtype=torch.int32, device=DEV), torch.empty(rows, device=DEV)
    top_p = torch.full((1,), 0.9, device=DEV)
    P.medusa_sample(logits, u, token, prob, top_p=top_p, rows_per_setting=max(rows, 1), ws=ws)
    return token.cpu().numpy(), prob.double().cpu().numpy()


def test_a_workspace_for_the_largest_batch_serves_the_others():
    vocab, most = 20000, 300
    logits = _rows(8, most, vocab)
    u = torch.rand(most, generator=torch.Generator().manual_seed(1)).to(DEV)
    ws = torch.full((P.medusa_sample_workspace_bytes(most, vocab),), 0xA5, dtype=torch.uint8, device=DEV)
    for rows in (300, 256, 255, 64, 1):
        token, prob = _draw(logits[:rows], u[:rows].contiguous(), ws)
        want = call(logits[:rows], u[:rows].contiguous(), rows_per_setting=rows, top_p=0.9)
        assert (token == want[0]).all() and (prob == want[1]).all(), rows
    token, prob = _draw(logits[:, :9000], u, ws)
    want = call(logits[:, :9000], u, rows_per_setting=most, top_p=0.9)
    assert (token == want[0]).all() and (prob == want[1]).all()


def test_many_rows_take_no_workspace():
    logits = _rows(9, 300, 20000)
    u = torch.rand(300, generator=torch.Generator().manual_seed(2)).to(DEV)
    token, prob = _draw(logits, u, None)
    want = call(logits, u, rows_per_setting=300, top_p=0.9)
    assert (token == want[0]).all() and (prob == want[1]).all()
