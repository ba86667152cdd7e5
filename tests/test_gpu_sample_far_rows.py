"""Sampling where rows lie more than 2^31 elements from the first, split and whole."""
import numpy as np
import pytest
import torch

import paper_2603_03383_amd as P
from oracle import sampling

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BORDER = 2e-8  # of the kept mass, by which sums may be off (see test_gpu_sample.py)


@pytest.mark.parametrize("vocab", [1003, 20001])
def test_rows_far_from_the_first(vocab):
    rows, ld = 18, 2 ** 27 + 1
    room = torch.empty(rows * ld, dtype=torch.bfloat16, device=DEV)
    logits = room.view(rows, ld)[:, :vocab]
    g = torch.Generator(DEV).manual_seed(vocab)
    logits.copy_(torch.empty(rows, vocab, device=DEV).normal_(0, 3, generator=g))
    u = torch.rand(rows, generator=torch.Generator().manual_seed(3)).to(DEV)
    token, prob = torch.empty(rows, dtype=torch.int32, device=DEV), torch.empty(rows, device=DEV)
    P.medusa_sample(logits, u, token, prob, top_k=torch.tensor([700], dtype=torch.int32, device=DEV), rows_per_setting=rows,
                    ws=torch.empty(P.medusa_sample_workspace_bytes(rows, vocab), dtype=torch.uint8, device=DEV))
    l, us = logits.double().cpu().numpy(), u.double().cpu().numpy()
    settled = 0
    for r in range(rows):
        want, p, border = sampling.draw(l[r], us[r], top_k=700)
        if border >= BORDER:
            assert int(token[r]) == want and abs(float(prob[r]) - p) <= p * 2.0 ** -24 + BORDER
            settled += 1
    assert settled >= rows - 1
