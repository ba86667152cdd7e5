"""Captured calls of the 4-bit products and of sampling whose graphs share one workspace, replayed in turn with other work between them."""
import numpy as np
import pytest
import torch

import paper_2603_03383_amd as P

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def test_graphs_that_share_a_workspace():
    rng = np.random.default_rng(5)
    n, k, group = 20000, 261, 32
    packed = torch.empty(P.medusa_packed_i4_bytes(n, k, group, True), dtype=torch.uint8, device=DEV)
    w = torch.from_numpy((rng.standard_normal((n, k)) / 8).astype(np.float32)).to(DEV, torch.float16)
    P.medusa_pack_weight_i4(w, group, packed, n, zeros=True)
    sizes = (1, 90, 300)  # few rows; rows copied to aligned ones, and split rows; rows of a workgroup each
    need = max(max(P.medusa_linear_i4_workspace_bytes(m, n, k), P.medusa_sample_workspace_bytes(m, n)) for m in sizes)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    runs = []
    for m in sizes:
        x = torch.from_numpy(rng.standard_normal((m, k)).astype(np.float32)).to(DEV, torch.float16)
        u = torch.from_numpy(rng.random(m, dtype=np.float32)).to(DEV)
        logits, token, prob = torch.empty(m, n, device=DEV), torch.empty(m, dtype=torch.int32, device=DEV), torch.empty(m, device=DEV)
        top_p = torch.full((m,), 0.95, device=DEV)

        def step(x=x, u=u, logits=logits, token=token, prob=prob, top_p=top_p):
            P.medusa_linear_i4(x, packed, group, True, logits, ws)
            P.medusa_sample(logits, u, token, prob, top_p=top_p, ws=ws)
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            step()
        runs.append((step, graph, x, u, logits, token, prob))
    for turn in range(3):
        wants = []
        for step, _, x, u, logits, token, prob in runs:  # other inputs, and what they give without a graph
            x.copy_(torch.from_numpy(rng.standard_normal(tuple(x.shape)).astype(np.float32)))
            u.copy_(torch.from_numpy(rng.random(u.numel(), dtype=np.float32)))
            step()
            wants.append((logits.clone(), token.clone(), prob.clone()))
            logits.zero_(), token.zero_(), prob.zero_()
        for at in (2, 0, 1):
            runs[at][1].replay()
            ws.fill_(0xFF if turn == 1 else 0x5A)  # nothing is kept in it
        torch.cuda.synchronize()
        for (_, _, _, _, logits, token, prob), want in zip(runs, wants):
            assert torch.equal(logits, want[0]) and torch.equal(token, want[1]) and torch.equal(prob, want[2])
