"""Sampled decoding: the tree step whose tokens are drawn, and the chain of operators of a step's end on 4-bit weights."""
import numpy as np
import pytest
import torch

import workload as W
import paper_2603_03383_amd as P
from oracle import medusa as O
from oracle import rows4, sampling
from tests import gpu_util as G
from tests import util as U
from tests.test_gpu_sample import BORDER

pytestmark = pytest.mark.gpu

SETTINGS = dict(temperature=0.9, top_k=50, top_p=0.95, min_p=0.001)
# as the library gets them: fp32
F32 = {k: (v if k == "top_k" else float(np.float32(v))) for k, v in SETTINGS.items()}


def _step(w, batch, seed, sampling_on=True):
    dm = G.device_model(w)
    T = w.tree.n_nodes
    S = 20
    kv = G.device_kv_random_prefix(dm, w.with_(prefix=(S,) * batch), cap=S + T)
    buf = P.StepBuffers(dm, batch, S, want_logits=True)
    buf.tree_tokens.copy_(torch.randint(0, w.vocab, (batch, T), generator=torch.Generator().manual_seed(seed)).to(torch.int32))
    smp = P.Sampling(dm, batch, **SETTINGS) if sampling_on else None
    if smp is not None:
        smp.u.copy_(torch.rand(batch, T, generator=torch.Generator().manual_seed(seed + 1)))
    seq_len = torch.full((batch,), S, dtype=torch.int32, device=G.DEV)
    return dm, kv, buf, smp, seq_len


@pytest.mark.parametrize("batch", [1, 3])
@pytest.mark.parametrize("name", ["cfg1_tiny_fp32"])
def test_a_step_accepts_the_path_of_drawn_tokens(name, batch):
    w = W.CONFIGS[name]
    dm, kv, buf, smp, seq_len = _step(w, batch, 5)
    T, tree = w.tree.n_nodes, U.oracle_tree(w)
    # a path that the draws follow: the model's own draws, put in as the nodes' tokens (a first pass finds them; a node's logits are its ancestors' alone)
    for _ in range(tree["K"] + 1):
        P.run_step(dm, kv, buf, None, None, None, seq_len.clone(), with_heads=False, sampling=smp)
        drawn = buf.node_argmax.clone()
        for n in range(1, T, 2):
            buf.tree_tokens[:, n] = drawn[:, int(tree["parent"][n])]
    n0 = seq_len.clone()
    P.run_step(dm, kv, buf, None, None, None, n0, with_heads=False, sampling=smp)
    torch.cuda.synchronize()
    logits, us = buf.logits.double().cpu().numpy(), smp.u.double().cpu().numpy()
    longest = 0
    for b in range(batch):
        tokens = buf.node_argmax[b].cpu().numpy()
        for n in range(T):
            want, p, border = sampling.draw(logits[b, n], us[b, n], **F32)
            if border >= BORDER:
                assert tokens[n] == want and abs(float(smp.prob[b, n]) - p) <= p * 2.0 ** -24 + BORDER
        acc = O.accept_longest_prefix(tree, buf.tree_tokens[b].cpu().numpy(), tokens)
        assert int(buf.accept_len[b]) == acc["accept_len"] and int(buf.next_root[b]) == acc["next_root"] and int(buf.last_node[b]) == acc["last_node"]
        assert buf.acc_tokens[b].cpu().tolist() == list(acc["acc_tokens"]) and int(n0[b]) == 20 + acc["accept_len"]
        longest = max(longest, acc["accept_len"])
    assert longest > 1  # drawn tokens were followed, not the root alone


def test_a_step_that_samples_needs_logits():
    w = W.CONFIGS["cfg1_tiny_fp32"]
    dm, kv, buf, smp, seq_len = _step(w, 1, 5)
    with pytest.raises(P.MedusaError):
        P.run_step(dm, kv, P.StepBuffers(dm, 1, 20), None, None, None, seq_len, with_heads=False, sampling=smp)
    dec = P.ChainedDecoder(dm, kv, 1, 20, use_graph=False, sampling=smp)
    with pytest.raises(P.MedusaError):
        dec.run(2)
    with pytest.raises(P.MedusaError):
        dec.run(2, torch.zeros(1, 1, w.tree.n_nodes))
    plain = P.ChainedDecoder(dm, kv, 1, 20, use_graph=False)
    with pytest.raises(P.MedusaError):
        plain.run(2, torch.zeros(2, 1, w.tree.n_nodes))


def test_the_chain_samples_the_same_text_from_a_graph_and_without():
    """And greedily (temperature 0) it gives what it gives without sampling."""
    w = W.CONFIGS["cfg1_tiny_fp32"]
    dm = G.device_model(w)
    S, steps, T = 24, 5, w.tree.n_nodes
    K1 = dm.tree_info["K"] + 1
    cap = S + steps * K1 + T
    hidden = W.hidden_state(w, "sampled_chain", 1, device=G.DEV)
    u = torch.rand(steps, 1, T, generator=torch.Generator().manual_seed(9)).to(G.DEV)

    def chain(use_graph, settings):
        kv = G.device_kv_random_prefix(dm, w.with_(prefix=(S,)), cap=cap)
        smp = None if settings is None else P.Sampling(dm, 1, **settings)
        dec = P.ChainedDecoder(dm, kv, 1, cap - T, use_graph=use_graph, sampling=smp)
        dec.prime(hidden, torch.tensor([3], dtype=torch.int32, device=G.DEV), torch.tensor([S], dtype=torch.int32, device=G.DEV))
        tokens, lens = dec.run(steps, None if smp is None else u)
        torch.cuda.synchronize()
        dec.check_status()
        return tokens.cpu(), lens.cpu()
    eager, graph = chain(False, SETTINGS), chain(True, SETTINGS)
    assert torch.equal(eager[0], graph[0]) and torch.equal(eager[1], graph[1])
    plain, greedy = chain(False, None), chain(False, dict(temperature=0.0))
    assert torch.equal(plain[0], greedy[0]) and torch.equal(plain[1], greedy[1])
    assert not torch.equal(eager[0], plain[0])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows", [1, 15, 64])
def test_feed_forward_vocabulary_and_draw_on_4_bit_weights(dtype, rows):
    """rows -> gated half -> down -> vocabulary -> token, as a step's end has them; the token is the definition's on the logits that came out, and the logits are
    those of the quantised matrices."""
    rng = np.random.default_rng(rows)
    d, ffn, vocab, group = 256, 688, 9000, 128
    td = {"bf16": torch.bfloat16, "fp16": torch.float16}[dtype]

    def matrix(n, k):
        w = torch.from_numpy((rng.standard_normal((n, k)) / np.sqrt(k)).astype(np.float32)).to(G.DEV, td)
        packed = torch.empty(P.medusa_packed_i4_bytes(n, k, group, True), dtype=torch.uint8, device=G.DEV)
        P.medusa_pack_weight_i4(w, group, packed, n, zeros=True)
        return packed, rows4.values(*rows4.quantize(w.float().cpu().numpy(), group, True, dtype), group)
    (gate, g64), (up, u64), (down, d64), (head, h64) = matrix(ffn, d), matrix(ffn, d), matrix(d, ffn), matrix(vocab, d)
    x = torch.from_numpy(rng.standard_normal((rows, d)).astype(np.float32)).to(G.DEV, td)
    u, y = torch.empty(rows, ffn, dtype=td, device=G.DEV), torch.empty(rows, d, dtype=td, device=G.DEV)
    logits = torch.empty(rows, vocab, device=G.DEV)
    token, prob, r = torch.empty(rows, dtype=torch.int32, device=G.DEV), torch.empty(rows, device=G.DEV), torch.rand(rows, generator=torch.Generator().manual_seed(rows)).to(G.DEV)
    need = max(P.medusa_swiglu_i4_workspace_bytes(rows, ffn, d), P.medusa_linear_i4_workspace_bytes(rows, d, ffn), P.medusa_linear_i4_workspace_bytes(rows, vocab, d),
               P.medusa_sample_workspace_bytes(rows, vocab))
    ws = torch.empty(need, dtype=torch.uint8, device=G.DEV)
    settings = dict(temperature=torch.tensor([0.8], device=G.DEV), top_p=torch.tensor([0.9], device=G.DEV))

    def end_of_step():
        P.medusa_swiglu_i4(x, gate, up, group, True, u, ws)
        P.medusa_linear_i4(u, down, group, True, y, ws)
        P.medusa_linear_i4(y, head, group, True, logits, ws)
        P.medusa_sample(logits, r, token, prob, rows_per_setting=rows, ws=ws, **settings)
    end_of_step()
    half = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}[dtype]
    xs, us, ys = (t.double().cpu().numpy() for t in (x, u, y))
    # each product on what it was given: its result's rounding (half a step), and fp32 sums, 2^-18 of the absolute sums at these lengths
    for got, want, size in [(us, rows4.swiglu(xs, g64, u64), np.abs(xs) @ np.abs(g64).T * (np.abs(xs) @ np.abs(u64).T)), (ys, rows4.linear(us, d64), np.abs(us) @ np.abs(d64).T)]:
        assert (np.abs(got - want) <= half * np.abs(want) + 2.0 ** -15 * size + 2.0 ** -24).all()
    assert (np.abs(logits.double().cpu().numpy() - rows4.linear(ys, h64)) <= 2.0 ** -15 * (np.abs(ys) @ np.abs(h64).T)).all()
    l = logits.double().cpu().numpy()
    for i in range(rows):
        want, p, border = sampling.draw(l[i], float(r[i]), temperature=float(np.float32(0.8)), top_p=float(np.float32(0.9)))
        if border >= BORDER:
            assert int(token[i]) == want and abs(float(prob[i]) - p) <= p * 2.0 ** -24 + BORDER
    keep = token.clone(), prob.clone()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        end_of_step()
    for _ in range(3):
        token.zero_(), prob.zero_(), logits.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(token, keep[0]) and torch.equal(prob, keep[1])
