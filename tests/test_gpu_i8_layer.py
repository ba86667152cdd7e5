"""GPU parity of models whose layers' products take 8-bit integers (the model descriptor's weights_i8), against the oracle's layer with the
same rows in 8 bits."""
import numpy as np
import pytest
import torch

import workload as W
import paper_2603_03383_amd as P
from oracle import medusa as O
from tests import gpu_util as G
from tests import util as U
from tests.test_gpu_parity import TOL, _i32, _layer_case, _scale

pytestmark = pytest.mark.gpu

# Oracle and library quantise the same rows, but the library's attention output, gate and up are rounded to 16 bits first, so some codes
# differ by one.  Were all of a row's rounding errors independent on the two sides, they would be apart by sqrt(2) times one side's error:
# 1 / sqrt(12) of a step of max / 127 per code; rows of bell-shaped numbers have their largest below 4.5 standard deviations and products of
# two of them below 12, so 1.0 % of what enters the O, QKV and gate/up products and 2.7 % of what enters the down product; gate and up hand
# on 1.0 % each to their product.  sqrt(1.0^2 + 1.0^2 + 2.7^2) = 3.0 %, times sqrt(2) 4.3 % of the layer's update, in the 2-norm.
UPDATE = 0.043


def check_layer(w, S_list, max_prefix, x_seed):
    r = _layer_case(w, S_list, max_prefix, x_seed=x_seed)
    x0 = W.hidden_state(w, x_seed, r["x"].shape[0], device=G.DEV).float().cpu().numpy().astype(np.float64)
    rel = np.linalg.norm(r["x"] - r["ref"]) / np.linalg.norm(r["ref"] - x0)
    assert rel <= UPDATE
    for b, S in enumerate(S_list):  # K and V come of codes that both sides have from the same fp32 rows
        k, v = r["kv"].read(0, b, S, r["T"])
        kc, vc = r["caches"][b]
        tol = TOL[w.dtype] if not w.kv_quant else 2.0 ** -4 + TOL[w.dtype]
        assert np.abs(U.to_np(k) - kc[:, S:]).max() <= tol * _scale(kc[:, S:])
        assert np.abs(U.to_np(v) - vc[:, S:]).max() <= tol * _scale(vc[:, S:])
        if S:  # prefix rows untouched
            k0, v0 = r["kv"].read(0, b, 0, S)
            if not w.kv_quant:
                assert np.array_equal(U.to_np(k0), kc[:, :S]) and np.array_equal(U.to_np(v0), vc[:, :S])
    print(f"{w.name} {S_list}: {rel:.2e} of the update")
    return r


SMALL = W.CONFIGS["cfg2_layer_bf16"].with_(d=256, n_heads=2, head_dim=128, ffn=704, weights_i8=True)


@pytest.mark.parametrize("S_list,max_prefix", [([0], 0), ([1], 5), ([77], 100), ([300, 0, 45], 300)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_small_layer(dtype, S_list, max_prefix):
    check_layer(SMALL.with_(dtype=dtype, name=f"i8_{dtype}"), S_list, max_prefix, f"i8_x{len(S_list)}")


@pytest.mark.parametrize("tree,prefix", [(W.TREE1, (0, 33, 700)), (W.TREE15, (64, 0, 130, 9, 200)), (W.TREE64K5, (50,))])
def test_other_trees(tree, prefix):
    check_layer(SMALL.with_(tree=tree, name=f"i8_{tree.name}"), list(prefix), max(prefix), f"i8_{tree.name}")


def test_grouped_heads_8_bit_cache_and_odd_widths():
    w = SMALL.with_(d=512, n_heads=4, n_kv_heads=2, ffn=1376, name="i8_gqa")
    check_layer(w, [100], 100, "i8_gqa")
    check_layer(w.with_(kv_quant="fp8e4m3", name="i8_gqa_kv8"), [100, 31], 100, "i8_gqa_kv8")
    # head_dim 64: q, k and v take the rotation's kernel of its own and the portable attention
    check_layer(SMALL.with_(d=192, n_heads=3, head_dim=64, ffn=352, name="i8_hd64"), [20, 3], 40, "i8_hd64")


def test_7b_width_layer():
    check_layer(W.CONFIGS["cfg2_layer_bf16"].with_(weights_i8=True, name="i8_7b"), [512], 512, "i8_7b")


def test_static_scratch_and_repeated_calls_give_the_same_bits():
    w = SMALL.with_(name="i8_static", prefix=(130,))
    dm = G.device_model(w.with_(vocab=1024), heads=False, n_layers=1)
    x0 = W.hidden_state(w, "i8_static", 64, device=G.DEV).float()
    out = []
    for call in range(3):
        kv = G.device_kv_random_prefix(dm, w, cap=130 + 64, n_layers=1)
        x, n = x0.clone(), _i32([130])
        if call < 2:
            P.tree_verify_layer(dm.desc, dm.layer(0), 0, x, kv.desc, n, 1, 130, dm.workspace(1, 130))
        else:
            P.tree_verify_layer_static(dm.desc, dm.layer(0), 0, x, kv.desc, n, 1, 130)
        torch.cuda.synchronize()
        out.append((x, kv.k.clone(), kv.v.clone()))
    for other in out[1:]:
        assert all(torch.equal(a, b) for a, b in zip(out[0], other))


@pytest.mark.parametrize("batch", [1, 2])
def test_two_layer_step_with_heads(batch):
    """heads -> verify -> accept -> compact on an 8-bit model.  Each layer may be off by UPDATE of its update, which is no longer than the
    stream; the second layer hands on what the first left: at most 2 UPDATE of the stream, and of the logits, which are a product of it."""
    w = W.CONFIGS["cfg3_step_1k"].with_(name="i8_step", d=512, n_heads=4, ffn=1408, vocab=2048, n_layers=2, weights_i8=True,
                                        prefix=(100, 40)[:batch])
    tree, model, dm = U.oracle_tree(w), U.oracle_model(w, device=G.DEV), G.device_model(w)
    S_max, T = max(w.prefix), 64
    kv = G.device_kv_random_prefix(dm, w, cap=S_max + T)
    h = W.hidden_state(w, "i8_heads", batch, device=G.DEV)
    buf = P.StepBuffers(dm, batch, S_max, want_logits=True)
    seq_len = _i32(list(w.prefix))
    P.run_step(dm, kv, buf, h.view(batch, 1, -1), None, None, seq_len)
    torch.cuda.synchronize()
    for b, S in enumerate(w.prefix):
        kc, vc = U.oracle_prefix_cache(w, b, S + T, device=G.DEV)
        tokens = buf.tree_tokens[b].cpu().numpy()
        ref = O.tree_verify_step(tokens, model, kc, vc, S, tree)
        for got, want in ((buf.logits[b], ref["logits"]), (buf.hidden[b], ref["hidden"])):
            assert np.linalg.norm(U.to_np(got) - want) <= 2 * UPDATE * np.linalg.norm(want)
        assert np.array_equal(buf.node_argmax[b].cpu().numpy(), O.argmax_lowest(buf.logits[b].cpu().numpy()))
        acc = O.accept_longest_prefix(tree, tokens, buf.node_argmax[b].cpu().numpy())
        assert int(buf.accept_len[b]) == acc["accept_len"] and int(seq_len[b]) == S + acc["accept_len"]


def test_chained_decoding_in_a_graph_equals_eager_steps():
    w = W.CONFIGS["cfg3_step_1k"].with_(name="i8_chain", d=512, n_heads=4, ffn=1408, vocab=2048, n_layers=2, weights_i8=True, prefix=(60,))
    dm = G.device_model(w)
    runs = []
    for use_graph in (False, True):
        kv = G.device_kv_random_prefix(dm, w, cap=60 + 64 + 64)
        dec = P.ChainedDecoder(dm, kv, 1, 60 + 64, use_graph=use_graph)
        dec.prime(W.hidden_state(w, "i8_chain", 1, device=G.DEV), _i32([7]), _i32([60]))
        tokens, lens = dec.run(5)
        torch.cuda.synchronize()
        dec.check_status()
        runs.append((tokens.cpu(), lens.cpu(), kv.k.cpu(), kv.v.cpu()))
    assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_view_with_tree_and_plain_models_are_unchanged():
    """The autoregressive view of an 8-bit model runs on the same weights; a model without the option has its own path."""
    w = SMALL.with_(name="i8_view", vocab=1024, n_layers=1, prefix=(20,))
    dm = G.device_model(w, heads=False)
    ar = dm.view_with_tree("tree1")
    assert ar.desc.weights_i8 == 1
    kv = G.device_kv_random_prefix(dm, w, cap=20 + 1)
    tokens, hidden = _i32([5]), torch.zeros(1, 1, 256, dtype=torch.bfloat16, device=G.DEV)
    argmax, ws = _i32([0]), ar.workspace(1, 20)
    P.tree_verify_step(ar.desc, ar.weights, tokens, kv.desc, _i32([20]), 1, 20, argmax, hidden, None, ws)
    model = U.oracle_model(w, device=G.DEV, heads=False)
    kc, vc = U.oracle_prefix_cache(w, 0, 21, device=G.DEV)
    _, want = O.causal_decode(np.array([5]), model, kc, vc, 20)
    assert np.linalg.norm(U.to_np(hidden)[0] - want) <= UPDATE * np.linalg.norm(want)


def test_refusals():
    w = SMALL.with_(name="i8_refuse", prefix=(8,))
    dm = G.device_model(w.with_(vocab=1024), heads=False, n_layers=1)
    kv = G.device_kv_random_prefix(dm, w, cap=8 + 64, n_layers=1)
    x, n, ws = torch.zeros(64, 256, device=G.DEV), _i32([8]), dm.workspace(1, 8)
    before = x.clone()
    lw = P.LayerWeights.from_buffer_copy(dm.layer(0))
    lw.wgateup += 4
    for layer, scratch in ((lw, ws), (dm.layer(0), torch.empty(ws.numel() + 16, dtype=torch.uint8, device=G.DEV)[8:8 + ws.numel()])):
        with pytest.raises(P.MedusaError) as e:
            P.tree_verify_layer(dm.desc, layer, 0, x, kv.desc, n, 1, 8, scratch)
        assert e.value.status == -1 and "16 bytes" in str(e.value)
    torch.cuda.synchronize()
    assert torch.equal(x, before)
