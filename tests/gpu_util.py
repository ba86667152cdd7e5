"""GPU-side test helpers: build the device model / KV cache of a workload through the C-ABI."""
from __future__ import annotations

import numpy as np
import torch

import workload as W
import paper_2603_03383_amd as P
from paper_2603_03383_amd import DeviceKV, DeviceModel

DEV = "cuda:0"


def device_model(w: W.Workload, heads: bool = True, n_layers=None, gen_device=DEV) -> DeviceModel:
    """Weights are generated by the seeded generator directly on ``gen_device`` (bit-identical to the
    CPU generation the oracle's helpers use) and packed by the library."""
    L = w.n_layers if n_layers is None else n_layers
    dm = DeviceModel(d=w.d, n_heads=w.n_heads, head_dim=w.head_dim, ffn=w.ffn, vocab=w.vocab, n_layers=L,
                     dtype=w.dtype, tree=w.tree.name, n_kv_heads=w.n_kv_heads, rms_eps=w.rms_eps, rope_base=w.rope_base, device=DEV,
                     ffn_f16=w.ffn_f16, weights_i8=w.weights_i8)
    for l in range(L):
        mats = [W.layer_weight(w, l, m, gen_device) for m in W.LAYER_MATS]
        dm.add_layer(*mats, W.norm_gain(w, f"layer{l}.g_attn", gen_device), W.norm_gain(w, f"layer{l}.g_ffn", gen_device))
        del mats
    dm.set_embed(W.embedding(w, gen_device))
    dm.set_lm_head(W.lm_head(w, gen_device))
    dm.set_final_gain(W.norm_gain(w, "g_final", gen_device))
    if heads:
        for k in range(1, w.n_medusa + 1):
            dm.add_medusa_head(W.medusa_w1(w, k, gen_device), W.medusa_b1(w, k, gen_device), W.medusa_lm(w, k, gen_device))
    return dm.finalize()


def attention_plan(w: W.Workload, batch: int, max_prefix: int, fused: bool = True) -> dict:
    """How the library cuts the attention of a pass over `batch` sequences of up to max_prefix keys."""
    m = P.ModelDesc(w.d, w.n_heads, w.head_dim, w.ffn, w.vocab, w.n_layers, P.DTYPES[w.dtype], P.TREES[w.tree.name], w.rms_eps, w.rope_base, w.n_kv_heads)
    return P.medusa_attention_plan(m, batch, max_prefix, w.kv_quant, fused)


def device_kv_from_oracle(dm: DeviceModel, kcs, vcs, S_list, cap: int, quant: str = "") -> DeviceKV:
    """kcs[b][l], vcs[b][l]: oracle caches [H,cap_o,hd] (float64, storage-valued); first S_list[b] rows copied."""
    kv = DeviceKV(dm, batch=len(S_list), cap=cap, quant=quant)
    for b, S in enumerate(S_list):
        if S == 0:
            continue
        for l in range(len(kcs[b])):
            kv.write(l, b, 0, torch.from_numpy(np.ascontiguousarray(kcs[b][l][:, :S])),
                     torch.from_numpy(np.ascontiguousarray(vcs[b][l][:, :S])))
    return kv


def device_kv_random_prefix(dm: DeviceModel, w: W.Workload, cap: int, n_layers=None) -> DeviceKV:
    L = dm.desc.n_layers if n_layers is None else n_layers
    kv = DeviceKV(dm, batch=w.batch, cap=cap, n_layers=L, quant=w.kv_quant)
    for b in range(w.batch):
        for l in range(L):
            k, v = W.prefix_kv(w, l, b, DEV)
            kv.write(l, b, 0, k, v)
    return kv
