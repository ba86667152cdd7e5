"""Pins of the oracle's decoder layer with 8-bit products: equal to the ordinary layer where nothing is lost, and to library operations on
what the rows stand for."""
import numpy as np
import torch

import workload as W
from oracle import medusa as O
from oracle import rows8
from tests import util as U


def _case(seed=3, S=5):
    w = W.CONFIGS["cfg1_tiny_fp32"].with_(name="i8_pin", d=64, n_heads=4, n_kv_heads=2, head_dim=16, ffn=96, vocab=64, n_layers=1)
    tree = U.oracle_tree(w)
    rng = np.random.default_rng(seed)
    cfg = dict(U.oracle_cfg(w), dtype="fp64")
    kc, vc = O.empty_cache(cfg, S + tree["T"])
    for c in (kc[0], vc[0]):
        c[:, :S] = rng.standard_normal(c[:, :S].shape)
    return w, tree, cfg, U.oracle_layer(w, 0), kc[0], vc[0], rng.standard_normal((tree["T"], w.d)), S


def test_layer_of_rows_in_8_bits_equals_library_operations_on_them():
    w, tree, cfg, lw, kc, vc, x, S = _case()
    T, H, Hkv, hd = tree["T"], 4, 2, 16
    ks, vs = kc.copy(), vc.copy()
    got = O.tree_verify_layer(x, lw, kc, vc, S, tree, dict(cfg, weights_i8=True))

    t = lambda a: torch.from_numpy(np.asarray(a, np.float64))  # noqa: E731
    f = torch.nn.functional

    def product(a, *names):
        codes, scale = rows8.quantize_rows(a.numpy())
        out = []
        for name in names:
            wc, ws = rows8.quantize_rows(lw[name])
            sums = t(codes).to(torch.int64) @ t(wc).to(torch.int64).T     # integers all the way
            out.append(sums.double() * t(scale)[:, None] * t(ws)[None, :])
        return out
    norm = lambda a, g: f.rms_norm(a, (w.d,), t(lw[g]), cfg["rms_eps"])  # noqa: E731
    pos = torch.tensor(S + tree["depth"].astype(np.int64))
    ang = pos[:, None] * cfg["rope_base"] ** (-2.0 * torch.arange(hd // 2, dtype=torch.float64) / hd)

    def rotated(a, heads):
        a = a.view(T, heads, hd).transpose(0, 1)
        z = torch.complex(a[..., :hd // 2], a[..., hd // 2:]) * torch.polar(torch.ones_like(ang), ang)
        return torch.cat([z.real, z.imag], dim=-1)
    q, k, v = product(norm(t(x), "g_attn"), "wq", "wk", "wv")
    q, k, v = rotated(q, H), rotated(k, Hkv), v.view(T, Hkv, hd).transpose(0, 1)
    K = torch.cat([t(ks[:, :S]), k], 1).repeat_interleave(H // Hkv, 0)
    V = torch.cat([t(vs[:, :S]), v], 1).repeat_interleave(H // Hkv, 0)
    att = f.scaled_dot_product_attention(q, K, V, attn_mask=torch.from_numpy(O.tree_visibility(tree, S)))
    y = t(x) + product(att.transpose(0, 1).reshape(T, H * hd), "wo")[0]
    gate, up = product(norm(y, "g_ffn"), "wgate", "wup")
    y = y + product(f.silu(gate) * up, "wdown")[0]
    assert np.abs(got - y.numpy()).max() < 1e-9
    assert np.abs(kc[:, S:S + T] - k.numpy()).max() < 1e-9 and np.abs(vc[:, S:S + T] - v.numpy()).max() < 1e-9


def test_layer_in_8_bits_is_near_the_ordinary_one():
    """A code is off by up to half a step: uniform, so 1 / sqrt(12) of a step on average.  Rows of 64 bell-shaped numbers have their largest
    at some 2.5 standard deviations, products of them at some 7: 0.6 % and 1.6 % of an input, as much again from each weight matrix.  The
    first product of the feed-forward block loses 0.6 % twice, in gate and in up, which the second's 1.6 % join: below 4 % of the update."""
    w, tree, cfg, lw, kc, vc, x, S = _case()
    plain = O.tree_verify_layer(x, lw, kc.copy(), vc.copy(), S, tree, cfg)
    eight = O.tree_verify_layer(x, lw, kc.copy(), vc.copy(), S, tree, dict(cfg, weights_i8=True))
    off = np.linalg.norm(eight - plain) / np.linalg.norm(plain - x)
    assert 1e-4 < off < 0.04
