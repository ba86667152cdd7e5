"""ctypes binding of libmedusa_hip.so: the same names as include/medusa.h, argument marshalling only.

Every computation runs inside the library's HIP kernels.  PyTorch appears here only as the owner of
device memory (``tensor.data_ptr()``) and of the current HIP stream.  If the shared library has not been
built (``python -c "import __graft_entry__ as g; g.build()"``) importing works but the first call raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmedusa_hip.so")

MDZ_OK = 0
MDZ_BF16, MDZ_FP32, MDZ_FP16 = 0, 1, 2
MDZ_TREE_15, MDZ_TREE_64, MDZ_TREE_1, MDZ_TREE_64_K5 = 0, 1, 2, 3
MDZ_MAX_HEADS = 8
DTYPES = {"bf16": MDZ_BF16, "fp32": MDZ_FP32, "fp16": MDZ_FP16}
MDZ_KV_PLAIN, MDZ_KV_FP8E4M3 = 0, 1
KV_QUANT = {"": MDZ_KV_PLAIN, "fp8e4m3": MDZ_KV_FP8E4M3}
TREES = {"tree15": MDZ_TREE_15, "tree64": MDZ_TREE_64, "tree1": MDZ_TREE_1, "tree64k5": MDZ_TREE_64_K5}


class MedusaError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"libmedusa_hip status {status}: {msg}")
        self.status = status


class ModelDesc(C.Structure):
    _fields_ = [("d", C.c_int32), ("n_heads", C.c_int32), ("head_dim", C.c_int32), ("ffn", C.c_int32),
                ("vocab", C.c_int32), ("n_layers", C.c_int32), ("dtype", C.c_int32), ("tree", C.c_int32),
                ("rms_eps", C.c_float), ("rope_base", C.c_float), ("n_kv_heads", C.c_int32),
                ("ffn_f16", C.c_int32), ("weights_i8", C.c_int32)]


class LayerWeights(C.Structure):
    _fields_ = [("wqkv", C.c_void_p), ("wo", C.c_void_p), ("wgateup", C.c_void_p), ("wdown", C.c_void_p),
                ("g_attn", C.c_void_p), ("g_ffn", C.c_void_p)]


class Weights(C.Structure):
    _fields_ = [("layers", C.POINTER(LayerWeights)), ("embed", C.c_void_p), ("lm_head", C.c_void_p),
                ("g_final", C.c_void_p), ("n_medusa", C.c_int32), ("head_w1", C.POINTER(C.c_void_p)),
                ("head_b1", C.POINTER(C.c_void_p)), ("head_lm", C.POINTER(C.c_void_p))]


class KvDesc(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("n_layers", C.c_int32), ("batch", C.c_int32),
                ("n_heads", C.c_int32), ("head_dim", C.c_int32), ("cap", C.c_int32), ("dtype", C.c_int32), ("quant", C.c_int32),
                ("status", C.c_void_p)]


_lib = None

_SIGNATURES = {
    "medusa_tree_info": (C.c_int, [C.c_int] + [C.c_void_p] * 5),
    "medusa_tree_tables": (C.c_int, [C.c_int] + [C.c_void_p] * 5),
    "medusa_gemm_plan": (C.c_int, [C.c_int] * 5 + [C.c_void_p] * 4),
    "medusa_gemm_slot_count": (C.c_int, [C.c_int] * 6),
    "medusa_attention_plan": (C.c_int, [C.POINTER(ModelDesc)] + [C.c_int] * 4 + [C.c_void_p] * 4),
    "medusa_gemm_many_rows_plan": (C.c_int, [C.c_int] * 6 + [C.c_void_p] * 4),
    "medusa_last_error": (C.c_char_p, []),
    "medusa_profile_begin": (C.c_int, [C.c_int]),
    "medusa_profile_end": (C.c_int, [C.c_char_p, C.c_int64]),
    "medusa_stream_read": (C.c_int, [C.c_void_p, C.c_int64, C.c_int, C.c_void_p, C.c_void_p]),
    "medusa_stream_read_bytes": (C.c_int64, [C.c_int64, C.c_int]),
    "medusa_stream_copy": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]),
    "medusa_pack_tile_rows": (C.c_int, [C.c_int]),
    "medusa_packed_bytes": (C.c_int64, [C.c_int, C.c_int64, C.c_int64]),
    "medusa_pack_weight_bf16_as_f16": (C.c_int, [C.c_void_p, C.c_int64, C.c_int64, C.c_void_p, C.c_int64, C.c_int64,
                                                 C.c_int64, C.c_void_p]),
    "medusa_pack_weight": (C.c_int, [C.c_int, C.c_void_p, C.c_int64, C.c_int64, C.c_void_p, C.c_int64, C.c_int64,
                                     C.c_int64, C.c_void_p]),
    "medusa_packed_i8_bytes": (C.c_int64, [C.c_int64, C.c_int64]),
    "medusa_pack_weight_i8": (C.c_int, [C.c_int, C.c_void_p, C.c_int64, C.c_int64, C.c_void_p, C.c_int64, C.c_int64, C.c_void_p]),
    "medusa_pack_codes_i8": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_int64, C.c_void_p, C.c_int64, C.c_int64, C.c_void_p]),
    "medusa_quantize_rows_i8": (C.c_int, [C.c_int, C.c_void_p, C.c_int, C.c_int] + [C.c_void_p] * 4),
    "medusa_residual_rmsnorm_i8": (C.c_int, [C.c_int, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_float, C.c_int, C.c_int] + [C.c_void_p] * 5),
    "medusa_swiglu_i8": (C.c_int, [C.c_int, C.c_void_p, C.c_int, C.c_int] + [C.c_void_p] * 4),
    "medusa_linear_i8_workspace_bytes": (C.c_int64, [C.c_int] * 3),
    "medusa_linear_i8_plan": (C.c_int, [C.c_int] * 3 + [C.c_void_p] * 3),
    "medusa_linear_i8_parts_plan": (C.c_int64, [C.c_int] * 3 + [C.c_void_p]),
    "medusa_test_i8_update_norm": (C.c_int, [C.c_int] + [C.c_void_p] * 3 + [C.c_int] * 3 + [C.c_void_p, C.c_void_p, C.c_float] + [C.c_void_p] * 4 +
                                   [C.c_int64, C.c_void_p]),
    "medusa_linear_i8": (C.c_int, [C.c_void_p] * 3 + [C.c_int] * 4 + [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]),
    "medusa_packed_i4_bytes": (C.c_int64, [C.c_int64, C.c_int64, C.c_int, C.c_int]),
    "medusa_pack_weight_i4": (C.c_int, [C.c_int, C.c_void_p, C.c_int64, C.c_int64, C.c_int, C.c_int, C.c_void_p, C.c_int64, C.c_int64, C.c_void_p]),
    "medusa_pack_codes_i4": (C.c_int, [C.c_int] + [C.c_void_p] * 3 + [C.c_int64, C.c_int64, C.c_int, C.c_void_p, C.c_int64, C.c_int64, C.c_void_p]),
    "medusa_linear_i4_workspace_bytes": (C.c_int64, [C.c_int] * 3),
    "medusa_linear_i4": (C.c_int, [C.c_int, C.c_void_p, C.c_void_p] + [C.c_int] * 6 + [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]),
    "medusa_swiglu_i4_workspace_bytes": (C.c_int64, [C.c_int] * 3),
    "medusa_swiglu_i4": (C.c_int, [C.c_int] + [C.c_void_p] * 3 + [C.c_int] * 5 + [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]),
    "medusa_sample_workspace_bytes": (C.c_int64, [C.c_int] * 2),
    "medusa_sample": (C.c_int, [C.c_int, C.c_void_p, C.c_int64, C.c_int, C.c_int] + [C.c_void_p] * 4 + [C.c_int] + [C.c_void_p] * 4 + [C.c_int64, C.c_void_p]),
    "medusa_kv_bytes": (C.c_int64, [C.POINTER(KvDesc)]),
    "medusa_kv_init": (C.c_int, [C.POINTER(KvDesc), C.c_void_p]),
    "medusa_test_force_unfused_rope": (C.c_int, [C.c_int]),
    "medusa_kv_write": (C.c_int, [C.POINTER(KvDesc), C.c_int, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p,
                                  C.c_void_p]),
    "medusa_kv_read": (C.c_int, [C.POINTER(KvDesc), C.c_int, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p,
                                 C.c_void_p]),
    "medusa_workspace_bytes": (C.c_int64, [C.POINTER(ModelDesc), C.c_int, C.c_int]),
    "medusa_heads": (C.c_int, [C.POINTER(ModelDesc), C.POINTER(Weights), C.c_void_p, C.c_void_p, C.c_void_p, C.c_int,
                               C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]),
    "tree_verify_layer": (C.c_int, [C.POINTER(ModelDesc), C.POINTER(LayerWeights), C.c_int, C.c_void_p,
                                    C.POINTER(KvDesc), C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_int64,
                                    C.c_void_p]),
    "tree_verify_layer_static_scratch_bytes": (C.c_int64, []),
    "tree_verify_layer_static": (C.c_int, [C.POINTER(ModelDesc), C.POINTER(LayerWeights), C.c_int, C.c_void_p,
                                           C.POINTER(KvDesc), C.c_void_p, C.c_int, C.c_int, C.c_void_p]),
    "tree_verify_step": (C.c_int, [C.POINTER(ModelDesc), C.POINTER(Weights), C.c_void_p, C.POINTER(KvDesc), C.c_void_p,
                                   C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64,
                                   C.c_void_p]),
    "accept_longest_prefix": (C.c_int, [C.c_int, C.c_void_p, C.c_void_p, C.c_int] + [C.c_void_p] * 7),
    "kv_compact": (C.c_int, [C.POINTER(KvDesc), C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int,
                             C.c_int, C.c_void_p]),
}

EXPORTED = tuple(_SIGNATURES)


def lib():
    """The loaded shared library; raises if it has not been built.  There is no fallback."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise MedusaError(-100, f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
        l = C.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            f = getattr(l, name)
            f.restype, f.argtypes = res, args
        _lib = l
    return _lib


def _check(status: int):
    if status < 0:
        raise MedusaError(int(status), lib().medusa_last_error().decode("utf-8", "replace"))
    return status


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    assert t.is_contiguous(), "tensors handed to the library must be contiguous"
    return C.c_void_p(t.data_ptr())


def _stream(stream) -> C.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


# ---------------------------------------------------------------------------------------------
# introspection
# ---------------------------------------------------------------------------------------------

def medusa_tree_info(tree: int) -> dict:
    T, K, P, NC = (C.c_int32() for _ in range(4))
    topk = (C.c_int32 * MDZ_MAX_HEADS)()
    _check(lib().medusa_tree_info(tree, C.byref(T), C.byref(K), C.byref(P), C.byref(NC), topk))
    return dict(T=T.value, K=K.value, n_paths=P.value, n_cand=NC.value, topk=tuple(topk[:K.value]))


def medusa_gemm_plan(dtype: int, M: int, N: int, K: int, max_split: int) -> dict:
    vals = [C.c_int32() for _ in range(4)]
    _check(lib().medusa_gemm_plan(dtype, M, N, K, max_split, *[C.byref(v) for v in vals]))
    return dict(zip(("grid", "band_cols", "n_stages", "max_slots"), [v.value for v in vals]))


def medusa_gemm_slot_count(dtype: int, M: int, N: int, K: int, max_split: int, col: int) -> int:
    n = lib().medusa_gemm_slot_count(dtype, M, N, K, max_split, col)
    _check(n)
    return n


def medusa_gemm_many_rows_plan(dtype: int, M: int, N: int, K: int, max_split: int, swiglu: bool = False) -> dict:
    vals = [C.c_int32() for _ in range(4)]
    _check(lib().medusa_gemm_many_rows_plan(dtype, M, N, K, max_split, int(swiglu), *[C.byref(v) for v in vals]))
    return dict(zip(("wide", "tile_rows", "tile_cols", "k_splits"), [v.value for v in vals]))


def medusa_attention_plan(model: "ModelDesc", B: int, max_prefix: int, kv_quant: str = "", fused: bool = True) -> dict:
    vals = [C.c_int32() for _ in range(4)]
    _check(lib().medusa_attention_plan(C.byref(model), KV_QUANT[kv_quant], B, max_prefix, int(fused), *[C.byref(v) for v in vals]))
    kernel, queries, splits, ordered = (v.value for v in vals)
    return dict(kernel=("portable", "tree", "one_mfma", "one_fma")[kernel], queries=queries, splits=splits, ordered=bool(ordered))


def medusa_tree_tables(tree: int) -> dict:
    info = medusa_tree_info(tree)
    T, K, P = info["T"], info["K"], info["n_paths"]
    parent = np.zeros(T, np.int32)
    depth = np.zeros(T, np.int32)
    cand_slot = np.zeros(T, np.int32)
    anc = np.zeros(T, np.uint64)
    retrieve = np.zeros((P, K + 1), np.int32)
    _check(lib().medusa_tree_tables(tree, parent.ctypes.data, depth.ctypes.data, cand_slot.ctypes.data,
                                    anc.ctypes.data, retrieve.ctypes.data))
    return dict(info, parent=parent, depth=depth, cand_slot=cand_slot, anc_mask=anc, retrieve=retrieve)


def medusa_profile_begin(max_launches: int) -> None:
    _check(lib().medusa_profile_begin(max_launches))


def medusa_profile_end() -> dict:
    """{family: dict(launches, total_us, min_us, max_us)}"""
    buf = C.create_string_buffer(4096)
    _check(lib().medusa_profile_end(buf, len(buf)))
    out = {}
    for line in buf.value.decode().splitlines():
        name, n, tot, mn, mx = line.split(",")
        out[name] = dict(launches=int(n), total_us=float(tot), min_us=float(mn), max_us=float(mx))
    return out


def medusa_stream_read(src: torch.Tensor, nbytes: int, n_workgroups: int, sink4: torch.Tensor, stream=None) -> int:
    """Enqueues the read stream over the first nbytes of src; returns the bytes actually read."""
    _check(lib().medusa_stream_read(_ptr(src), nbytes, n_workgroups, _ptr(sink4), _stream(stream)))
    return lib().medusa_stream_read_bytes(nbytes, n_workgroups)


def medusa_stream_copy(src: torch.Tensor, dst: torch.Tensor, nbytes: int, stream=None) -> None:
    _check(lib().medusa_stream_copy(_ptr(src), _ptr(dst), nbytes, _stream(stream)))


def medusa_pack_tile_rows(dtype: int) -> int:
    return _check(lib().medusa_pack_tile_rows(dtype))


def medusa_packed_bytes(dtype: int, n_rows: int, k: int) -> int:
    return _check(lib().medusa_packed_bytes(dtype, n_rows, k))


def medusa_pack_weight_bf16_as_f16(src: torch.Tensor, dst: torch.Tensor, dst_rows: int, tile_offset: int = 0,
                                   tile_stride: int = 1, stream=None) -> None:
    n_rows, k = src.shape
    _check(lib().medusa_pack_weight_bf16_as_f16(_ptr(src), n_rows, k, _ptr(dst), dst_rows, tile_offset, tile_stride,
                                                _stream(stream)))


def medusa_pack_weight(dtype: int, src: torch.Tensor, dst: torch.Tensor, dst_rows: int, tile_offset: int = 0,
                       tile_stride: int = 1, stream=None) -> None:
    n_rows, k = src.shape
    _check(lib().medusa_pack_weight(dtype, _ptr(src), n_rows, k, _ptr(dst), dst_rows, tile_offset, tile_stride,
                                    _stream(stream)))


# ---------------------------------------------------------------------------------------------
# 8-bit integer products
# ---------------------------------------------------------------------------------------------
MDZ_I8_TILE_ROWS = 16
_STORAGE = {torch.bfloat16: MDZ_BF16, torch.float16: MDZ_FP16, torch.float32: MDZ_FP32}


def _operand(name: str, t: Optional[torch.Tensor], shape, dtype, device: int) -> Optional[int]:
    """Address of a tensor that has this shape and type and lies on this GPU; None stays None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device or not t.is_contiguous():
        if t.dtype is not dtype or t.shape != shape:
            raise MedusaError(-2, f"{name}: {tuple(t.shape)} {t.dtype}, expected {tuple(shape)} {dtype}")
        if not t.is_contiguous():
            raise MedusaError(-2, f"{name}: tensors handed to the library must be contiguous")
        raise MedusaError(-1, f"{name}: on {t.device}; a call's tensors lie on one GPU")
    return t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_of(device: int, stream):
    """The caller's stream, or the current one, for tensors on this GPU: the library launches on the current device."""
    if device < 0 or torch.cuda.current_device() != device:
        raise MedusaError(-1, "the tensors do not lie on a GPU" if device < 0 else
                          f"the tensors lie on cuda:{device}, the current device is cuda:{torch.cuda.current_device()}")
    # (the handle itself where torch has a call for it: a Stream object takes 3 us to make)
    return _raw_stream(device) if stream is None and _raw_stream is not None else _stream(stream)


def _int32(what: str, *sizes: int) -> None:
    """The library takes these sizes as 32-bit integers (ctypes would hand on their low bits)."""
    if max(sizes) > 0x7FFFFFFF:
        raise MedusaError(-3, f"{what}: {sizes}: sizes up to 2^31 - 1")


def _fits(what: str, bits: int, *numbers: int) -> None:
    """The same for numbers that may lie below zero too."""
    if any(n >> (bits - 1) not in (0, -1) for n in numbers):
        raise MedusaError(-3, f"{what}: {numbers}: {bits}-bit integers")


def _rows(name: str, t: torch.Tensor):
    """(shape, storage dtype, GPU) of a tensor of rows."""
    shape, dtype = t.shape, _STORAGE.get(t.dtype)
    if len(shape) != 2 or dtype is None:
        raise MedusaError(-2, f"{name}: {tuple(shape)} {t.dtype}, expected rows of a storage dtype")
    if (shape[0] | shape[1]) >> 31:
        _int32(name, *shape)
    return shape, dtype, t.get_device()


@functools.lru_cache(maxsize=None)
def medusa_packed_i8_bytes(n_rows: int, k: int) -> int:
    return _check(lib().medusa_packed_i8_bytes(n_rows, k))


def _packed_i8(dst: torch.Tensor, dst_rows: int, k: int, device: int, whole: bool = False) -> int:
    """whole: the matrix is read, and its scales stand where its rows end: a buffer of other sizes was packed for another."""
    got, want = dst.numel() * dst.element_size(), medusa_packed_i8_bytes(dst_rows, k)
    if got < want or (whole and got != want):
        raise MedusaError(-2, f"packed: {got} bytes are not those of [{dst_rows}, {k}], {want}")
    return _operand("packed", dst, dst.shape, dst.dtype, device)


def medusa_pack_weight_i8(src: torch.Tensor, dst: torch.Tensor, dst_rows: int, tile_offset: int = 0, stream=None) -> None:
    """src [n, k] of a storage dtype -> rows 16 * tile_offset .. of the packed 8-bit matrix dst, quantised per row."""
    shape, dtype, gpu = _rows("src", src)
    _check(lib().medusa_pack_weight_i8(dtype, _operand("src", src, shape, src.dtype, gpu), shape[0], shape[1],
                                       _packed_i8(dst, dst_rows, shape[1], gpu), dst_rows, tile_offset, _stream_of(gpu, stream)))


def medusa_pack_codes_i8(codes: torch.Tensor, scales: torch.Tensor, dst: torch.Tensor, dst_rows: int, tile_offset: int = 0,
                         stream=None) -> None:
    """codes int8 [n, k] with scales fp32 [n] -> the same rows of the packed 8-bit matrix dst."""
    if codes.dim() != 2:
        raise MedusaError(-2, f"codes: {tuple(codes.shape)}, expected rows")
    (n, k), gpu = codes.shape, codes.get_device()
    _check(lib().medusa_pack_codes_i8(_operand("codes", codes, (n, k), torch.int8, gpu), _operand("scales", scales, (n,), torch.float32, gpu),
                                      n, k, _packed_i8(dst, dst_rows, k, gpu), dst_rows, tile_offset, _stream_of(gpu, stream)))


def medusa_quantize_rows_i8(src, codes, scales, values=None, stream=None) -> None:
    """src [rows, d] -> codes int8 [rows, d], scales fp32 [rows]; values (optional, src's type): what they stand for."""
    shape, dtype, gpu = _rows("src", src)
    rows, d = shape
    _check(lib().medusa_quantize_rows_i8(
        dtype, _operand("src", src, shape, src.dtype, gpu), rows, d, _operand("codes", codes, shape, torch.int8, gpu),
        _operand("scales", scales, (rows,), torch.float32, gpu), _operand("values", values, shape, src.dtype, gpu), _stream_of(gpu, stream)))


def medusa_residual_rmsnorm_i8(x, delta, gain, eps: float, x_out, codes, scales, values=None, stream=None) -> None:
    """x [rows, d] fp32 (+ delta, fp32 or gain's type, or None) -> x_out (x itself, another, or None) and RMSNorm(x') in 8 bits."""
    shape, _, gpu = _rows("x", x)
    rows, d = shape
    td, td_delta = gain.dtype, torch.float32 if delta is None or delta.dtype is torch.float32 else gain.dtype
    if td not in _STORAGE:
        raise MedusaError(-2, f"gain: {td} is no storage dtype")
    _check(lib().medusa_residual_rmsnorm_i8(
        _STORAGE[td], _operand("x", x, shape, torch.float32, gpu), _operand("delta", delta, shape, td_delta, gpu), _STORAGE[td_delta],
        _operand("gain", gain, (d,), td, gpu), eps, rows, d, _operand("x_out", x_out, shape, torch.float32, gpu),
        _operand("codes", codes, shape, torch.int8, gpu), _operand("scales", scales, (rows,), torch.float32, gpu),
        _operand("values", values, shape, td, gpu), _stream_of(gpu, stream)))


def medusa_swiglu_i8(gate_up, codes, scales, values=None, stream=None) -> None:
    """gate_up [rows, 2 ffn] (gate | up) -> SiLU(gate) * up in 8 bits, codes [rows, ffn]."""
    (rows, width), dtype, gpu = _rows("gate_up", gate_up)
    shape = (rows, width // 2)
    _check(lib().medusa_swiglu_i8(
        dtype, _operand("gate_up", gate_up, (rows, shape[1] * 2), gate_up.dtype, gpu), rows, shape[1],
        _operand("codes", codes, shape, torch.int8, gpu), _operand("scales", scales, (rows,), torch.float32, gpu),
        _operand("values", values, shape, gate_up.dtype, gpu), _stream_of(gpu, stream)))


def medusa_linear_i8_workspace_bytes(M: int, N: int, K: int) -> int:
    _int32("linear_i8", M, N, K)
    return _check(lib().medusa_linear_i8_workspace_bytes(M, N, K))


def medusa_linear_i8_plan(M: int, N: int, K: int) -> dict:
    _int32("linear_i8", M, N, K)
    vals = [C.c_int32() for _ in range(3)]
    _check(lib().medusa_linear_i8_plan(M, N, K, *[C.byref(v) for v in vals]))
    return dict(zip(("tile_rows", "tile_cols", "k_splits"), [v.value for v in vals]))


def medusa_linear_i8_parts_plan(M: int, N: int, K: int) -> dict:
    _int32("linear_i8", M, N, K)
    splits = C.c_int32()
    need = _check(lib().medusa_linear_i8_parts_plan(M, N, K, C.byref(splits)))
    return dict(k_splits=splits.value, workspace_bytes=need)


def medusa_test_i8_update_norm(codes, scales, packed, x, gain, eps: float, codes_out, scales_out, part, ws, stream=None) -> None:
    """Test hook (include/medusa_bench.h): x += product, and the next norm's codes and scales, as an 8-bit layer makes them."""
    (M, d), _, gpu = _rows("x", x)
    K = codes.shape[-1]
    _check(lib().medusa_test_i8_update_norm(
        _STORAGE[gain.dtype], _operand("codes", codes, (M, K), torch.int8, gpu), _operand("scales", scales, (M,), torch.float32, gpu),
        _packed_i8(packed, d, K, gpu, whole=True), M, d, K, _operand("x", x, (M, d), torch.float32, gpu), _operand("gain", gain, (d,), gain.dtype, gpu), eps,
        _operand("codes_out", codes_out, (M, d), torch.int8, gpu), _operand("scales_out", scales_out, (M,), torch.float32, gpu),
        _operand("part", part, (M, d), torch.float32, gpu), _operand("ws", ws, ws.shape, ws.dtype, gpu), ws.numel() * ws.element_size(),
        _stream_of(gpu, stream)))


def medusa_linear_i8(codes, scales, packed, y, ws=None, stream=None) -> None:
    """y [M, N] (any storage dtype) = rows (codes [M, K], scales [M]) x the packed 8-bit matrix [N, K], transposed; packed: its
    medusa_packed_i8_bytes(N, K) bytes."""
    shape, out, gpu = _rows("y", y)
    M, N = shape
    if codes.dim() != 2:
        raise MedusaError(-2, f"codes: {tuple(codes.shape)}, expected rows")
    K = codes.shape[1]
    _check(lib().medusa_linear_i8(
        _operand("codes", codes, (M, K), torch.int8, gpu), _operand("scales", scales, (M,), torch.float32, gpu),
        _packed_i8(packed, N, K, gpu, whole=True), M, N, K, out, _operand("y", y, shape, y.dtype, gpu),
        None if ws is None else _operand("ws", ws, ws.shape, ws.dtype, gpu), 0 if ws is None else ws.numel() * ws.element_size(),
        _stream_of(gpu, stream)))


# ---------------------------------------------------------------------------------------------
# 4-bit weights
# ---------------------------------------------------------------------------------------------
MDZ_I4_TILE_ROWS = 16


@functools.lru_cache(maxsize=None)
def medusa_packed_i4_bytes(n_rows: int, k: int, group: int, zeros: bool = False) -> int:
    _fits("packed_i4_bytes", 64, n_rows, k)
    _fits("packed_i4_bytes", 32, group, int(zeros))
    return _check(lib().medusa_packed_i4_bytes(n_rows, k, group, int(zeros)))


def _whole(name: str, t: torch.Tensor, device: int) -> int:
    """Address of a contiguous tensor on this GPU whose shape and type are known to be right, or free."""
    if t.get_device() != device or not t.is_contiguous():
        return _operand(name, t, t.shape, t.dtype, device)
    return t.data_ptr()


def _packed_i4(name: str, t: torch.Tensor, n: int, k: int, group: int, zeros: bool, device: int) -> int:
    """Scales and zero points stand where the codes end: a buffer of other sizes was packed for another matrix."""
    got, want = t.nbytes, medusa_packed_i4_bytes(n, k, group, zeros)
    if got != want:
        raise MedusaError(-2, f"{name}: {got} bytes are not those of [{n}, {k}] in groups of {group}, {want}")
    return _whole(name, t, device)


def medusa_pack_weight_i4(src: torch.Tensor, group: int, dst: torch.Tensor, dst_rows: int, tile_offset: int = 0, zeros: bool = False, stream=None) -> None:
    """src [n, k] of bf16 or fp16 -> rows 16 * tile_offset .. of the packed 4-bit matrix dst, quantised in groups of a row's features."""
    shape, dtype, gpu = _rows("src", src)
    _fits("tile_offset", 64, tile_offset)
    _check(lib().medusa_pack_weight_i4(dtype, _operand("src", src, shape, src.dtype, gpu), shape[0], shape[1], group, int(zeros),
                                       _packed_i4("packed", dst, dst_rows, shape[1], group, zeros, gpu), dst_rows, tile_offset, _stream_of(gpu, stream)))


def medusa_pack_codes_i4(codes: torch.Tensor, scales: torch.Tensor, zeros: Optional[torch.Tensor], group: int, dst: torch.Tensor, dst_rows: int,
                         tile_offset: int = 0, stream=None) -> None:
    """codes uint8 [n, k] with scales (bf16 or fp16) and zeros (uint8, or None) [n, ceil(k / group)] -> the same rows of the packed matrix dst."""
    if codes.dim() != 2 or scales.dtype not in _STORAGE:
        raise MedusaError(-2, f"codes: {tuple(codes.shape)}, scales: {scales.dtype}, expected rows and scales of a storage dtype")
    (n, k), gpu = codes.shape, codes.get_device()
    _fits("tile_offset", 64, tile_offset)
    packed = _packed_i4("packed", dst, dst_rows, k, group, zeros is not None, gpu)
    groups = (n, -(-k // group))
    _check(lib().medusa_pack_codes_i4(_STORAGE[scales.dtype], _operand("codes", codes, (n, k), torch.uint8, gpu), _operand("scales", scales, groups, scales.dtype, gpu),
                                      _operand("zeros", zeros, groups, torch.uint8, gpu), n, k, group, packed, dst_rows, tile_offset, _stream_of(gpu, stream)))


def medusa_linear_i4_workspace_bytes(M: int, N: int, K: int) -> int:
    _int32("linear_i4", M, N, K)
    return _check(lib().medusa_linear_i4_workspace_bytes(M, N, K))


def medusa_swiglu_i4_workspace_bytes(M: int, ffn: int, K: int) -> int:
    _int32("swiglu_i4", M, ffn, K)
    return _check(lib().medusa_swiglu_i4_workspace_bytes(M, ffn, K))


def medusa_linear_i4(x: torch.Tensor, packed: torch.Tensor, group: int, zeros: bool, y: torch.Tensor, ws: Optional[torch.Tensor] = None, stream=None) -> None:
    """y [M, N] (any storage dtype) = x [M, K] (bf16 or fp16) times the packed 4-bit matrix [N, K], transposed."""
    (M, K), dtype, gpu = _rows("x", x)
    (rows, N), out, _ = _rows("y", y)
    if rows != M:
        _operand("y", y, (M, N), y.dtype, gpu)
    _check(lib().medusa_linear_i4(
        dtype, _whole("x", x, gpu), _packed_i4("packed", packed, N, K, group, zeros, gpu), M, N, K, group, int(zeros), out, _whole("y", y, gpu),
        None if ws is None else _whole("ws", ws, gpu), 0 if ws is None else ws.nbytes, _stream_of(gpu, stream)))


def medusa_swiglu_i4(x: torch.Tensor, gate: torch.Tensor, up: torch.Tensor, group: int, zeros: bool, y: torch.Tensor, ws: Optional[torch.Tensor] = None,
                     stream=None) -> None:
    """y [M, ffn] = SiLU(x gate^T) * (x up^T): x [M, K] and y of bf16 or fp16, gate and up packed 4-bit matrices [ffn, K]."""
    (M, K), dtype, gpu = _rows("x", x)
    (rows, N), out, _ = _rows("y", y)
    if rows != M or out != dtype:
        _operand("y", y, (M, N), x.dtype, gpu)
    _check(lib().medusa_swiglu_i4(
        dtype, _whole("x", x, gpu), _packed_i4("gate", gate, N, K, group, zeros, gpu), _packed_i4("up", up, N, K, group, zeros, gpu), M, N, K, group, int(zeros),
        _whole("y", y, gpu), None if ws is None else _whole("ws", ws, gpu), 0 if ws is None else ws.nbytes, _stream_of(gpu, stream)))


# ---------------------------------------------------------------------------------------------
# sampling
# ---------------------------------------------------------------------------------------------
def medusa_sample_workspace_bytes(rows: int, vocab: int) -> int:
    _int32("sample", rows, vocab)
    return _check(lib().medusa_sample_workspace_bytes(rows, vocab))


def medusa_sample(logits: torch.Tensor, u: torch.Tensor, token: torch.Tensor, prob: Optional[torch.Tensor] = None, *, temperature=None, top_k=None,
                  top_p=None, min_p=None, rows_per_setting: int = 1, ws: Optional[torch.Tensor] = None, stream=None) -> None:
    """logits [rows, vocab] of a storage dtype (rows may lie further apart), u fp32 [rows] -> token int32 [rows], prob fp32 [rows] (optional).  The settings:
    device tensors [ceil(rows / rows_per_setting)], top_k int32 and the others fp32, or None."""
    (rows, vocab), dtype, gpu = _rows("logits", logits)
    if rows_per_setting <= 0 or rows_per_setting >> 31:
        raise MedusaError(-1, f"sample: {rows_per_setting} rows per setting")
    ld, step = logits.stride()
    if rows <= 1:
        ld = vocab
    if (step != 1 and vocab > 1) or ld < vocab:
        raise MedusaError(-2, "logits: a row's logits must lie side by side, and rows must not overlap")
    n, f32 = (-(-rows // rows_per_setting),), torch.float32
    _check(lib().medusa_sample(
        dtype, logits.data_ptr(), ld, rows, vocab, _operand("temperature", temperature, n, f32, gpu), _operand("top_k", top_k, n, torch.int32, gpu),
        _operand("top_p", top_p, n, f32, gpu), _operand("min_p", min_p, n, f32, gpu), rows_per_setting, _operand("u", u, (rows,), f32, gpu),
        _operand("token", token, (rows,), torch.int32, gpu), _operand("prob", prob, (rows,), f32, gpu),
        None if ws is None else _whole("ws", ws, gpu), 0 if ws is None else ws.nbytes, _stream_of(gpu, stream)))


def medusa_kv_bytes(kv: KvDesc) -> int:
    return _check(lib().medusa_kv_bytes(C.byref(kv)))


def medusa_kv_init(kv: KvDesc, stream=None) -> None:
    _check(lib().medusa_kv_init(C.byref(kv), _stream(stream)))


def medusa_test_force_unfused_rope(on: bool) -> bool:
    """Test hook (include/medusa_bench.h): returns the previous setting."""
    return bool(lib().medusa_test_force_unfused_rope(1 if on else 0))


MDZ_STATUS_SEQ_RANGE = 1


def medusa_kv_write(kv: KvDesc, layer: int, seq: int, pos0: int, n: int, k_rows, v_rows, stream=None) -> None:
    _check(lib().medusa_kv_write(C.byref(kv), layer, seq, pos0, n, _ptr(k_rows), _ptr(v_rows), _stream(stream)))


def medusa_kv_read(kv: KvDesc, layer: int, seq: int, pos0: int, n: int, k_rows, v_rows, stream=None) -> None:
    _check(lib().medusa_kv_read(C.byref(kv), layer, seq, pos0, n, _ptr(k_rows), _ptr(v_rows), _stream(stream)))


def medusa_workspace_bytes(model: ModelDesc, B: int, max_prefix: int) -> int:
    return _check(lib().medusa_workspace_bytes(C.byref(model), B, max_prefix))


# ---------------------------------------------------------------------------------------------
# the hot path
# ---------------------------------------------------------------------------------------------

def medusa_heads(model: ModelDesc, w: Weights, hidden, src_row, root_token, B: int, Tsrc: int, cand_flat, tree_tokens,
                 head_logits_opt, ws, stream=None) -> None:
    _check(lib().medusa_heads(C.byref(model), C.byref(w), _ptr(hidden), _ptr(src_row), _ptr(root_token), B, Tsrc,
                              _ptr(cand_flat), _ptr(tree_tokens), _ptr(head_logits_opt), _ptr(ws), ws.numel(),
                              _stream(stream)))


def tree_verify_layer(model: ModelDesc, lw: LayerWeights, layer: int, x_inout, kv: KvDesc, seq_len, B: int,
                      max_prefix: int, ws, stream=None) -> None:
    _check(lib().tree_verify_layer(C.byref(model), C.byref(lw), layer, _ptr(x_inout), C.byref(kv), _ptr(seq_len), B,
                                   max_prefix, _ptr(ws), ws.numel(), _stream(stream)))


def tree_verify_layer_static_scratch_bytes() -> int:
    return int(lib().tree_verify_layer_static_scratch_bytes())


def tree_verify_layer_static(model: ModelDesc, lw: LayerWeights, layer: int, x_inout, kv: KvDesc, seq_len, B: int,
                             max_prefix: int, stream=None) -> None:
    _check(lib().tree_verify_layer_static(C.byref(model), C.byref(lw), layer, _ptr(x_inout), C.byref(kv), _ptr(seq_len),
                                          B, max_prefix, _stream(stream)))


def tree_verify_step(model: ModelDesc, w: Weights, tree_tokens, kv: KvDesc, seq_len, B: int, max_prefix: int,
                     node_argmax, hidden_out, logits_opt, ws, stream=None) -> None:
    _check(lib().tree_verify_step(C.byref(model), C.byref(w), _ptr(tree_tokens), C.byref(kv), _ptr(seq_len), B,
                                  max_prefix, _ptr(node_argmax), _ptr(hidden_out), _ptr(logits_opt), _ptr(ws),
                                  ws.numel(), _stream(stream)))


def accept_longest_prefix(tree: int, tree_tokens, node_argmax, B: int, accept_len, best_path, acc_nodes, acc_tokens,
                          next_root, last_node, stream=None) -> None:
    _check(lib().accept_longest_prefix(tree, _ptr(tree_tokens), _ptr(node_argmax), B, _ptr(accept_len),
                                       _ptr(best_path), _ptr(acc_nodes), _ptr(acc_tokens), _ptr(next_root),
                                       _ptr(last_node), _stream(stream)))


def kv_compact(kv: KvDesc, tree: int, acc_nodes, accept_len, seq_len_inout, kv_src_slots, B: int, max_prefix: int,
               stream=None) -> None:
    _check(lib().kv_compact(C.byref(kv), tree, _ptr(acc_nodes), _ptr(accept_len), _ptr(seq_len_inout),
                            _ptr(kv_src_slots), B, max_prefix, _stream(stream)))
