"""ctypes binding of ``libepd_encode.so`` -- argument marshalling only.

The functions below carry the same names and arguments as the C ABI in
``include/epd_encode.h`` (V_m = E(I_m), paper section 3.1, Eq. 1).  PyTorch is used for
device memory and streams and nothing else: every step of the encoder runs in the HIP
library.  There is no fallback: if the library cannot be loaded, importing this module
raises.
"""

from __future__ import annotations

import ctypes as C
from typing import Dict, Iterable, Optional, Sequence

import numpy as np
import torch

from . import build as _build

EPD_OK, EPD_ERR_INVALID_ARG, EPD_ERR_UNSUPPORTED, EPD_ERR_SHAPE, EPD_ERR_WORKSPACE, EPD_ERR_HIP = 0, -1, -2, -3, -4, -5
EPD_MISS = 1
EPD_F32, EPD_BF16 = 0, 1
EPD_LAYERNORM, EPD_RMSNORM = 0, 1
EPD_GELU_ERF, EPD_GELU_TANH, EPD_SWIGLU, EPD_GEGLU_ERF, EPD_GEGLU_TANH = 0, 1, 2, 3, 4
_GATED = {"swiglu": EPD_SWIGLU, "geglu_erf": EPD_GEGLU_ERF, "geglu_tanh": EPD_GEGLU_TANH}
_ACTS = {"gelu_erf": EPD_GELU_ERF, "gelu_tanh": EPD_GELU_TANH, **_GATED}
EPD_ROPE_NONE, EPD_ROPE_2D, EPD_ROPE_3D = 0, 2, 3
EPD_ROPE_SECTIONS, EPD_ROPE_INTERLEAVED = 0, 1
EPD_ROPE_LADDER_AXIS, EPD_ROPE_LADDER_HEAD = 0, 1
EPD_ROPE_HALF, EPD_ROPE_ADJACENT = 0, 1
(EPD_STEP_PLAN, EPD_STEP_PATCH_EMBED, EPD_STEP_NORM, EPD_STEP_QKV, EPD_STEP_ATTN, EPD_STEP_PROJ,
 EPD_STEP_FC1, EPD_STEP_FC2, EPD_STEP_MERGE, EPD_STEP_COUNT) = range(10)
STEP_NAMES = ["plan", "patch_embed", "norm", "qkv", "attn", "proj", "fc1", "fc2", "merge"]

_LAYER_FIELDS = ["norm1_g", "norm1_b", "qkv_w", "qkv_b", "proj_w", "proj_b",
                 "norm2_g", "norm2_b", "fc1_w", "fc1_b", "fc2_w", "fc2_b"]


class epd_layer_weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in _LAYER_FIELDS]


class epd_weights(C.Structure):
    _fields_ = [("patch_w", C.c_void_p), ("patch_b", C.c_void_p),
                ("layers", C.POINTER(epd_layer_weights)),
                ("final_norm_g", C.c_void_p), ("final_norm_b", C.c_void_p),
                ("merge_w", C.c_void_p), ("merge_b", C.c_void_p)]


class epd_encode_cfg(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int32), ("num_layers", C.c_int32),
                ("hidden", C.c_int32), ("num_heads", C.c_int32), ("head_dim", C.c_int32),
                ("mlp_dim", C.c_int32), ("in_channels", C.c_int32), ("patch", C.c_int32),
                ("temporal_patch", C.c_int32), ("norm", C.c_int32), ("norm_eps", C.c_float),
                ("act", C.c_int32), ("use_bias", C.c_int32), ("rope", C.c_int32),
                ("rope_base", C.c_float), ("rope_pairs", C.c_int32 * 3), ("final_norm", C.c_int32),
                ("merge", C.c_int32), ("out_dim", C.c_int32), ("max_tokens", C.c_int32),
                ("max_segments", C.c_int32), ("max_items", C.c_int32),
                ("weights", C.POINTER(epd_weights)), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_uint64)]


class epd_rope_cfg(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int32), ("head_dim", C.c_int32), ("axes", C.c_int32),
                ("pairs", C.c_int32 * 4), ("layout", C.c_int32), ("ladder", C.c_int32), ("pairing", C.c_int32),
                ("base", C.c_double)]


class epd_rope_tensor(C.Structure):
    _fields_ = [("input", C.c_void_p), ("output", C.c_void_p), ("in_token", C.c_int64), ("in_head", C.c_int64),   # C names: in, out
                ("out_token", C.c_int64), ("out_head", C.c_int64), ("heads", C.c_int32)]


class epd_gated_mlp_cfg(C.Structure):
    _fields_ = [(n, C.c_uint32 if n == "struct_size" else C.c_int32)
                for n in ("struct_size", "dtype", "hidden", "mlp_dim", "act", "use_bias", "max_tokens", "training")]


_GATED_FIELDS = ["gate_up_w", "gate_up_b", "down_w", "down_b"]


class epd_gated_mlp_weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in _GATED_FIELDS]


class epd_gated_mlp_grads(C.Structure):
    _fields_ = [("dx", C.c_void_p), ("ld_dx", C.c_int64)] + [(n, C.c_void_p) for n in _GATED_FIELDS]


class epd_embed_cfg(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int32), ("out_dtype", C.c_int32), ("vocab", C.c_int32), ("hidden", C.c_int32),
                ("max_tokens", C.c_int32), ("scale", C.c_float)]


class epd_add_norm_cfg(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int32), ("residual_dtype", C.c_int32), ("hidden", C.c_int32), ("max_tokens", C.c_int32),
                ("eps", C.c_float)]


class epd_add_norm_rows(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("x", "residual", "sum", "y", "q", "scale")] +
                [(n, C.c_int64) for n in ("ld_x", "ld_residual", "ld_sum", "ld_y", "ld_q")])


class epd_add_norm_grads(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("sum", "dy", "dsum", "dx", "dresidual", "gain")] +
                [(n, C.c_int64) for n in ("ld_sum", "ld_dy", "ld_dsum", "ld_dx", "ld_dresidual")])


class epd_int8_linear_cfg(C.Structure):
    _fields_ = [(n, C.c_uint32 if n == "struct_size" else C.c_int32)
                for n in ("struct_size", "in_features", "out_features", "out_dtype", "use_bias", "max_tokens")]


class epd_int8_linear_weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("w", "scale", "bias")]


EXPORTS = ["epd_encode_workspace_bytes", "epd_encode_create", "epd_encode", "epd_encode_destroy",
           "epd_encode_last_error", "epd_encode_debug_hidden", "epd_encode_set_timing", "epd_encode_set_tuning", "epd_encode_set_compute_units",
           "epd_encode_get_timing", "epd_preprocess", "epd_encode_cached", "epd_store_create",
           "epd_store_destroy", "epd_store_last_error", "epd_store_hash", "epd_store_hash_noalloc", "epd_store_lookup", "epd_store_insert",
           "epd_store_stats", "epd_probe_stream_read", "epd_probe_mfma_rate", "epd_probe_gemm_plan"]
OPERATOR_EXPORTS = ["epd_op_last_error", "epd_rope_apply", "epd_rope_tokens", "epd_rope_positions", "epd_gated_mlp_workspace_bytes", "epd_gated_mlp_saved_bytes",
                    "epd_gated_mlp", "epd_gated_mlp_backward"]    # the operators beside the encoder

ENTRY_EXPORTS = ["epd_embed", "epd_embed_workspace_bytes", "epd_embed_backward", "epd_add_norm", "epd_add_norm_workspace_bytes", "epd_add_norm_backward",
                 "epd_quant_rows", "epd_dequant_rows", "epd_int8_linear_workspace_bytes", "epd_int8_linear"]    # those at the entry of the next stage


def _load() -> C.CDLL:
    lib = C.CDLL(_build.library_path())
    lib.epd_encode_workspace_bytes.restype = C.c_uint64
    lib.epd_encode_workspace_bytes.argtypes = [C.POINTER(epd_encode_cfg)]
    lib.epd_encode_create.restype = C.c_int
    lib.epd_encode_create.argtypes = [C.POINTER(epd_encode_cfg), C.POINTER(C.c_void_p)]
    lib.epd_encode.restype = C.c_int
    lib.epd_encode.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(C.c_int32), C.c_int32,
                               C.POINTER(C.c_int32), C.c_int32, C.c_void_p, C.c_void_p]
    lib.epd_encode_destroy.restype = C.c_int
    lib.epd_encode_destroy.argtypes = [C.c_void_p]
    U64P, I32P, F32P = C.POINTER(C.c_uint64), C.POINTER(C.c_int32), C.POINTER(C.c_float)
    lib.epd_store_create.restype = C.c_int
    lib.epd_store_create.argtypes = [C.c_void_p, C.c_uint64, C.POINTER(C.c_void_p)]
    lib.epd_store_destroy.restype = C.c_int
    lib.epd_store_destroy.argtypes = [C.c_void_p]
    lib.epd_store_last_error.restype = C.c_char_p
    lib.epd_store_last_error.argtypes = [C.c_void_p]
    lib.epd_store_hash.restype = C.c_int
    lib.epd_store_hash.argtypes = [C.c_void_p, C.c_void_p, U64P, U64P, C.c_int32, U64P, C.c_void_p]
    lib.epd_store_hash_noalloc.restype = C.c_int
    lib.epd_store_hash_noalloc.argtypes = [C.c_void_p, U64P, U64P, C.c_int32, C.c_void_p, C.c_void_p]
    lib.epd_store_lookup.restype = C.c_int
    lib.epd_store_lookup.argtypes = [C.c_void_p, U64P, C.POINTER(C.c_void_p), U64P]
    lib.epd_store_insert.restype = C.c_int
    lib.epd_store_insert.argtypes = [C.c_void_p, U64P, C.c_uint64, C.POINTER(C.c_void_p)]
    lib.epd_store_stats.restype = C.c_int
    lib.epd_store_stats.argtypes = [C.c_void_p, U64P, U64P, U64P, U64P]
    lib.epd_encode_cached.restype = C.c_int
    lib.epd_encode_cached.argtypes = [C.c_void_p, C.c_void_p, C.c_uint64, C.c_void_p, I32P, I32P, C.c_int32, F32P, F32P,
                                      C.c_void_p, C.c_void_p, C.c_void_p, I32P, U64P, C.c_void_p]
    lib.epd_preprocess.restype = C.c_int
    lib.epd_preprocess.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(C.c_int32), C.POINTER(C.c_int32), C.c_int32,
                                   C.POINTER(C.c_float), C.POINTER(C.c_float), C.c_void_p, C.c_void_p]
    lib.epd_encode_last_error.restype = C.c_char_p
    lib.epd_encode_last_error.argtypes = [C.c_void_p]
    lib.epd_encode_debug_hidden.restype = C.c_int
    lib.epd_encode_debug_hidden.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p]
    lib.epd_encode_set_timing.restype = C.c_int
    lib.epd_encode_set_timing.argtypes = [C.c_void_p, C.c_int32]
    lib.epd_encode_set_compute_units.restype = C.c_int
    lib.epd_encode_set_compute_units.argtypes = [C.c_void_p, C.c_int32]
    lib.epd_probe_stream_read.restype = C.c_int
    lib.epd_probe_stream_read.argtypes = [C.c_void_p, C.c_uint64, C.c_void_p, C.c_int32, C.c_void_p]
    lib.epd_probe_mfma_rate.restype = C.c_int
    lib.epd_probe_mfma_rate.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.POINTER(C.c_double), C.c_void_p]
    lib.epd_probe_gemm_plan.restype = C.c_int
    lib.epd_probe_gemm_plan.argtypes = [C.c_int32] * 6 + [C.POINTER(C.c_int32)] * 3
    lib.epd_encode_set_tuning.restype = C.c_int
    lib.epd_encode_set_tuning.argtypes = [C.c_void_p, C.c_int32, C.c_int32]
    lib.epd_encode_get_timing.restype = C.c_int
    lib.epd_encode_get_timing.argtypes = [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_int64),
                                          C.POINTER(C.c_double)]
    lib.epd_op_last_error.restype = C.c_char_p
    lib.epd_op_last_error.argtypes = []
    lib.epd_rope_apply.restype = C.c_int
    lib.epd_rope_apply.argtypes = [C.POINTER(epd_rope_cfg), C.POINTER(epd_rope_tensor), C.c_int32, C.c_void_p, C.c_int64,
                                   C.c_int32, C.c_int32, C.c_void_p]
    lib.epd_rope_tokens.restype = C.c_int64
    lib.epd_rope_tokens.argtypes = [C.c_void_p, C.c_int32]
    lib.epd_rope_positions.restype = C.c_int
    lib.epd_rope_positions.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p, C.c_int64,
                                       C.c_void_p, C.c_void_p]
    lib.epd_gated_mlp_workspace_bytes.restype = C.c_uint64
    lib.epd_gated_mlp_workspace_bytes.argtypes = [C.POINTER(epd_gated_mlp_cfg)]
    lib.epd_gated_mlp_saved_bytes.restype = C.c_uint64
    lib.epd_gated_mlp_saved_bytes.argtypes = [C.POINTER(epd_gated_mlp_cfg), C.c_int32]
    lib.epd_gated_mlp.restype = C.c_int
    lib.epd_gated_mlp.argtypes = [C.POINTER(epd_gated_mlp_cfg), C.POINTER(epd_gated_mlp_weights), C.c_void_p, C.c_int64, C.c_int32, C.c_void_p,
                                  C.c_int64, C.c_void_p, C.c_void_p, C.c_uint64, C.c_void_p]
    lib.epd_gated_mlp_backward.restype = C.c_int
    lib.epd_gated_mlp_backward.argtypes = [C.POINTER(epd_gated_mlp_cfg), C.POINTER(epd_gated_mlp_weights), C.c_void_p, C.c_int64, C.c_void_p,
                                           C.c_int64, C.c_int32, C.c_void_p, C.POINTER(epd_gated_mlp_grads), C.c_void_p, C.c_uint64, C.c_void_p]
    V, I32, I64, U64 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64
    for name, cfg in (("embed", epd_embed_cfg), ("add_norm", epd_add_norm_cfg), ("int8_linear", epd_int8_linear_cfg)):
        f = getattr(lib, "epd_%s_workspace_bytes" % name)
        f.restype, f.argtypes = U64, [C.POINTER(cfg)]
    for name, args in {"epd_embed": [C.POINTER(epd_embed_cfg), V, V, I32, V, I32, V, I64, V],
                       "epd_embed_backward": [C.POINTER(epd_embed_cfg), V, I32, V, I64, I32, V, V, V, U64, V],
                       "epd_add_norm": [C.POINTER(epd_add_norm_cfg), C.POINTER(epd_add_norm_rows), V, I32, V],
                       "epd_add_norm_backward": [C.POINTER(epd_add_norm_cfg), C.POINTER(epd_add_norm_grads), V, I32, V, U64, V],
                       "epd_quant_rows": [I32, V, I64, I32, I32, V, I64, V, V],
                       "epd_dequant_rows": [V, I64, V, I32, I32, I32, V, I64, V],
                       "epd_int8_linear": [C.POINTER(epd_int8_linear_cfg), C.POINTER(epd_int8_linear_weights), V, I64, V, I32, V, I64, V, U64, V]}.items():
        f = getattr(lib, name)
        f.restype, f.argtypes = C.c_int, args
    return lib


lib = _load()


class EpdError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("epd status %d: %s" % (status, message))
        self.status = status


# ---------------------------------------------------------------- same-name wrappers

def epd_encode_workspace_bytes(cfg: epd_encode_cfg) -> int:
    return int(lib.epd_encode_workspace_bytes(C.byref(cfg)))


def epd_encode_last_error(handle: Optional[int]) -> str:
    return lib.epd_encode_last_error(handle).decode()


def epd_encode_create(cfg: epd_encode_cfg) -> int:
    h = C.c_void_p()
    st = lib.epd_encode_create(C.byref(cfg), C.byref(h))
    if st != EPD_OK:
        raise EpdError(st, epd_encode_last_error(None))
    return h.value


def epd_encode(handle, packed_patches: int, cu_seqlens: np.ndarray, grid_thw: np.ndarray,
               out_visual_tokens: int, stream: int) -> None:
    cu = np.ascontiguousarray(cu_seqlens, dtype=np.int32)
    grid = np.ascontiguousarray(grid_thw, dtype=np.int32).reshape(-1, 3)
    st = lib.epd_encode(handle, packed_patches, cu.ctypes.data_as(C.POINTER(C.c_int32)), len(cu) - 1,
                        grid.ctypes.data_as(C.POINTER(C.c_int32)), grid.shape[0], out_visual_tokens, stream)
    if st != EPD_OK:
        raise EpdError(st, epd_encode_last_error(handle))


def epd_preprocess(handle, pixels: int, src_hw: np.ndarray, grid_thw: np.ndarray, mean, std,
                   packed_patches: int, stream: int) -> None:
    src = np.ascontiguousarray(src_hw, dtype=np.int32).reshape(-1, 2)
    grid = np.ascontiguousarray(grid_thw, dtype=np.int32).reshape(-1, 3)
    mu = np.ascontiguousarray(mean, dtype=np.float32)
    sd = np.ascontiguousarray(std, dtype=np.float32)
    st = lib.epd_preprocess(handle, pixels, src.ctypes.data_as(C.POINTER(C.c_int32)),
                            grid.ctypes.data_as(C.POINTER(C.c_int32)), grid.shape[0],
                            mu.ctypes.data_as(C.POINTER(C.c_float)), sd.ctypes.data_as(C.POINTER(C.c_float)),
                            packed_patches, stream)
    if st != EPD_OK:
        raise EpdError(st, epd_encode_last_error(handle))


class StoreError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("epd store status %d: %s" % (status, message))
        self.status = status


def epd_store_last_error(store: Optional[int]) -> str:
    return lib.epd_store_last_error(store).decode()


def epd_store_create(pool_ptr: int, pool_bytes: int) -> int:
    s = C.c_void_p()
    st = lib.epd_store_create(pool_ptr, pool_bytes, C.byref(s))
    if st != EPD_OK:
        raise StoreError(st, epd_store_last_error(None))
    return s.value


def epd_store_destroy(store) -> None:
    lib.epd_store_destroy(store)


def _key(key):
    return (C.c_uint64 * 2)(int(key[0]), int(key[1]))


def epd_store_lookup(store, key):
    """(device pointer, bytes) of a stored value, or None."""
    p, n = C.c_void_p(), C.c_uint64()
    st = lib.epd_store_lookup(store, _key(key), C.byref(p), C.byref(n))
    if st == EPD_MISS:
        return None
    if st != EPD_OK:
        raise StoreError(st, epd_store_last_error(store))
    return p.value, n.value


def epd_store_insert(store, key, nbytes: int) -> int:
    p = C.c_void_p()
    st = lib.epd_store_insert(store, _key(key), nbytes, C.byref(p))
    if st != EPD_OK:
        raise StoreError(st, epd_store_last_error(store))
    return p.value


def epd_store_stats(store):
    v = [C.c_uint64() for _ in range(4)]
    st = lib.epd_store_stats(store, *[C.byref(x) for x in v])
    if st != EPD_OK:
        raise StoreError(st, epd_store_last_error(store))
    return dict(zip(("hits", "misses", "evictions", "entries"), (x.value for x in v)))


def epd_store_hash(store, data_ptr: int, offsets, salts, stream: int) -> np.ndarray:
    """uint64 [n, 2] keys of the byte ranges [offsets[i], offsets[i+1]) of one device buffer."""
    off = np.ascontiguousarray(offsets, dtype=np.uint64)
    sa = np.ascontiguousarray(salts, dtype=np.uint64)
    n = len(sa)
    assert len(off) == n + 1
    keys = np.zeros((n, 2), dtype=np.uint64)
    U64P = C.POINTER(C.c_uint64)
    st = lib.epd_store_hash(store, data_ptr, off.ctypes.data_as(U64P), sa.ctypes.data_as(U64P), n,
                            keys.ctypes.data_as(U64P), stream)
    if st != EPD_OK:
        raise StoreError(st, epd_store_last_error(store))
    return keys


def epd_store_hash_noalloc(data_ptr: int, offsets, salts, keys_device_ptr: int, stream: int) -> None:
    """Keys of the byte ranges into a device buffer uint64 [n, 2]; enqueues only (no wait)."""
    off = np.ascontiguousarray(offsets, dtype=np.uint64)
    sa = np.ascontiguousarray(salts, dtype=np.uint64)
    assert len(off) == len(sa) + 1
    U64P = C.POINTER(C.c_uint64)
    st = lib.epd_store_hash_noalloc(data_ptr, off.ctypes.data_as(U64P), sa.ctypes.data_as(U64P), len(sa), keys_device_ptr, stream)
    if st != EPD_OK:
        raise StoreError(st, epd_store_last_error(None))


def epd_encode_cached(handle, store, model_salt: int, pixels: int, src_hw, grid_thw, mean, std, rows_scratch: int,
                      out_scratch: int, out_visual_tokens: int, stream: int):
    """Returns (hit flags int32 [items], keys uint64 [items, 2])."""
    src = np.ascontiguousarray(src_hw, dtype=np.int32).reshape(-1, 2)
    grid = np.ascontiguousarray(grid_thw, dtype=np.int32).reshape(-1, 3)
    mu = np.ascontiguousarray(mean, dtype=np.float32)
    sd = np.ascontiguousarray(std, dtype=np.float32)
    hit = np.zeros(grid.shape[0], dtype=np.int32)
    keys = np.zeros((grid.shape[0], 2), dtype=np.uint64)
    I32P, F32P, U64P = C.POINTER(C.c_int32), C.POINTER(C.c_float), C.POINTER(C.c_uint64)
    st = lib.epd_encode_cached(handle, store, model_salt, pixels, src.ctypes.data_as(I32P), grid.ctypes.data_as(I32P),
                               grid.shape[0], mu.ctypes.data_as(F32P), sd.ctypes.data_as(F32P), rows_scratch, out_scratch,
                               out_visual_tokens, hit.ctypes.data_as(I32P), keys.ctypes.data_as(U64P), stream)
    if st != EPD_OK:
        raise EpdError(st, epd_encode_last_error(handle))
    return hit, keys


def epd_encode_destroy(handle) -> None:
    lib.epd_encode_destroy(handle)


def epd_encode_debug_hidden(handle, out_ptr: int, stream: int) -> None:
    st = lib.epd_encode_debug_hidden(handle, out_ptr, stream)
    if st != EPD_OK:
        raise EpdError(st, epd_encode_last_error(handle))


def epd_encode_set_timing(handle, step: int) -> None:
    st = lib.epd_encode_set_timing(handle, step)
    if st != EPD_OK:
        raise EpdError(st, epd_encode_last_error(handle))


def epd_encode_set_tuning(handle, gemm_tile: int, attn_groups: int) -> None:
    st = lib.epd_encode_set_tuning(handle, gemm_tile, attn_groups)
    if st != EPD_OK:
        raise EpdError(st, epd_encode_last_error(handle))


def epd_encode_set_compute_units(handle, compute_units: int) -> None:
    st = lib.epd_encode_set_compute_units(handle, compute_units)
    if st != EPD_OK:
        raise EpdError(st, epd_encode_last_error(handle))


def epd_probe_stream_read(buf_ptr: int, nbytes: int, out_ptr: int, blocks: int, stream: int) -> None:
    st = lib.epd_probe_stream_read(buf_ptr, nbytes, out_ptr, blocks, stream)
    if st != EPD_OK:
        raise EpdError(st, "epd_probe_stream_read: bad argument or launch failure")


def epd_probe_mfma_rate(shape: int, zero_operands: bool, iters: int, out_ptr: int, stream: int) -> float:
    """Enqueue one launch of the matrix-core rate probe; returns the flops it executes."""
    fl = C.c_double()
    st = lib.epd_probe_mfma_rate(shape, 1 if zero_operands else 0, iters, out_ptr, C.byref(fl), stream)
    if st != EPD_OK:
        raise EpdError(st, "epd_probe_mfma_rate: bad argument or launch failure")
    return fl.value


def epd_encode_get_timing(handle):
    ms, n, work = C.c_double(), C.c_int64(), C.c_double()
    st = lib.epd_encode_get_timing(handle, C.byref(ms), C.byref(n), C.byref(work))
    if st != EPD_OK:
        raise EpdError(st, epd_encode_last_error(handle))
    return ms.value, n.value, work.value


# ---------------------------------------------------------------- config marshalling

def make_cfg(cfg, max_tokens: int, max_segments: int, max_items: int) -> epd_encode_cfg:
    """Fill the C config struct from an object with the attribute names of
    ``workloads.EncoderConfig`` (shape fields only; weights / workspace are left empty)."""
    c = epd_encode_cfg()
    c.struct_size = C.sizeof(epd_encode_cfg)
    c.dtype = {"f32": EPD_F32, "bf16": EPD_BF16}[cfg.dtype]
    c.num_layers, c.hidden, c.num_heads, c.head_dim = cfg.num_layers, cfg.hidden, cfg.num_heads, cfg.head_dim
    c.mlp_dim, c.in_channels, c.patch, c.temporal_patch = cfg.mlp_dim, cfg.in_channels, cfg.patch, cfg.temporal_patch
    c.norm = {"layernorm": EPD_LAYERNORM, "rmsnorm": EPD_RMSNORM}[cfg.norm]
    c.norm_eps = cfg.norm_eps
    c.act = _ACTS[cfg.act]
    c.use_bias = 1 if cfg.use_bias else 0
    c.rope = {"none": EPD_ROPE_NONE, "2d": EPD_ROPE_2D, "3d": EPD_ROPE_3D}[cfg.rope]
    c.rope_base = cfg.rope_base
    c.rope_pairs = (C.c_int32 * 3)(*cfg.rope_pairs)
    c.final_norm = 1 if cfg.final_norm else 0
    c.merge, c.out_dim = cfg.merge, cfg.out_dim
    c.max_tokens, c.max_segments, c.max_items = max_tokens, max_segments, max_items
    return c


def torch_dtype(name: str) -> torch.dtype:
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


class EpdEncoder:
    """Owns the device tensors (weights during create, the workspace) and the handle."""

    def __init__(self, cfg, global_weights: Dict[str, np.ndarray], layers: Iterable[Dict[str, np.ndarray]],
                 max_tokens: int, max_segments: int = 64, max_items: int = 64, device: str = "cuda:0"):
        self.cfg = cfg
        self.device = torch.device(device)
        self.dtype = torch_dtype(cfg.dtype)
        self.handle = None
        ccfg = make_cfg(cfg, max_tokens, max_segments, max_items)
        need = epd_encode_workspace_bytes(ccfg)
        if need == 0:
            # let create produce the precise message
            ccfg.weights = C.pointer(epd_weights())
            ccfg.workspace = 256
            epd_encode_create(ccfg)
            raise EpdError(EPD_ERR_INVALID_ARG, "invalid configuration")
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(self.device).to(self.dtype).contiguous()
        gw = {k: up(v) for k, v in global_weights.items()}
        lws = [{k: up(v) for k, v in lw.items()} for lw in layers]
        if len(lws) != cfg.num_layers:
            raise ValueError("expected %d layers, got %d" % (cfg.num_layers, len(lws)))
        ptr = lambda d, k: d[k].data_ptr() if k in d else None
        arr = (epd_layer_weights * max(1, len(lws)))()
        for i, lw in enumerate(lws):
            for f in _LAYER_FIELDS:
                setattr(arr[i], f, ptr(lw, f))
        w = epd_weights()
        w.patch_w, w.patch_b = ptr(gw, "patch_w"), ptr(gw, "patch_b")
        w.layers = C.cast(arr, C.POINTER(epd_layer_weights))
        w.final_norm_g, w.final_norm_b = ptr(gw, "final_norm_g"), ptr(gw, "final_norm_b")
        w.merge_w, w.merge_b = ptr(gw, "merge_w"), ptr(gw, "merge_b")
        self.workspace = torch.empty(need + 256, dtype=torch.uint8, device=self.device)
        base = (self.workspace.data_ptr() + 255) // 256 * 256
        ccfg.weights = C.pointer(w)
        ccfg.workspace = base
        ccfg.workspace_bytes = need
        self.workspace_bytes = need
        torch.cuda.synchronize(self.device)
        with torch.cuda.device(self.device):
            self.handle = epd_encode_create(ccfg)
        del gw, lws   # the library holds its own copy inside the workspace

    def encode(self, patches: torch.Tensor, cu_seqlens, grid_thw, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """patches: device tensor [T, Pdim] of the configuration's dtype."""
        assert patches.is_cuda and patches.dtype == self.dtype and patches.is_contiguous()
        grid = np.ascontiguousarray(grid_thw, dtype=np.int32).reshape(-1, 3)
        m = self.cfg.merge
        tm = int(sum(int(t) * (int(h) // m) * (int(w) // m) for t, h, w in grid))
        if out is None:
            out = torch.empty((tm, self.cfg.out_dim), dtype=self.dtype, device=self.device)
        assert out.is_cuda and out.dtype == self.dtype and out.is_contiguous() and out.numel() >= tm * self.cfg.out_dim
        with torch.cuda.device(self.device):
            stream = torch.cuda.current_stream(self.device).cuda_stream
            epd_encode(self.handle, patches.data_ptr(), cu_seqlens, grid, out.data_ptr(), stream)
        self._last_T = int(patches.shape[0])
        return out

    def preprocess(self, pixels: torch.Tensor, src_hw, grid_thw, mean, std,
                   out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """pixels: device uint8 tensor, items packed in order, each planar [C, t*tp, Hs, Ws].
        Returns the packed patch rows [T, Pdim] that ``encode`` takes."""
        assert pixels.is_cuda and pixels.dtype == torch.uint8 and pixels.is_contiguous()
        grid = np.ascontiguousarray(grid_thw, dtype=np.int32).reshape(-1, 3)
        src = np.ascontiguousarray(src_hw, dtype=np.int32).reshape(-1, 2)
        assert len(src) == len(grid) and len(mean) == len(std) == self.cfg.in_channels
        need = int(sum(self.cfg.in_channels * int(t) * self.cfg.temporal_patch * int(hs) * int(ws)
                       for (t, _, _), (hs, ws) in zip(grid, src)))
        assert pixels.numel() >= need, "pixel buffer shorter than the items described"
        T = int(sum(int(t) * int(h) * int(w) for t, h, w in grid))
        if out is None:
            out = torch.empty((T, self.cfg.patch_dim), dtype=self.dtype, device=self.device)
        assert out.is_cuda and out.dtype == self.dtype and out.is_contiguous() and out.numel() >= T * self.cfg.patch_dim
        with torch.cuda.device(self.device):
            stream = torch.cuda.current_stream(self.device).cuda_stream
            epd_preprocess(self.handle, pixels.data_ptr(), src, grid, mean, std, out.data_ptr(), stream)
        return out

    def encode_cached(self, store: "MMStore", model_salt: int, pixels: torch.Tensor, src_hw, grid_thw, mean, std,
                      out: Optional[torch.Tensor] = None):
        """Raw pixels -> visual tokens through the store.  Returns (out, hit flags, keys)."""
        assert pixels.is_cuda and pixels.dtype == torch.uint8 and pixels.is_contiguous()
        grid = np.ascontiguousarray(grid_thw, dtype=np.int32).reshape(-1, 3)
        src = np.ascontiguousarray(src_hw, dtype=np.int32).reshape(-1, 2)
        assert len(src) == len(grid)
        need = int(sum(self.cfg.in_channels * int(t) * self.cfg.temporal_patch * int(hs) * int(ws)
                       for (t, _, _), (hs, ws) in zip(grid, src)))
        assert pixels.numel() >= need, "pixel buffer shorter than the items described"
        m = self.cfg.merge
        T = int(sum(int(t) * int(h) * int(w) for t, h, w in grid))
        tm = int(sum(int(t) * (int(h) // m) * (int(w) // m) for t, h, w in grid))
        rows = torch.empty((max(T, 1), self.cfg.patch_dim), dtype=self.dtype, device=self.device)
        tmp = torch.empty((max(tm, 1), self.cfg.out_dim), dtype=self.dtype, device=self.device)
        if out is None:
            out = torch.empty((tm, self.cfg.out_dim), dtype=self.dtype, device=self.device)
        assert out.is_cuda and out.dtype == self.dtype and out.is_contiguous() and out.numel() >= tm * self.cfg.out_dim
        with torch.cuda.device(self.device):
            stream = torch.cuda.current_stream(self.device).cuda_stream
            hit, keys = epd_encode_cached(self.handle, store.handle, model_salt, pixels.data_ptr(), src, grid, mean, std,
                                          rows.data_ptr(), tmp.data_ptr(), out.data_ptr(), stream)
            # the scratch tensors are read by work queued on this stream: keep them until it is through
            rows.record_stream(torch.cuda.current_stream(self.device))
            tmp.record_stream(torch.cuda.current_stream(self.device))
        return out, hit, keys

    def hidden(self) -> torch.Tensor:
        """fp32 residual stream [T, D] of the last call (before the final norm)."""
        out = torch.empty((self._last_T, self.cfg.hidden), dtype=torch.float32, device=self.device)
        with torch.cuda.device(self.device):
            epd_encode_debug_hidden(self.handle, out.data_ptr(), torch.cuda.current_stream(self.device).cuda_stream)
        return out

    def set_timing(self, step: int) -> None:
        epd_encode_set_timing(self.handle, step)

    def get_timing(self):
        return epd_encode_get_timing(self.handle)

    def set_tuning(self, gemm_tile: int = -1, attn_groups: int = 0) -> None:
        epd_encode_set_tuning(self.handle, gemm_tile, attn_groups)

    def set_compute_units(self, compute_units: int = 0) -> None:
        epd_encode_set_compute_units(self.handle, compute_units)

    def close(self) -> None:
        if self.handle is not None:
            torch.cuda.synchronize(self.device)
            epd_encode_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class MMStore:
    """Device pool + the library's store handle (single-node stand-in for the paper's MM Store)."""

    def __init__(self, pool_bytes: int, device: str = "cuda:0"):
        self.device = torch.device(device)
        self.pool = torch.empty(pool_bytes + 256, dtype=torch.uint8, device=self.device)
        base = (self.pool.data_ptr() + 255) // 256 * 256
        self.base = base
        self.handle = epd_store_create(base, pool_bytes)

    def hash(self, data: torch.Tensor, offsets, salts) -> np.ndarray:
        assert data.is_cuda and data.dtype == torch.uint8 and data.is_contiguous()
        assert int(np.asarray(offsets)[-1]) <= data.numel()
        with torch.cuda.device(self.device):
            return epd_store_hash(self.handle, data.data_ptr(), offsets, salts, torch.cuda.current_stream(self.device).cuda_stream)

    def stats(self):
        return epd_store_stats(self.handle)

    def close(self) -> None:
        if self.handle is not None:
            torch.cuda.synchronize(self.device)
            epd_store_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def to_device_patches(patches_f32: np.ndarray, dtype: str, device: str = "cuda:0") -> torch.Tensor:
    """Host float32 rows (already rounded to ``dtype``) -> device tensor of that dtype."""
    return torch.from_numpy(np.ascontiguousarray(patches_f32)).to(device).to(torch_dtype(dtype)).contiguous()


# ---------------------------------------------------------------- operators beside the encoder

def epd_op_last_error() -> str:
    return lib.epd_op_last_error().decode()


def _op_check(status: int) -> None:
    if status != EPD_OK:
        raise EpdError(status, epd_op_last_error())


def epd_rope_apply(cfg: epd_rope_cfg, tensors, positions: int, position_stride: int, tokens: int, inverse: bool, stream: int) -> None:
    """tensors: a ctypes array of ``epd_rope_tensor``."""
    _op_check(lib.epd_rope_apply(C.byref(cfg), tensors, len(tensors), positions, position_stride, tokens, 1 if inverse else 0, stream))


def epd_rope_tokens(span_thw: np.ndarray) -> int:
    """Tokens of all spans."""
    span = _int32(span_thw, "span_thw").reshape(-1, 3)
    tokens = lib.epd_rope_tokens(_address(span), len(span))
    if tokens < 0:
        raise EpdError(EPD_ERR_SHAPE, epd_op_last_error())
    return tokens


def epd_rope_positions(span_thw: np.ndarray, cu_spans: np.ndarray, start: Optional[np.ndarray], t_step: int, positions: int,
                       position_stride: int, stream: int) -> np.ndarray:
    """Returns the next position of every sequence, int32 [num_sequences]."""
    return _positions(*_spans(span_thw, cu_spans), start, t_step, positions, position_stride, stream)


def _positions(span: np.ndarray, cu: np.ndarray, start, t_step: int, positions: int, position_stride: int, stream: int) -> np.ndarray:
    n = len(cu) - 1
    if not -1 << 31 <= t_step < 1 << 31:
        raise ValueError("t_step must be an int32")
    if start is not None:
        start = _int32(start, "start")
        if start.shape != (n,):
            raise ValueError("start must be [num_sequences]")
    after = np.empty(n, dtype=np.int32)
    _op_check(lib.epd_rope_positions(_address(span), _address(cu), n, None if start is None else _address(start), t_step, positions, position_stride,
                                     _address(after), stream))
    return after


def _address(a: np.ndarray) -> int:
    return a.__array_interface__["data"][0]       # (a.ctypes.data makes an object for it)


def _int32(a, name: str) -> np.ndarray:
    """``a`` as a contiguous int32 array: itself where it is one, else its values, which have to be such."""
    if type(a) is np.ndarray and a.dtype == np.int32 and a.flags.c_contiguous:
        return a
    a = np.asarray(a)
    if a.size and a.dtype != np.int32:
        lo, hi = a.min(), a.max()
        if not (lo >= -2 ** 31 and hi < 2 ** 31) or (a.dtype.kind not in "iu" and not (a == np.trunc(a)).all()):
            raise ValueError("%s must hold 32-bit integers" % name)
    return np.ascontiguousarray(a, dtype=np.int32)


def _spans(span_thw, cu_spans):
    # (what is right already is not passed through _int32: two calls cost a plan 0.4 us of 11)
    if type(span_thw) is not np.ndarray or span_thw.dtype != np.int32 or span_thw.ndim != 2 or span_thw.shape[1] != 3 or not span_thw.flags.c_contiguous:
        span_thw = _int32(span_thw, "span_thw").reshape(-1, 3)
    if type(cu_spans) is not np.ndarray or cu_spans.dtype != np.int32 or not cu_spans.flags.c_contiguous:
        cu_spans = _int32(cu_spans, "cu_spans")
    if cu_spans.ndim != 1 or len(cu_spans) < 1 or int(cu_spans[-1]) > len(span_thw):      # the library refuses cu_spans that decrease
        raise ValueError("cu_spans must be [num_sequences + 1] and end within the spans")
    return span_thw, cu_spans


def _on(index: int, call, *args):
    """call(*args, stream) with the device's current stream, the device made the current one around it where it is not.
    (The raw stream, where this torch has it: the objects of torch.cuda cost a call for one token a third of its time.)"""
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    stream = raw(index) if raw is not None else torch.cuda.current_stream(index).cuda_stream
    if torch.cuda.current_device() == index:
        return call(*args, stream)
    with torch.cuda.device(index):
        return call(*args, stream)


def rope_positions(span_thw, cu_spans, start=None, t_step: int = 1, device: str = "cuda:0", out: Optional[torch.Tensor] = None):
    """(t, h, w) positions of sequences of texts (n, 0, 0) and items (t, h, w), sequence s being the spans
    [cu_spans[s], cu_spans[s + 1]) and starting at start[s].  Returns (int32 device tensor [3, tokens], next position of every
    sequence int32 [sequences])."""
    span, cu = _spans(span_thw, cu_spans)
    tokens = lib.epd_rope_tokens(_address(span), int(cu[-1]))
    if tokens < 0:
        raise EpdError(EPD_ERR_SHAPE, epd_op_last_error())
    dev = torch.device(device) if out is None else out.device
    if dev.index is None:
        dev = torch.device(dev.type, torch.cuda.current_device())
    if out is None:
        out = torch.empty((3, tokens), dtype=torch.int32, device=dev)
    if not out.is_cuda or out.dtype != torch.int32 or out.dim() != 2 or out.shape[0] != 3 or out.shape[1] < tokens or (out.shape[1] > 1 and out.stride(1) != 1):
        raise ValueError("out must be a device int32 [3, >= tokens] whose rows are contiguous")
    return out, _on(dev.index, _positions, span, cu, start, t_step, out.data_ptr() or 256, out.stride(0))      # no tokens: nothing is written


class Rope:
    """Rotation of q / k rows by positions on several axes (``epd_rope_apply``).  Not seen by autograd: results carry no gradient, the
    backward pass is ``apply(..., inverse=True)`` on the gradients of the outputs."""

    def __init__(self, dtype: str, head_dim: int, pairs: Sequence[int], layout: str = "sections", ladder: str = "axis", pairing: str = "half",
                 base: float = 10000.0):
        c = self.cfg = epd_rope_cfg()
        c.struct_size = C.sizeof(epd_rope_cfg)
        c.dtype = {"f32": EPD_F32, "bf16": EPD_BF16}[dtype]
        c.head_dim, c.axes = head_dim, len(pairs)
        if not 1 <= len(pairs) <= 4:
            raise ValueError("pairs: one to four axes")
        c.pairs = (C.c_int32 * 4)(*pairs)
        c.layout = {"sections": EPD_ROPE_SECTIONS, "interleaved": EPD_ROPE_INTERLEAVED}[layout]
        c.ladder = {"axis": EPD_ROPE_LADDER_AXIS, "head": EPD_ROPE_LADDER_HEAD}[ladder]
        c.pairing = {"half": EPD_ROPE_HALF, "adjacent": EPD_ROPE_ADJACENT}[pairing]
        c.base = base
        self.dtype, self.head_dim, self.axes = torch_dtype(dtype), head_dim, len(pairs)

    def apply(self, tensors: Sequence[torch.Tensor], positions: torch.Tensor, inverse: bool = False,
              out: Optional[Sequence[torch.Tensor]] = None):
        """tensors: one to four of [tokens, heads, head_dim] (views with any strides but the last), positions int32 [axes, tokens].
        Returns the turned tensors: ``out``, which may be ``tensors`` itself, or new ones.  ``inverse`` turns back: the gradients of
        the inputs, given those of the outputs."""
        dev, axes = positions.get_device(), positions.shape
        if dev < 0 or positions.dtype != torch.int32 or len(axes) != 2 or axes[0] != self.axes or (axes[1] > 1 and positions.stride(1) != 1):
            raise ValueError("positions must be a device int32 [%d, tokens] whose rows are contiguous" % self.axes)
        T, d = axes[1], self.head_dim
        if T >= 1 << 31:
            raise ValueError("at most 2^31 - 1 tokens")

        def strides(v, shape):
            if v.get_device() != dev or v.dtype != self.dtype or v.shape != shape or len(shape) != 3 or shape[0] != T or shape[2] != d:
                raise ValueError("tensors must be [tokens, heads, %d] of %s on the positions' device" % (d, self.dtype))
            a, b, c = v.stride()
            if c != 1 and v.numel():
                raise ValueError("the elements of a head must be contiguous")
            return a, b

        if out is not None and len(out) != len(tensors):
            raise ValueError("as many outputs as tensors")
        arr, made = (epd_rope_tensor * len(tensors))(), []
        for i, x in enumerate(tensors):
            shape = x.shape
            si = strides(x, shape)
            if out is None:
                y, so = x.new_empty(shape), (shape[1] * d, d)
            else:
                y, so = out[i], strides(out[i], shape)
            made.append(y)
            arr[i] = (x.data_ptr(), y.data_ptr(), *si, *so, min(shape[1], 1 << 30))      # (the library takes 256 heads at most)
        _on(dev, epd_rope_apply, self.cfg, arr, positions.data_ptr() or 256, positions.stride(0), T, inverse)
        return made


def epd_gated_mlp_workspace_bytes(cfg: epd_gated_mlp_cfg) -> int:
    return int(lib.epd_gated_mlp_workspace_bytes(C.byref(cfg)))


def epd_gated_mlp_saved_bytes(cfg: epd_gated_mlp_cfg, tokens: int) -> int:
    return int(lib.epd_gated_mlp_saved_bytes(C.byref(cfg), tokens))


def epd_gated_mlp(cfg: epd_gated_mlp_cfg, weights: epd_gated_mlp_weights, x: int, ld_x: int, tokens: int, y: int, ld_y: int,
                  saved: Optional[int], workspace: int, workspace_bytes: int, stream: int) -> None:
    _op_check(lib.epd_gated_mlp(C.byref(cfg), C.byref(weights), x, ld_x, tokens, y, ld_y, saved, workspace, workspace_bytes, stream))


def epd_gated_mlp_backward(cfg: epd_gated_mlp_cfg, weights: epd_gated_mlp_weights, x: int, ld_x: int, dy: int, ld_dy: int, tokens: int,
                           saved: int, grads: epd_gated_mlp_grads, workspace: int, workspace_bytes: int, stream: int) -> None:
    _op_check(lib.epd_gated_mlp_backward(C.byref(cfg), C.byref(weights), x, ld_x, dy, ld_dy, tokens, saved, C.byref(grads), workspace,
                                         workspace_bytes, stream))


class GatedMLP:
    """Y = (act(X Wg^T) * (X Wu^T)) Wd^T with optional biases, and its backward pass.  Owns the workspace of its calls, so one call at
    a time: calls on other streams have to be ordered by the caller, as do replays of graphs that captured calls of one object, which
    has to outlive them.  Not seen by autograd, whatever requires gradients: ``forward`` returns values only, the backward pass is ``backward``.
    Weights are passed with every call, as a dict of gate_up_w [2F, D] (gate rows, then up rows), down_w [D, F] and, with biases,
    gate_up_b [2F], down_b [D]."""

    def __init__(self, dtype: str, hidden: int, mlp_dim: int, act: str = "swiglu", max_tokens: int = 1, use_bias: bool = False,
                 training: bool = False, device: str = "cuda:0"):
        c = self.cfg = epd_gated_mlp_cfg()
        c.struct_size = C.sizeof(epd_gated_mlp_cfg)
        c.dtype, c.act = {"f32": EPD_F32, "bf16": EPD_BF16}[dtype], _GATED[act]
        c.hidden, c.mlp_dim, c.max_tokens, c.use_bias, c.training = hidden, mlp_dim, max_tokens, int(use_bias), int(training)
        self.hidden, self.mlp_dim, self.dtype = hidden, mlp_dim, torch_dtype(dtype)
        self.workspace_bytes = epd_gated_mlp_workspace_bytes(c)
        if self.workspace_bytes == 0:
            raise EpdError(EPD_ERR_INVALID_ARG, epd_op_last_error())
        dev = torch.device(device)
        self.device = torch.device(dev.type, torch.cuda.current_device()) if dev.index is None else dev
        self.workspace = torch.empty(self.workspace_bytes + 256, dtype=torch.uint8, device=self.device)
        self._base = (self.workspace.data_ptr() + 255) // 256 * 256
        self._stream = torch.cuda.current_stream(self.device).cuda_stream       # on which the workspace may be handed on
        self._shapes = {"gate_up_w": (2 * mlp_dim, hidden), "down_w": (hidden, mlp_dim)}
        if use_bias:
            self._shapes.update(gate_up_b=(2 * mlp_dim,), down_b=(hidden,))

    def _weights(self, weights) -> epd_gated_mlp_weights:
        w = epd_gated_mlp_weights()
        for n, shape in self._shapes.items():
            t = weights[n]
            if t.shape != shape or t.dtype != self.dtype or t.get_device() != self.device.index or not t.is_contiguous():
                raise ValueError("%s must be a contiguous %s %s on %s" % (n, list(shape), self.dtype, self.device))
            setattr(w, n, t.data_ptr())
        return w

    def _rows(self, t: torch.Tensor, name: str, tokens: Optional[int] = None):
        """Address of the rows and what they are apart."""
        shape = t.shape
        if len(shape) != 2 or shape[1] != self.hidden or t.dtype != self.dtype or t.get_device() != self.device.index or (tokens is not None and shape[0] != tokens):
            raise ValueError("%s must be [tokens, %d] of %s on %s" % (name, self.hidden, self.dtype, self.device))
        ld, one = t.stride()
        if one != 1 and t.numel() and self.hidden > 1:
            raise ValueError("the rows of %s must be contiguous" % name)
        if shape[0] > self.cfg.max_tokens:
            raise EpdError(EPD_ERR_SHAPE, "%s has %d rows: 0 .. max_tokens %d" % (name, shape[0], self.cfg.max_tokens))
        return t.data_ptr(), self.hidden if shape[0] < 2 else ld      # one row: its stride means nothing

    def _call(self, call, *args) -> None:
        def on(*a):
            if a[-1] != self._stream:         # the allocator may not hand the workspace on before this stream is through
                self.workspace.record_stream(torch.cuda.current_stream(self.device))
            call(*a)
        _on(self.device.index, on, *args)

    def forward(self, weights, x: torch.Tensor, save: bool = False, out: Optional[torch.Tensor] = None):
        """x: [tokens, D], rows any stride apart.  Returns y, or (y, saved) with what ``backward`` needs (a uint8 tensor)."""
        px, ld_x = self._rows(x, "x")
        T = x.shape[0]
        y = torch.empty((T, self.hidden), dtype=self.dtype, device=self.device) if out is None else out
        py, ld_y = self._rows(y, "out", T)
        saved = torch.empty(epd_gated_mlp_saved_bytes(self.cfg, T), dtype=torch.uint8, device=self.device) if save else None
        self._call(epd_gated_mlp, self.cfg, self._weights(weights), px, ld_x, T, py, ld_y, None if saved is None else saved.data_ptr(), self._base,
                   self.workspace_bytes)
        return (y, saved) if save else y

    def backward(self, weights, x: torch.Tensor, dy: torch.Tensor, saved: torch.Tensor, want: Optional[Sequence[str]] = None) -> Dict[str, torch.Tensor]:
        """Gradients of sum(y * dy) by x ("dx") and by the weights; ``want`` names those to compute (all)."""
        px, ld_x = self._rows(x, "x")
        T = x.shape[0]
        pdy, ld_dy = self._rows(dy, "dy", T)
        if saved.dim() != 1 or saved.shape[0] != epd_gated_mlp_saved_bytes(self.cfg, T) or saved.dtype != torch.uint8 or saved.device != self.device or not saved.is_contiguous():
            raise ValueError("saved must be what forward returned for these rows")
        shapes = {"dx": (T, self.hidden), **self._shapes}
        grads, out = epd_gated_mlp_grads(), {}
        for n in (shapes if want is None else want):
            out[n] = torch.empty(shapes[n], dtype=self.dtype, device=self.device)
            setattr(grads, n, out[n].data_ptr())
        grads.ld_dx = self.hidden
        self._call(epd_gated_mlp_backward, self.cfg, self._weights(weights), px, ld_x, pdy, ld_dy, T, saved.data_ptr(), grads, self._base, self.workspace_bytes)
        return out


def _beyond_int32(who: str) -> None:
    raise ValueError("%s: sizes must be int32" % who)


# What these entries take as int32 is looked at here, or-ed together, as ctypes would cut it to its lower 32 bits: a number beyond takes all of it
# out of -2^31 ... 2^31 - 1, or stands beside a negative one, which the library refuses.
def epd_embed(cfg: epd_embed_cfg, table: int, rows: Optional[int], num_rows: int, ids: int, tokens: int, out: int, ld_out: int, stream: int) -> None:
    if not -1 << 31 <= num_rows | tokens < 1 << 31:
        _beyond_int32("epd_embed")
    _op_check(lib.epd_embed(cfg, table, rows, num_rows, ids, tokens, out, ld_out, stream))


def epd_embed_workspace_bytes(cfg: epd_embed_cfg) -> int:
    return int(lib.epd_embed_workspace_bytes(cfg))


def epd_embed_backward(cfg: epd_embed_cfg, ids: int, tokens: int, dout: int, ld_dout: int, num_rows: int, dtable: Optional[int], drows: Optional[int],
                       workspace: int, workspace_bytes: int, stream: int) -> None:
    if not -1 << 31 <= num_rows | tokens < 1 << 31:
        _beyond_int32("epd_embed_backward")
    _op_check(lib.epd_embed_backward(cfg, ids, tokens, dout, ld_dout, num_rows, dtable, drows, workspace, workspace_bytes, stream))


def epd_add_norm(cfg: epd_add_norm_cfg, rows: epd_add_norm_rows, gain: Optional[int], tokens: int, stream: int) -> None:
    if not -1 << 31 <= tokens < 1 << 31:
        _beyond_int32("epd_add_norm")
    _op_check(lib.epd_add_norm(cfg, rows, gain, tokens, stream))


def epd_add_norm_workspace_bytes(cfg: epd_add_norm_cfg) -> int:
    return int(lib.epd_add_norm_workspace_bytes(cfg))


def epd_add_norm_backward(cfg: epd_add_norm_cfg, grads: epd_add_norm_grads, gain: int, tokens: int, workspace: Optional[int], workspace_bytes: int, stream: int) -> None:
    if not -1 << 31 <= tokens < 1 << 31:
        _beyond_int32("epd_add_norm_backward")
    _op_check(lib.epd_add_norm_backward(cfg, grads, gain, tokens, workspace, workspace_bytes, stream))


def epd_quant_rows(dtype: int, x: int, ld_x: int, rows: int, cols: int, q: int, ld_q: int, scale: int, stream: int) -> None:
    if not -1 << 31 <= dtype | rows | cols < 1 << 31:
        _beyond_int32("epd_quant_rows")
    _op_check(lib.epd_quant_rows(dtype, x, ld_x, rows, cols, q, ld_q, scale, stream))


def epd_dequant_rows(q: int, ld_q: int, scale: int, rows: int, cols: int, dtype: int, out: int, ld_out: int, stream: int) -> None:
    if not -1 << 31 <= dtype | rows | cols < 1 << 31:
        _beyond_int32("epd_dequant_rows")
    _op_check(lib.epd_dequant_rows(q, ld_q, scale, rows, cols, dtype, out, ld_out, stream))


def epd_int8_linear_workspace_bytes(cfg: epd_int8_linear_cfg) -> int:
    return int(lib.epd_int8_linear_workspace_bytes(cfg))


def epd_int8_linear(cfg: epd_int8_linear_cfg, weights: epd_int8_linear_weights, x: int, ld_x: int, x_scale: int, tokens: int, y: int, ld_y: int,
                    workspace: int, workspace_bytes: int, stream: int) -> None:
    if not -1 << 31 <= tokens < 1 << 31:
        _beyond_int32("epd_int8_linear")
    _op_check(lib.epd_int8_linear(cfg, weights, x, ld_x, x_scale, tokens, y, ld_y, workspace, workspace_bytes, stream))


_DTYPES = {"f32": EPD_F32, "bf16": EPD_BF16}
_CODES = {torch.float32: EPD_F32, torch.bfloat16: EPD_BF16}


def _sizes(cfg, **values) -> None:
    """Fields of a configuration; numbers beyond 32 bits are refused, not wrapped."""
    cfg.struct_size = C.sizeof(cfg)
    for n, v in values.items():
        if isinstance(v, int) and not -1 << 31 <= v < 1 << 31:
            raise ValueError("%s must be an int32" % n)
        setattr(cfg, n, v)


def _matrix(t: torch.Tensor, name: str, rows: Optional[int], cols: int, dtype: torch.dtype, index: int):
    """Address of a matrix whose rows are contiguous, and what they are apart (one row: its stride means nothing)."""
    shape = t.shape
    if len(shape) != 2 or shape[1] != cols or (rows is not None and shape[0] != rows) or t.dtype != dtype or t.get_device() != index:
        raise ValueError("%s must be [%s, %d] of %s on device %d" % (name, "rows" if rows is None else rows, cols, dtype, index))
    if shape[0] < 2:
        ld, one = cols, t.stride(1)
    else:
        ld, one = t.stride()
    if one != 1 and cols > 1 and shape[0]:
        raise ValueError("the rows of %s must be contiguous" % name)
    return t.data_ptr() or 256, ld       # no rows: nothing is read or written


def _dense(t: torch.Tensor, name: str, shape, dtype: torch.dtype, index: int) -> int:
    if t.shape != shape or t.dtype != dtype or t.get_device() != index or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s %s on device %d" % (name, list(shape), dtype, index))
    return t.data_ptr() or 256


class _Operator:
    """Device of an operator's object and the workspace that its calls share: one call at a time."""

    def _own(self, nbytes: Optional[int], device: str) -> None:
        if nbytes == 0:
            raise EpdError(EPD_ERR_INVALID_ARG, epd_op_last_error())
        dev = torch.device(device)
        self.device = torch.device(dev.type, torch.cuda.current_device()) if dev.index is None else dev
        self._index = self.device.index
        self.workspace, self._base, self.workspace_bytes = None, None, 0
        if nbytes is not None:
            self.workspace_bytes = nbytes
            self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
            self._base = (self.workspace.data_ptr() + 255) // 256 * 256
            self._stream = torch.cuda.current_stream(self.device).cuda_stream       # on which the workspace may be handed on

    def _with_workspace(self, call, *args) -> None:
        i = self._index                       # (as _on, without a function made for every call)
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        stream = raw(i) if raw is not None else torch.cuda.current_stream(i).cuda_stream
        if stream != self._stream:            # the allocator may not hand the workspace on before this stream is through
            self.workspace.record_stream(torch.cuda.current_stream(self.device))
        if torch.cuda.current_device() == i:
            call(*args, self._base, self.workspace_bytes, stream)
        else:
            with torch.cuda.device(i):
                call(*args, self._base, self.workspace_bytes, stream)


class Embedding(_Operator):
    """Rows of sequences of text and visual tokens (``epd_embed``) and the gradients of both.  ids: int32, a row of the table (scaled),
    -1 - j for row j of ``rows``, anything else for zeros.  Not seen by autograd.  With ``training`` it owns the workspace of
    ``backward``: one such call at a time; calls on other streams have to be ordered by the caller, as do replays of graphs that
    captured calls of one object, which has to outlive them."""

    def __init__(self, dtype: str, vocab: int, hidden: int, out: Optional[str] = None, scale: float = 1.0, max_tokens: int = 1, training: bool = False,
                 device: str = "cuda:0"):
        c = self.cfg = epd_embed_cfg()
        _sizes(c, dtype=_DTYPES[dtype], out_dtype=_DTYPES[out or dtype], vocab=vocab, hidden=hidden, max_tokens=max_tokens, scale=scale)
        self.vocab, self.hidden, self.dtype, self.out_dtype, self.training = vocab, hidden, torch_dtype(dtype), torch_dtype(out or dtype), training
        nbytes = epd_embed_workspace_bytes(c)
        self._own(nbytes if training or nbytes == 0 else None, device)

    def _ids(self, ids: torch.Tensor):
        if ids.dim() != 1 or ids.dtype != torch.int32 or ids.get_device() != self._index or not ids.is_contiguous():
            raise ValueError("ids must be a contiguous int32 [tokens] on %s" % self.device)
        T = ids.shape[0]
        if T > self.cfg.max_tokens:
            raise EpdError(EPD_ERR_SHAPE, "%d ids: 0 .. max_tokens %d" % (T, self.cfg.max_tokens))
        return ids.data_ptr() or 256, T

    def forward(self, table: torch.Tensor, ids: torch.Tensor, rows: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Returns [tokens, hidden]: ``out``, whose rows may be any stride apart, or a new tensor."""
        pids, T = self._ids(ids)
        ptable = _dense(table, "table", (self.vocab, self.hidden), self.dtype, self._index)
        R = 0 if rows is None else rows.shape[0]
        prows = _dense(rows, "rows", (R, self.hidden), self.dtype, self._index) if R else None
        if out is None:
            out = torch.empty((T, self.hidden), dtype=self.out_dtype, device=self.device)
            py, ld = out.data_ptr() or 256, self.hidden
        else:
            py, ld = _matrix(out, "out", T, self.hidden, self.out_dtype, self._index)
        _on(self._index, epd_embed, self.cfg, ptable, prows, R, pids, T, py, ld)
        return out

    def backward(self, ids: torch.Tensor, dout: torch.Tensor, num_rows: int = 0, want: Optional[Sequence[str]] = None) -> Dict[str, torch.Tensor]:
        """Gradients of sum(out * dout) by the table ("table") and the ``num_rows`` rows ("rows"), every row of them; ``want`` names those
        to compute (all)."""
        if not self.training:
            raise EpdError(EPD_ERR_INVALID_ARG, "the object was made without training")
        pids, T = self._ids(ids)
        pd, ld = _matrix(dout, "dout", T, self.hidden, self.out_dtype, self._index)
        if not 0 <= num_rows < 1 << 31:
            raise ValueError("num_rows must be an int32 and not negative")
        out = {}
        for n in (("table", "rows") if num_rows else ("table",)) if want is None else want:
            out[n] = torch.empty(({"table": self.vocab, "rows": num_rows}[n], self.hidden), dtype=self.dtype, device=self.device)
        t, r = out.get("table"), out.get("rows")
        self._with_workspace(epd_embed_backward, self.cfg, pids, T, pd, ld, num_rows, None if t is None else t.data_ptr(),
                             None if r is None else r.data_ptr() or None)
        return out


class AddNorm(_Operator):
    """s = x + residual and its RMS norm y = s / sqrt(mean(s^2) + eps) * gain (``epd_add_norm``), in its own type or in 8 bits, and the
    backward pass.  ``residual``: type of the residual stream (that of x, or "f32").  Not seen by autograd.  With ``training`` it owns the
    workspace of ``backward``: one such call at a time; calls on other streams have to be ordered by the caller, as do replays of graphs
    that captured calls of one object, which has to outlive them."""

    def __init__(self, dtype: str, hidden: int, residual: Optional[str] = None, eps: float = 1e-6, max_tokens: int = 1, training: bool = False,
                 device: str = "cuda:0"):
        c = self.cfg = epd_add_norm_cfg()
        _sizes(c, dtype=_DTYPES[dtype], residual_dtype=_DTYPES[residual or dtype], hidden=hidden, max_tokens=max_tokens, eps=eps)
        self.hidden, self.dtype, self.residual_dtype, self.training = hidden, torch_dtype(dtype), torch_dtype(residual or dtype), training
        self._types = {"sum": self.residual_dtype, "y": self.dtype, "q": torch.int8, "dy": self.dtype,
                       "dsum": self.residual_dtype, "dx": self.dtype, "dresidual": self.residual_dtype}
        nbytes = epd_add_norm_workspace_bytes(c)
        self._own(nbytes if training or nbytes == 0 else None, device)

    def _tokens(self, t: torch.Tensor) -> int:
        T = t.shape[0]
        if T > self.cfg.max_tokens:
            raise EpdError(EPD_ERR_SHAPE, "%d rows: 0 .. max_tokens %d" % (T, self.cfg.max_tokens))
        return T

    def _output(self, out, name: str, T: int, like: Sequence[Optional[torch.Tensor]]):
        """The caller's tensor of that name, or a new one, its address and what its rows are apart."""
        t, kind = out.get(name) if out else None, self._types[name]
        if t is not None:
            return (t, *_matrix(t, name, T, self.hidden, kind, self._index))
        like = like[0] if like[0] is not None else like[-1]
        t = torch.empty_like(like, dtype=kind)      # (two thirds of the time of torch.empty; its rows lie side by side where those of `like` are contiguous)
        return t, t.data_ptr() or 256, self.hidden

    def forward(self, gain: Optional[torch.Tensor], x: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None, want: Sequence[str] = ("sum", "y"),
                out: Optional[Dict[str, torch.Tensor]] = None) -> Dict[str, torch.Tensor]:
        """x, residual: [tokens, hidden], rows any stride apart; one of them may be None.  ``want``: any of "sum", "y" and "q", which comes
        with "scale" (``quant_rows``).  ``out`` may name tensors for the outputs; sum may be ``residual``, y may be ``x``."""
        # (arguments are put together in one go: for 16 rows the call is a third of the host's time, its preparation another)
        some, D, i = x if x is not None else residual, self.hidden, self._index
        if some is None:
            raise ValueError("neither x nor residual")
        T = self._tokens(some)
        px, ld_x = (None, 0) if x is None else _matrix(x, "x", T, D, self.dtype, i)
        pr, ld_r = (None, 0) if residual is None else _matrix(residual, "residual", T, D, self.residual_dtype, i)
        made, at = {}, {}
        for n in want:
            if n not in ("sum", "y", "q"):
                raise ValueError("%r is no output" % (n,))
            made[n], *at[n] = self._output(out, n, T, (residual, x))
        ps = None
        if "q" in made:
            t = out.get("scale") if out else None
            made["scale"] = t = torch.empty(T, dtype=torch.float32, device=self.device) if t is None else t
            ps = _dense(t, "scale", (T,), torch.float32, i)
        none = (None, 0)
        (psum, ld_s), (py, ld_y), (pq, ld_q) = at.get("sum", none), at.get("y", none), at.get("q", none)
        pg = None if gain is None else _dense(gain, "gain", (D,), self.dtype, i)
        _on(i, epd_add_norm, self.cfg, epd_add_norm_rows(px, pr, psum, py, pq, ps, ld_x, ld_r, ld_s, ld_y, ld_q), pg, T)
        return made

    def backward(self, gain: torch.Tensor, sum: torch.Tensor, dy: torch.Tensor, dsum: Optional[torch.Tensor] = None, want: Optional[Sequence[str]] = None,
                 out: Optional[Dict[str, torch.Tensor]] = None) -> Dict[str, torch.Tensor]:
        """Gradients of sum(y * dy) + sum(s * dsum) at the kept ``sum``: "dx" (in the type of x), "dresidual" (the same values in that of
        the residual) and "gain".  ``want`` names those to compute (all; dresidual only where its type is another); ``out`` may name
        tensors for them; dx may be ``dy``, dresidual may be ``dsum``."""
        if not self.training:
            raise EpdError(EPD_ERR_INVALID_ARG, "the object was made without training")
        if want is None:
            want = ("dx", "gain") if self.dtype == self.residual_dtype else ("dx", "dresidual", "gain")
        if any(n not in ("dx", "dresidual", "gain") for n in want):
            raise ValueError("gradients are dx, dresidual and gain")
        T, D, i = self._tokens(sum), self.hidden, self._index
        ps, ld_s = _matrix(sum, "sum", T, D, self.residual_dtype, i)
        pdy, ld_dy = _matrix(dy, "dy", T, D, self.dtype, i)
        pds, ld_ds = (None, 0) if dsum is None else _matrix(dsum, "dsum", T, D, self.residual_dtype, i)
        made, none = {}, (None, 0)
        dx, dr, pgain = none, none, None
        if "dx" in want:
            made["dx"], *dx = self._output(out, "dx", T, (dy,))
        if "dresidual" in want:
            made["dresidual"], *dr = self._output(out, "dresidual", T, (sum,))
        if "gain" in want:
            t = out.get("gain") if out else None
            made["gain"] = t = torch.empty_like(gain) if t is None else t
            pgain = _dense(t, "gain", (D,), self.dtype, i)
        g = epd_add_norm_grads(ps, pdy, pds, dx[0], dr[0], pgain, ld_s, ld_dy, ld_ds, dx[1], dr[1])
        self._with_workspace(epd_add_norm_backward, self.cfg, g, _dense(gain, "gain", (D,), self.dtype, i), T)
        return made


def quant_rows(x: torch.Tensor, out: Optional[torch.Tensor] = None):
    """Rows in 8 bits (``epd_quant_rows``): (q int8, scale fp32 [rows]) with x ~ q * scale; rows any stride apart."""
    index, shape = x.get_device(), x.shape
    if index < 0 or len(shape) != 2 or x.dtype not in _CODES or shape[0] >= 1 << 31 or shape[1] >= 1 << 31:
        raise ValueError("x must be a device matrix of float32 or bfloat16")
    px, ld_x = _matrix(x, "x", shape[0], shape[1], x.dtype, index)
    if out is None:
        q = torch.empty_like(x, dtype=torch.int8)       # (rows side by side; see AddNorm._output)
        pq, ld_q = q.data_ptr() or 256, shape[1]
    else:
        q, (pq, ld_q) = out, _matrix(out, "out", shape[0], shape[1], torch.int8, index)
    scale = torch.empty(shape[0], dtype=torch.float32, device=x.device)
    _on(index, epd_quant_rows, _CODES[x.dtype], px, ld_x, shape[0], shape[1], pq, ld_q, scale.data_ptr() or 256)
    return q, scale


def dequant_rows(q: torch.Tensor, scale: torch.Tensor, dtype: str = "bf16", out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """q * scale of its row (``epd_dequant_rows``)."""
    index, shape, kind = q.get_device(), q.shape, torch_dtype(dtype)
    if index < 0 or len(shape) != 2 or shape[0] >= 1 << 31 or shape[1] >= 1 << 31:
        raise ValueError("q must be a device matrix of int8")
    pq, ld_q = _matrix(q, "q", shape[0], shape[1], torch.int8, index)
    ps = _dense(scale, "scale", (shape[0],), torch.float32, index)
    if out is None:
        out = torch.empty_like(q, dtype=kind)
        po, ld_o = out.data_ptr() or 256, shape[1]
    else:
        po, ld_o = _matrix(out, "out", shape[0], shape[1], kind, index)
    _on(index, epd_dequant_rows, pq, ld_q, ps, shape[0], shape[1], _DTYPES[dtype], po, ld_o)
    return out


class Int8Linear(_Operator):
    """y = (x w^T) * x_scale * scale (+ bias) of rows in 8 bits (``epd_int8_linear``, ``quant_rows``).  Owns the workspace of its calls, so
    one call at a time: calls on other streams have to be ordered by the caller, as do replays of graphs that captured calls of one
    object, which has to outlive them.  Weights are passed with every call, as a dict of w int8 [N, K], scale fp32 [N] and, with a bias,
    bias fp32 [N]."""

    def __init__(self, in_features: int, out_features: int, out: str = "bf16", max_tokens: int = 1, use_bias: bool = False, device: str = "cuda:0"):
        c = self.cfg = epd_int8_linear_cfg()
        _sizes(c, in_features=in_features, out_features=out_features, out_dtype=_DTYPES[out], use_bias=int(use_bias), max_tokens=max_tokens)
        self.in_features, self.out_features, self.use_bias, self.out_dtype = in_features, out_features, use_bias, torch_dtype(out)
        self._own(epd_int8_linear_workspace_bytes(c), device)

    def forward(self, weights: Dict[str, torch.Tensor], x: torch.Tensor, x_scale: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """x: int8 [tokens, K], rows a multiple of 16 apart; x_scale: fp32 [tokens].  Returns y [tokens, N]: ``out``, rows a multiple of 8
        apart, or a new tensor."""
        K, N, i = self.in_features, self.out_features, self._index
        w = epd_int8_linear_weights(_dense(weights["w"], "w", (N, K), torch.int8, i), _dense(weights["scale"], "scale", (N,), torch.float32, i),
                                    _dense(weights["bias"], "bias", (N,), torch.float32, i) if self.use_bias else None)
        T = x.shape[0]
        if T > self.cfg.max_tokens:
            raise EpdError(EPD_ERR_SHAPE, "x has %d rows: 0 .. max_tokens %d" % (T, self.cfg.max_tokens))
        px, ld_x = _matrix(x, "x", T, K, torch.int8, i)
        ps = _dense(x_scale, "x_scale", (T,), torch.float32, i)
        if out is None:
            out = torch.empty((T, N), dtype=self.out_dtype, device=self.device)
            py, ld_y = out.data_ptr() or 256, N
        else:
            py, ld_y = _matrix(out, "out", T, N, self.out_dtype, i)
        self._with_workspace(epd_int8_linear, self.cfg, w, px, ld_x, ps, T, py, ld_y)
        return out


EPI_STORE, EPI_GELU, EPI_RESIDUAL, EPI_QKV = 0, 1, 2, 3


def epd_probe_gemm_plan(M: int, N: int, K: int, epilogue: int = EPI_STORE, qk_cols: int = 0, compute_units: int = 0):
    """(tile_rows, tile_cols, body_rows) of the layer GEMM's launch plan for an M x N x K product (host only)."""
    tr, tc, br = C.c_int32(), C.c_int32(), C.c_int32()
    st = lib.epd_probe_gemm_plan(M, N, K, epilogue, qk_cols, compute_units, C.byref(tr), C.byref(tc), C.byref(br))
    if st != EPD_OK:
        raise EpdError(st, "epd_probe_gemm_plan: bad argument")
    return tr.value, tc.value, br.value
