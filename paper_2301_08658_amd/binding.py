"""ctypes binding of libatp.so (include/atp.h).

Argument marshalling only: every step of the path runs in the library's
HIP kernels.  Functions keep the C names; tensors are passed as torch
tensors (device pointer + leading dimension), streams as torch streams.
Sizes a C call cannot see (row counts of the buffers) are checked here so
that a short buffer never reaches a kernel.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libatp.so")

ATP_OK = 0
ATP_ERR_INVALID_ARGUMENT = 1
ATP_ERR_SHAPE = 2
ATP_ERR_UNSUPPORTED = 3
ATP_ERR_DEVICE = 4

ATP_ROW_FIRST = 0
ATP_COL_FIRST = 1
ATP_BLOCK_COL = 0
ATP_BLOCK_ROW = 1
ATP_EPI_NONE = 0
ATP_EPI_BIAS = 1
ATP_EPI_BIAS_GELU = 2
ATP_EPI_GELU_BWD = 3
ATP_F32 = 0
ATP_BF16 = 1
ATP_W_KN = 0
ATP_W_NK = 1
ATP_MAX_GROUP = 64
ATP_MAX_CHUNKS = 64

LINEARS = ("qkv", "out", "fc1", "fc2")


class AtpError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{status_string(status)}: {msg}")
        self.status = status


class atp_mesh(ctypes.Structure):
    _fields_ = [("d1", ctypes.c_int32), ("d2", ctypes.c_int32),
                ("i1", ctypes.c_int32), ("i2", ctypes.c_int32)]


class atp_shard(ctypes.Structure):
    _fields_ = [("k_loc", ctypes.c_int64), ("n_loc", ctypes.c_int64),
                ("k_off", ctypes.c_int64), ("n_off", ctypes.c_int64),
                ("red_axis", ctypes.c_int32), ("red_size", ctypes.c_int32),
                ("red_index", ctypes.c_int32), ("bwd_axis", ctypes.c_int32),
                ("bwd_size", ctypes.c_int32), ("bwd_index", ctypes.c_int32)]

    def as_dict(self):
        return {f: getattr(self, f) for f, _ in self._fields_}


_vp = ctypes.c_void_p
_fpp = ctypes.POINTER(ctypes.c_void_p)   # float* const* (host array of device ptrs)


class atp_block_weights(ctypes.Structure):
    _fields_ = [("w", _vp * 4), ("ldw", ctypes.c_int64 * 4), ("b", _vp * 4),
                ("layout", ctypes.c_int32)]


class atp_block_fwd_io(ctypes.Structure):
    _fields_ = [("x_loc", _vp), ("ldx", ctypes.c_int64),
                ("attn_loc", _vp), ("lda", ctypes.c_int64),
                ("partials", _fpp * 4), ("ldp", ctypes.c_int64 * 4),
                ("qkv", _vp), ("ld_qkv", ctypes.c_int64),
                ("o", _vp), ("ld_o", ctypes.c_int64),
                ("h", _vp), ("ld_h", ctypes.c_int64),
                ("pre", _vp),
                ("z", _vp), ("ld_z", ctypes.c_int64),
                ("partial_dtype", ctypes.c_int32)]


class atp_block_bwd_io(ctypes.Structure):
    _fields_ = [("x_loc", _vp), ("ldx", ctypes.c_int64),
                ("attn_loc", _vp), ("lda", ctypes.c_int64),
                ("h", _vp), ("ld_h", ctypes.c_int64),
                ("pre", _vp),
                ("dz", _vp), ("ld_dz", ctypes.c_int64),
                ("dqkv", _vp), ("ld_dqkv", ctypes.c_int64),
                ("d_o", _vp), ("ld_do", ctypes.c_int64),
                ("dx_partials", _fpp * 4), ("ld_dxp", ctypes.c_int64 * 4),
                ("dh_pre", _vp),
                ("dx_qkv", _vp), ("ld_dx_qkv", ctypes.c_int64),
                ("dx_fc1", _vp), ("ld_dx_fc1", ctypes.c_int64),
                ("d_attn", _vp), ("ld_d_attn", ctypes.c_int64),
                ("dw", _vp * 4), ("db", _vp * 4),
                ("partial_dtype", ctypes.c_int32)]


class atp_attn_block_fwd_io(ctypes.Structure):
    _fields_ = [("x_loc", _vp), ("ldx", ctypes.c_int64),
                ("qkv_partials", _fpp), ("ldp_qkv", ctypes.c_int64),
                ("qkv", _vp), ("ld_qkv", ctypes.c_int64),
                ("attn", _vp), ("ld_attn", ctypes.c_int64),
                ("lse", _vp),
                ("o_partials", _fpp), ("ldp_o", ctypes.c_int64),
                ("o", _vp), ("ld_o", ctypes.c_int64),
                ("partial_dtype", ctypes.c_int32)]


class atp_attn_block_bwd_io(ctypes.Structure):
    _fields_ = [("x_loc", _vp), ("ldx", ctypes.c_int64),
                ("qkv", _vp), ("ld_qkv", ctypes.c_int64),
                ("attn", _vp), ("ld_attn", ctypes.c_int64),
                ("lse", _vp),
                ("d_o", _vp), ("ld_do", ctypes.c_int64),
                ("d_attn_partials", _fpp), ("ldp_da", ctypes.c_int64),
                ("d_attn", _vp), ("ld_d_attn", ctypes.c_int64),
                ("delta", _vp),
                ("d_qkv", _vp), ("ld_dqkv", ctypes.c_int64),
                ("dx_partials", _fpp), ("ldp_dx", ctypes.c_int64),
                ("dx", _vp), ("ld_dx", ctypes.c_int64),
                ("dw", _vp * 2), ("db", _vp * 2),
                ("partial_dtype", ctypes.c_int32)]


class atp_qk_norm_rope(ctypes.Structure):
    _fields_ = [("q_weight", _vp), ("k_weight", _vp), ("inv_freq", _vp), ("eps", ctypes.c_float),
                ("norm", ctypes.c_int32), ("rotary_dims", ctypes.c_int32),
                ("interleaved", ctypes.c_int32)]


class atp_kv_cache(ctypes.Structure):
    _fields_ = [("pages", _vp), ("n_pages", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("page_size", ctypes.c_int32)]


class atp_kv_batch(ctypes.Structure):
    _fields_ = [("table", _vp), ("ld_table", ctypes.c_int64), ("max_pages", ctypes.c_int32),
                ("n_seqs", ctypes.c_int32), ("ctx", _vp), ("cu_new", _vp)]


class atp_layer_norm(ctypes.Structure):
    _fields_ = [("weight", _vp), ("bias", _vp), ("eps", ctypes.c_float)]


class atp_attention_docs(ctypes.Structure):
    _fields_ = [("cu_docs", _vp), ("prefix", _vp), ("slopes", _vp), ("n_docs", ctypes.c_int32),
                ("cap", ctypes.c_float)]


class atp_grad(ctypes.Structure):
    _fields_ = [("src", _vp), ("dst", _vp), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("ld_src", ctypes.c_int64), ("ld_dst", ctypes.c_int64),
                ("src_dtype", ctypes.c_int32), ("dst_dtype", ctypes.c_int32)]


class atp_kernel_stat(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 64), ("launches", ctypes.c_int64),
                ("total_ms", ctypes.c_double), ("flops", ctypes.c_double),
                ("bytes", ctypes.c_double)]


class atp_hcm_layer(ctypes.Structure):
    _fields_ = [("ranks", ctypes.c_int32), ("group_bw", ctypes.c_double),
                ("p2p", ctypes.POINTER(ctypes.c_double))]


class atp_model_dims(ctypes.Structure):
    _fields_ = [("layers", ctypes.c_int64), ("batch", ctypes.c_int64), ("seq", ctypes.c_int64),
                ("hidden", ctypes.c_int64), ("elem_bytes", ctypes.c_int32)]


class atp_mesh_cost(ctypes.Structure):
    _fields_ = [("d1", ctypes.c_int32), ("d2", ctypes.c_int32),
                ("b1_eff", ctypes.c_double), ("b2_eff", ctypes.c_double),
                ("b1", ctypes.c_double), ("b2", ctypes.c_double), ("t_comm", ctypes.c_double)]

    def as_dict(self):
        return {f: getattr(self, f) for f, _ in self._fields_}


EXPORTS = (
    "atp_shard_geometry", "atp_shard_linear_fwd", "atp_chunked_partial_reduce",
    "atp_shard_linear_bwd", "atp_block_workspace_bytes", "atp_block_fwd", "atp_block_bwd",
    "atp_profile_enable", "atp_profile_collect", "atp_status_string", "atp_last_error",
    "atp_version", "atp_tcomm", "atp_hcm_mesh_cost", "atp_plan_mesh", "atp_transpose_bf16",
    "atp_attention_fwd", "atp_attention_bwd", "atp_chunked_partial_reduce_bf16",
    "atp_shard_linear_fwd_fused", "atp_block_workspace_path", "atp_block_geometry",
    "atp_attention_heads", "atp_attention_block_fwd", "atp_attention_block_bwd",
    "atp_attention_bwd_noalloc", "atp_qk_norm_rope_fwd", "atp_qk_norm_rope_bwd",
    "atp_qk_norm_rope_workspace_bytes", "atp_qk_norm_rope_cache", "atp_cache_reserve",
    "atp_cache_workspace_bytes", "atp_cache_fork", "atp_cache_release", "atp_cache_copy_pages",
    "atp_cache_compact", "atp_attention_cache_fwd", "atp_attention_cache_workspace_bytes",
    "atp_embedding_fwd", "atp_embedding_bwd", "atp_embedding_workspace_bytes",
    "atp_layer_norm_fwd", "atp_layer_norm_stats", "atp_layer_norm_bwd", "atp_layer_norm_bwd_sums",
    "atp_layer_norm_workspace_bytes", "atp_attention_docs_fwd", "atp_attention_docs_bwd",
    "atp_attention_docs_workspace_bytes", "atp_grad_sq_sum", "atp_grad_clip",
    "atp_grad_workspace_bytes",
)
ATP_MAX_QUERY_GROUP = 64
ATP_MAX_FORKS = 4096
HEAD_DIM = 128
ATP_NOALLOC_DELTA_MAX = 1 << 20   # values of atp_attention_bwd_noalloc's scratch

_lib = None


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """Load libatp.so.  Raises if it has not been built: there is no fallback."""
    global _lib
    if _lib is not None:
        return _lib
    path = path or LIB_PATH
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build the HIP library first "
                          "(python -m paper_2301_08658_amd.build)")
    lib = ctypes.CDLL(path)
    i32, i64, sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    mp = ctypes.POINTER(atp_mesh)
    lib.atp_shard_geometry.argtypes = [mp, i32, i64, i64, ctypes.POINTER(atp_shard)]
    lib.atp_shard_geometry.restype = i32
    lib.atp_shard_linear_fwd.argtypes = [mp, i32, i64, i64, i64, i32, _vp, i64, _vp, i64, _vp,
                                         i32, _vp, i32, i64, _vp, _vp, _fpp]
    lib.atp_shard_linear_fwd.restype = i32
    lib.atp_chunked_partial_reduce.argtypes = [i32, i64, i64, i32, _fpp, i64, _vp, i32, _vp, _vp,
                                               i32, i64, _vp, _vp, _fpp]
    lib.atp_chunked_partial_reduce.restype = i32
    lib.atp_chunked_partial_reduce_bf16.argtypes = lib.atp_chunked_partial_reduce.argtypes
    lib.atp_chunked_partial_reduce_bf16.restype = i32
    lib.atp_shard_linear_fwd_fused.argtypes = [mp, i32, i64, i64, i64, _vp, i64, _vp, i64, _fpp,
                                               i64, _vp, i32, _vp, i32, i64, _vp, _vp]
    lib.atp_shard_linear_fwd_fused.restype = i32
    lib.atp_shard_linear_bwd.argtypes = [mp, i32, i64, i64, i64, i32, _vp, i64, _vp, i64, _vp, i64,
                                         _vp, i64, _vp, i64, _vp, _vp, _fpp]
    lib.atp_shard_linear_bwd.restype = i32
    lib.atp_block_workspace_bytes.argtypes = [mp, i32, i64, i64, i32, i32]
    lib.atp_block_workspace_bytes.restype = sz
    lib.atp_block_workspace_path.argtypes = [mp, i32, i64, i64, i32, sz, i32]
    lib.atp_block_workspace_path.restype = i32
    lib.atp_block_geometry.argtypes = [mp, i32, i64, ctypes.POINTER(atp_shard)]
    lib.atp_block_geometry.restype = i32
    i32p = ctypes.POINTER(i32)
    lib.atp_attention_heads.argtypes = [mp, i32, i64, i32, i32p, i32p, i32p]
    lib.atp_attention_heads.restype = i32
    lib.atp_attention_block_fwd.argtypes = [mp, i32, i64, i64, i64, i32, i32,
                                            ctypes.POINTER(atp_block_weights),
                                            ctypes.POINTER(atp_attn_block_fwd_io), _vp,
                                            ctypes.c_size_t, _vp, _vp]
    lib.atp_attention_block_fwd.restype = i32
    lib.atp_attention_block_bwd.argtypes = [mp, i32, i64, i64, i64, i32, i32,
                                            ctypes.POINTER(atp_block_weights),
                                            ctypes.POINTER(atp_attn_block_bwd_io), _vp,
                                            ctypes.c_size_t, _vp, _vp]
    lib.atp_attention_block_bwd.restype = i32
    lib.atp_block_fwd.argtypes = [mp, i32, i64, i64, i32, ctypes.POINTER(atp_block_weights),
                                  ctypes.POINTER(atp_block_fwd_io), _vp, sz, _vp, _vp]
    lib.atp_block_fwd.restype = i32
    lib.atp_block_bwd.argtypes = [mp, i32, i64, i64, i32, ctypes.POINTER(atp_block_weights),
                                  ctypes.POINTER(atp_block_bwd_io), _vp, sz, _vp, _vp]
    lib.atp_block_bwd.restype = i32
    lib.atp_profile_enable.argtypes = [i32]
    lib.atp_profile_enable.restype = None
    lib.atp_profile_collect.argtypes = [ctypes.POINTER(atp_kernel_stat), i32]
    lib.atp_profile_collect.restype = i32
    lib.atp_status_string.argtypes = [i32]
    lib.atp_status_string.restype = ctypes.c_char_p
    lib.atp_last_error.argtypes = []
    lib.atp_last_error.restype = ctypes.c_char_p
    lib.atp_version.argtypes = []
    lib.atp_version.restype = ctypes.c_char_p
    lib.atp_transpose_bf16.argtypes = [i64, i64, _vp, i64, _vp, i64, _vp]
    lib.atp_transpose_bf16.restype = i32
    lib.atp_attention_fwd.argtypes = [mp, i32, i64, i64, i64, i32, _vp, i64, _vp, i64, _vp, _vp]
    lib.atp_attention_fwd.restype = i32
    lib.atp_attention_bwd.argtypes = [mp, i32, i64, i64, i64, i32, _vp, i64, _vp, i64, _vp, _vp,
                                      i64, _vp, i64, _vp, _vp]
    lib.atp_attention_bwd.restype = i32
    lib.atp_attention_bwd_noalloc.argtypes = [mp, i32, i64, i64, i64, i32, _vp, i64, _vp, i64,
                                              _vp, _vp, i64, _vp, i64, _vp]
    lib.atp_attention_bwd_noalloc.restype = i32
    nrp, kcp, kbp = (ctypes.POINTER(atp_qk_norm_rope), ctypes.POINTER(atp_kv_cache),
                     ctypes.POINTER(atp_kv_batch))
    lib.atp_qk_norm_rope_fwd.argtypes = [i64, i64, i32, i32, nrp, _vp, _vp, i64, _vp, i64, _vp]
    lib.atp_qk_norm_rope_bwd.argtypes = [i64, i64, i32, i32, nrp, _vp, _vp, i64, _vp, i64, _vp,
                                         i64, _vp, _vp, _vp, sz, _vp]
    lib.atp_qk_norm_rope_workspace_bytes.argtypes = [i64]
    lib.atp_qk_norm_rope_cache.argtypes = [kcp, kbp, i64, i32, nrp, _vp, _vp, i64, _vp, i64, _vp]
    lib.atp_cache_reserve.argtypes = [i32, i32, _vp, kbp, _vp, _vp, _vp, _vp, _vp, sz, _vp]
    lib.atp_cache_workspace_bytes.argtypes = [i32, i32]
    lib.atp_cache_fork.argtypes = [i32, i32, _vp, kbp, i32, _vp, _vp, _vp, _vp]
    lib.atp_cache_release.argtypes = [i32, i32, _vp, kbp, _vp, _vp]
    lib.atp_cache_copy_pages.argtypes = [kcp, i32, _vp, _vp, _vp, _vp]
    lib.atp_cache_compact.argtypes = [kcp, kbp, _vp, _vp, i32, _vp, _vp]
    lib.atp_attention_cache_fwd.argtypes = [kcp, kbp, i64, i32, i32, _vp, i64, _vp, i32, _vp, i64,
                                            _vp, _vp, sz, _vp]
    lib.atp_attention_cache_workspace_bytes.argtypes = [i32, i32, i32]
    f32 = ctypes.c_float
    lnp, adp, gp = (ctypes.POINTER(atp_layer_norm), ctypes.POINTER(atp_attention_docs),
                    ctypes.POINTER(atp_grad))
    lib.atp_embedding_fwd.argtypes = [i64, _vp, i64, i64, i64, _vp, i64, f32, _vp, i32, i64, _vp]
    lib.atp_embedding_bwd.argtypes = [i64, _vp, i64, i64, i64, _vp, i64, f32, _vp, i64, i32, _vp,
                                      sz, _vp]
    lib.atp_embedding_workspace_bytes.argtypes = [i64, i64, i64]
    lib.atp_layer_norm_stats.argtypes = [i64, i64, i32, _vp, i64, _vp, i64, _vp, i64, _vp, _vp]
    lib.atp_layer_norm_fwd.argtypes = [i64, i64, i32, lnp, _vp, i64, _vp, i64, _vp, i64, i32, _fpp,
                                       _vp, i64, _vp, _vp, _vp]
    lib.atp_layer_norm_bwd_sums.argtypes = [i64, i64, i32, lnp, _vp, i64, _vp, _vp, _vp, i64, _vp,
                                            _vp]
    lib.atp_layer_norm_bwd.argtypes = [i64, i64, i32, lnp, _vp, i64, _vp, _vp, _vp, i64, _vp, i64,
                                       i32, _fpp, _vp, i64, _vp, i64, _vp, _vp, _vp, sz, _vp]
    lib.atp_layer_norm_workspace_bytes.argtypes = [i64, i64]
    lib.atp_attention_docs_fwd.argtypes = [i64, i32, i32, adp, _vp, i64, _vp, i64, _vp, _vp]
    lib.atp_attention_docs_bwd.argtypes = [i64, i32, i32, adp, _vp, i64, _vp, i64, _vp, _vp, i64,
                                           _vp, i64, _vp, sz, _vp]
    lib.atp_attention_docs_workspace_bytes.argtypes = [i64, i32, i32]
    lib.atp_grad_sq_sum.argtypes = [i32, gp, _vp, _vp, sz, _vp]
    lib.atp_grad_clip.argtypes = [i32, gp, i32, _fpp, f32, f32, _vp, _vp]
    lib.atp_grad_workspace_bytes.argtypes = [i32, gp]
    for name in EXPORTS[EXPORTS.index("atp_qk_norm_rope_fwd"):]:
        getattr(lib, name).restype = sz if name.endswith("_bytes") else i32
    hp, dp, cp = (ctypes.POINTER(atp_hcm_layer), ctypes.POINTER(atp_model_dims),
                  ctypes.POINTER(atp_mesh_cost))
    lib.atp_tcomm.argtypes = [dp, i32, i32, ctypes.c_double, ctypes.c_double,
                              ctypes.POINTER(ctypes.c_double)]
    lib.atp_tcomm.restype = i32
    lib.atp_hcm_mesh_cost.argtypes = [hp, i32, dp, i32, i32, cp]
    lib.atp_hcm_mesh_cost.restype = i32
    lib.atp_plan_mesh.argtypes = [hp, i32, dp, cp, cp, i32, ctypes.POINTER(i32)]
    lib.atp_plan_mesh.restype = i32
    _lib = lib
    return lib


def status_string(s: int) -> str:
    return load_library().atp_status_string(int(s)).decode()


def last_error() -> str:
    return load_library().atp_last_error().decode()


def _check(status: int):
    if status != ATP_OK:
        raise AtpError(status, last_error())


# ---------------------------------------------------------------- marshalling
def mesh(d1, d2, i1=0, i2=0) -> atp_mesh:
    return atp_mesh(int(d1), int(d2), int(i1), int(i2))


def _on_device(t: torch.Tensor, name: str):
    """The library reads and writes device memory of the current HIP device."""
    if not t.is_cuda:
        raise ValueError(f"{name}: must be a tensor on the GPU, got one on {t.device}")
    if t.device.index != torch.cuda.current_device():
        raise ValueError(f"{name}: on {t.device}, but the current device is "
                         f"cuda:{torch.cuda.current_device()}")


def _ptr(t: Optional[torch.Tensor], name: str = "tensor") -> Optional[int]:
    if t is None:
        return None
    _on_device(t, name)
    return t.data_ptr()


def _mat(t: Optional[torch.Tensor], rows: int, cols: int, dtype, name: str):
    """(pointer, ld) of a row-major device matrix with at least rows x cols."""
    if t is None:
        return None, 0
    _on_device(t, name)
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.dim() != 2 or (t.size(1) > 1 and t.stride(1) != 1):
        raise ValueError(f"{name}: needs a 2-D row-major tensor")
    if t.size(0) < rows or t.size(1) < cols:
        raise ValueError(f"{name}: {tuple(t.shape)} smaller than [{rows}, {cols}]")
    return t.data_ptr(), (t.stride(0) if t.size(0) > 1 else max(t.size(1), cols))


def _vec(t: Optional[torch.Tensor], n: int, dtype, name: str):
    if t is None:
        return None
    _on_device(t, name)
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.numel() < n or not t.is_contiguous():
        raise ValueError(f"{name}: needs {n} contiguous elements")
    return t.data_ptr()


# the raw handle of a device's current stream, without a Stream object around it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(s, dev: Optional[int] = None) -> Optional[int]:
    if s is None:
        if dev is not None and _raw_stream is not None:
            return _raw_stream(dev)
        return torch.cuda.current_stream().cuda_stream
    if isinstance(s, int):
        return s
    return s.cuda_stream


def _opt_stream(s) -> Optional[int]:
    """A stream that may be absent (NULL)."""
    return None if s is None else _stream(s)


def _events(evs: Optional[Sequence]) -> Optional[ctypes.Array]:
    if evs is None:
        return None
    return (ctypes.c_void_p * len(evs))(*[e.handle if isinstance(e, HipEvent) else e
                                          for e in evs])


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return ATP_F32
    if t.dtype == torch.bfloat16:
        return ATP_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _ptr_table(ts: Sequence[Optional[torch.Tensor]], rows: int, cols: int, name: str,
               dtype=torch.float32):
    """Host array of device pointers (None entries stay NULL) and their common ld."""
    arr = (ctypes.c_void_p * len(ts))()
    ld = None
    for j, t in enumerate(ts):
        if t is None:
            continue
        p, l = _mat(t, rows, cols, dtype, f"{name}[{j}]")
        arr[j] = p
        if ld is None:
            ld = l
        elif l != ld:
            raise ValueError(f"{name}: all buffers need the same leading dimension")
    return ctypes.cast(arr, _fpp), arr, (ld or cols)


class HipEvent:
    """A raw hipEvent_t (created through the HIP runtime) for chunk signalling."""
    _hip = None

    def __init__(self, timing: bool = False):
        if HipEvent._hip is None:
            HipEvent._hip = ctypes.CDLL("libamdhip64.so")
        h = ctypes.c_void_p()
        flags = 0 if timing else 0x2   # hipEventDisableTiming
        rc = HipEvent._hip.hipEventCreateWithFlags(ctypes.byref(h), ctypes.c_uint(flags))
        if rc != 0:
            raise RuntimeError(f"hipEventCreateWithFlags failed ({rc})")
        self.handle = h.value

    def synchronize(self):
        rc = HipEvent._hip.hipEventSynchronize(ctypes.c_void_p(self.handle))
        if rc != 0:
            raise RuntimeError(f"hipEventSynchronize failed ({rc})")

    def __del__(self):
        if HipEvent._hip is not None and getattr(self, "handle", None):
            HipEvent._hip.hipEventDestroy(ctypes.c_void_p(self.handle))


# ---------------------------------------------------------------- the ABI
def atp_version() -> str:
    return load_library().atp_version().decode()


def atp_shard_geometry(m: atp_mesh, mode: int, k: int, n: int) -> atp_shard:
    out = atp_shard()
    _check(load_library().atp_shard_geometry(ctypes.byref(m), int(mode), int(k), int(n),
                                             ctypes.byref(out)))
    return out


def atp_shard_linear_fwd(m: atp_mesh, mode: int, tokens: int, k: int, n: int, chunks: int,
                         x_loc, w_loc, bias_loc, epi: int, y, preact=None, stream=None,
                         chunk_done=None):
    g = atp_shard_geometry(m, mode, k, n)
    xp, ldx = _mat(x_loc, tokens, g.k_loc, torch.bfloat16, "x_loc")
    wp, ldw = _mat(w_loc, g.k_loc, g.n_loc, torch.bfloat16, "w_loc")
    yp, ldy = _mat(y, tokens, g.n_loc, y.dtype, "y")
    pp, ldp = _mat(preact, tokens, g.n_loc, torch.bfloat16, "preact")
    if preact is not None and ldp != ldy:
        raise ValueError("preact must share y's leading dimension")
    bp = _vec(bias_loc, g.n_loc, torch.bfloat16, "bias_loc")
    _check(load_library().atp_shard_linear_fwd(
        ctypes.byref(m), int(mode), int(tokens), int(k), int(n), int(chunks), xp, ldx, wp, ldw,
        bp, int(epi), yp, _dtype_code(y), ldy, pp, _stream(stream), _events(chunk_done)))


def atp_chunked_partial_reduce(red_size: int, tokens: int, n_loc: int, chunks: int, partials,
                               bias_loc, epi: int, out, preact_in=None, preact_out=None,
                               stream=None, chunk_ready=None):
    if len(partials) != red_size:
        raise ValueError("need exactly red_size partial buffers")
    tab, _keep, ldp = _ptr_table(partials, tokens, n_loc, "partials")
    op, ldo = _mat(out, tokens, n_loc, out.dtype, "out")
    ip, ldi = _mat(preact_in, tokens, n_loc, torch.bfloat16, "preact_in")
    qp, ldq = _mat(preact_out, tokens, n_loc, torch.bfloat16, "preact_out")
    for t, l in ((preact_in, ldi), (preact_out, ldq)):
        if t is not None and l != ldo:
            raise ValueError("pre-activation buffers must share out's leading dimension")
    bp = _vec(bias_loc, n_loc, torch.bfloat16, "bias_loc")
    _check(load_library().atp_chunked_partial_reduce(
        int(red_size), int(tokens), int(n_loc), int(chunks), tab, ldp, bp, int(epi), ip, op,
        _dtype_code(out), ldo, qp, _stream(stream), _events(chunk_ready)))


def atp_chunked_partial_reduce_bf16(red_size: int, tokens: int, n_loc: int, chunks: int,
                                    partials, bias_loc, epi: int, out, preact_in=None,
                                    preact_out=None, stream=None, chunk_ready=None):
    if len(partials) != red_size:
        raise ValueError("need exactly red_size partial buffers")
    tab, _keep, ldp = _ptr_table(partials, tokens, n_loc, "partials", torch.bfloat16)
    op, ldo = _mat(out, tokens, n_loc, out.dtype, "out")
    ip, ldi = _mat(preact_in, tokens, n_loc, torch.bfloat16, "preact_in")
    qp, ldq = _mat(preact_out, tokens, n_loc, torch.bfloat16, "preact_out")
    for t, l in ((preact_in, ldi), (preact_out, ldq)):
        if t is not None and l != ldo:
            raise ValueError("pre-activation buffers must share out's leading dimension")
    bp = _vec(bias_loc, n_loc, torch.bfloat16, "bias_loc")
    _check(load_library().atp_chunked_partial_reduce_bf16(
        int(red_size), int(tokens), int(n_loc), int(chunks), tab, ldp, bp, int(epi), ip, op,
        _dtype_code(out), ldo, qp, _stream(stream), _events(chunk_ready)))


def atp_shard_linear_fwd_fused(m: atp_mesh, mode: int, tokens: int, k: int, n: int, x_loc,
                               w_loc, peers, bias_loc, epi: int, out, preact=None, stream=None):
    """peers: red_size entries, the other members' f32 partials (the own
    entry may be None; it is not read)."""
    g = atp_shard_geometry(m, mode, k, n)
    if len(peers) != g.red_size:
        raise ValueError("need exactly red_size peer entries")
    xp, ldx = _mat(x_loc, tokens, g.k_loc, torch.bfloat16, "x_loc")
    wp, ldw = _mat(w_loc, g.k_loc, g.n_loc, torch.bfloat16, "w_loc")
    tab, _keep, ldp = _ptr_table(peers, tokens, g.n_loc, "peers")
    op, ldo = _mat(out, tokens, g.n_loc, out.dtype, "out")
    pp, ldq = _mat(preact, tokens, g.n_loc, torch.bfloat16, "preact")
    if preact is not None and ldq != ldo:
        raise ValueError("preact must share out's leading dimension")
    bp = _vec(bias_loc, g.n_loc, torch.bfloat16, "bias_loc")
    _check(load_library().atp_shard_linear_fwd_fused(
        ctypes.byref(m), int(mode), int(tokens), int(k), int(n), xp, ldx, wp, ldw,
        tab if g.red_size > 1 else None, ldp, bp, int(epi), op, _dtype_code(out), ldo, pp,
        _stream(stream)))


def atp_shard_linear_bwd(m: atp_mesh, mode: int, tokens: int, k: int, n: int, chunks: int,
                         x_loc, w_loc, dy, dx_partial, dw, db=None, stream=None,
                         dx_chunk_done=None):
    g = atp_shard_geometry(m, mode, k, n)
    xp, ldx = _mat(x_loc, tokens, g.k_loc, torch.bfloat16, "x_loc")
    wp, ldw = _mat(w_loc, g.k_loc, g.n_loc, torch.bfloat16, "w_loc")
    yp, ldy = _mat(dy, tokens, g.n_loc, torch.bfloat16, "dy")
    dxp, lddx = _mat(dx_partial, tokens, g.k_loc, torch.float32, "dx_partial")
    dwp, lddw = _mat(dw, g.k_loc, g.n_loc, torch.float32, "dw")
    dbp = _vec(db, g.n_loc, torch.float32, "db")
    _check(load_library().atp_shard_linear_bwd(
        ctypes.byref(m), int(mode), int(tokens), int(k), int(n), int(chunks), xp, ldx, wp, ldw,
        yp, ldy, dxp, lddx, dwp, lddw, dbp, _stream(stream), _events(dx_chunk_done)))


def block_geometry(m: atp_mesh, block_mode: int, h: int):
    """Shard geometry of the block's four linears (qkv, out, fc1, fc2)."""
    out = (atp_shard * 4)()
    _check(load_library().atp_block_geometry(ctypes.byref(m), int(block_mode), int(h), out))
    return [out[i] for i in range(4)]


def atp_block_workspace_bytes(m: atp_mesh, block_mode: int, tokens: int, h: int,
                              chunks: int, weight_layout: int = ATP_W_KN) -> int:
    return int(load_library().atp_block_workspace_bytes(ctypes.byref(m), int(block_mode),
                                                         int(tokens), int(h), int(chunks),
                                                         int(weight_layout)))


def atp_block_workspace_path(m: atp_mesh, block_mode: int, tokens: int, h: int,
                             weight_layout: int, ws_bytes: int, pass_: int) -> int:
    """1: a block call of the pass (0 fwd, 1 bwd) with ws_bytes of workspace
    takes the transposed-layout path; 0: the direct path; -1: invalid."""
    return int(load_library().atp_block_workspace_path(ctypes.byref(m), int(block_mode),
                                                        int(tokens), int(h), int(weight_layout),
                                                        int(ws_bytes), int(pass_)))


def _weights(G, w: Sequence[torch.Tensor], b: Sequence[torch.Tensor], layout: int):
    """Weights [k_loc, n_loc] (ATP_W_KN) or [n_loc, k_loc] (ATP_W_NK)."""
    W = atp_block_weights()
    W.layout = int(layout)
    for i, g in enumerate(G):
        r, c = (g.k_loc, g.n_loc) if layout == ATP_W_KN else (g.n_loc, g.k_loc)
        p, ld = _mat(w[i], r, c, torch.bfloat16, f"w[{LINEARS[i]}]")
        W.w[i] = p
        W.ldw[i] = ld
        W.b[i] = _vec(b[i], g.n_loc, torch.bfloat16, f"b[{LINEARS[i]}]")
    return W


def _partial_dtype(tables) -> tuple:
    """(ATP dtype code, torch dtype) shared by every partial buffer given."""
    dts = {t.dtype for tab in tables if tab for t in tab if t is not None}
    if len(dts) > 1:
        raise TypeError(f"partial buffers mix dtypes {sorted(map(str, dts))}")
    dt = dts.pop() if dts else torch.float32
    if dt not in (torch.float32, torch.bfloat16):
        raise TypeError(f"partial buffers must be float32 or bfloat16, not {dt}")
    return (ATP_F32 if dt == torch.float32 else ATP_BF16), dt


def _workspace(workspace):
    if workspace is None:
        return None, 0
    _on_device(workspace, "workspace")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def atp_block_fwd(m: atp_mesh, block_mode: int, tokens: int, h: int, chunks: int, w, b,
                  x_loc, attn_loc, partials, qkv, o, h_out, pre, z, workspace=None,
                  compute_stream=None, comm_stream=None, weight_layout: int = ATP_W_KN):
    """partials[i]: list of the red_size buffers of linear i's group (own
    entry written; all float32, or all bfloat16 for 16-bit partials), or
    None for a group of one."""
    G = block_geometry(m, block_mode, h)
    W = _weights(G, w, b, weight_layout)
    io = atp_block_fwd_io()
    io.partial_dtype, pdt = _partial_dtype(partials)
    io.x_loc, io.ldx = _mat(x_loc, tokens, G[0].k_loc, torch.bfloat16, "x_loc")
    io.attn_loc, io.lda = _mat(attn_loc, tokens, G[1].k_loc, torch.bfloat16, "attn_loc")
    keep = []
    for i, g in enumerate(G):
        if g.red_size > 1:
            if len(partials[i]) != g.red_size:
                raise ValueError(f"partials[{LINEARS[i]}] needs {g.red_size} buffers")
            tab, arr, ld = _ptr_table(partials[i], tokens, g.n_loc, f"partials[{LINEARS[i]}]",
                                      pdt)
            io.partials[i] = tab
            io.ldp[i] = ld
            keep.append(arr)
    io.qkv, io.ld_qkv = _mat(qkv, tokens, G[0].n_loc, torch.bfloat16, "qkv")
    io.o, io.ld_o = _mat(o, tokens, G[1].n_loc, torch.bfloat16, "o")
    io.h, io.ld_h = _mat(h_out, tokens, G[2].n_loc, torch.bfloat16, "h")
    pp, ldpre = _mat(pre, tokens, G[2].n_loc, torch.bfloat16, "pre")
    if ldpre != io.ld_h:
        raise ValueError("pre must share h's leading dimension")
    io.pre = pp
    io.z, io.ld_z = _mat(z, tokens, G[3].n_loc, torch.bfloat16, "z")
    wsp, wsb = _workspace(workspace)
    _check(load_library().atp_block_fwd(ctypes.byref(m), int(block_mode), int(tokens), int(h),
                                        int(chunks), ctypes.byref(W), ctypes.byref(io), wsp, wsb,
                                        _stream(compute_stream), _stream(comm_stream)))


def atp_block_bwd(m: atp_mesh, block_mode: int, tokens: int, h: int, chunks: int, w, b,
                  x_loc, attn_loc, h_act, pre, dz, dqkv, d_o, dx_partials, dh_pre, dx_qkv,
                  dx_fc1, d_attn, dw, db, workspace=None, compute_stream=None,
                  comm_stream=None, weight_layout: int = ATP_W_KN):
    """dx_partials[i]: list of the bwd_size buffers of linear i's backward
    group (own entry written; float32 or bfloat16), or None for a group of
    one.  dw[i] has the weight's layout and leading dimension."""
    G = block_geometry(m, block_mode, h)
    W = _weights(G, w, b, weight_layout)
    io = atp_block_bwd_io()
    io.partial_dtype, pdt = _partial_dtype(dx_partials)
    io.x_loc, io.ldx = _mat(x_loc, tokens, G[0].k_loc, torch.bfloat16, "x_loc")
    io.attn_loc, io.lda = _mat(attn_loc, tokens, G[1].k_loc, torch.bfloat16, "attn_loc")
    io.h, io.ld_h = _mat(h_act, tokens, G[2].n_loc, torch.bfloat16, "h")
    pp, ldpre = _mat(pre, tokens, G[2].n_loc, torch.bfloat16, "pre")
    dp, lddp = _mat(dh_pre, tokens, G[2].n_loc, torch.bfloat16, "dh_pre")
    if ldpre != io.ld_h or lddp != io.ld_h:
        raise ValueError("pre and dh_pre must share h's leading dimension")
    io.pre, io.dh_pre = pp, dp
    io.dz, io.ld_dz = _mat(dz, tokens, G[3].n_loc, torch.bfloat16, "dz")
    io.dqkv, io.ld_dqkv = _mat(dqkv, tokens, G[0].n_loc, torch.bfloat16, "dqkv")
    io.d_o, io.ld_do = _mat(d_o, tokens, G[1].n_loc, torch.bfloat16, "d_o")
    keep = []
    for i, g in enumerate(G):
        if g.bwd_size > 1:
            if len(dx_partials[i]) != g.bwd_size:
                raise ValueError(f"dx_partials[{LINEARS[i]}] needs {g.bwd_size} buffers")
            tab, arr, ld = _ptr_table(dx_partials[i], tokens, g.k_loc,
                                      f"dx_partials[{LINEARS[i]}]", pdt)
            io.dx_partials[i] = tab
            io.ld_dxp[i] = ld
            keep.append(arr)
    io.dx_qkv, io.ld_dx_qkv = _mat(dx_qkv, tokens, G[0].k_loc, torch.bfloat16, "dx_qkv")
    io.dx_fc1, io.ld_dx_fc1 = _mat(dx_fc1, tokens, G[2].k_loc, torch.bfloat16, "dx_fc1")
    io.d_attn, io.ld_d_attn = _mat(d_attn, tokens, G[1].k_loc, torch.bfloat16, "d_attn")
    for i, g in enumerate(G):
        r, c = (g.k_loc, g.n_loc) if weight_layout == ATP_W_KN else (g.n_loc, g.k_loc)
        p, ld = _mat(dw[i], r, c, torch.float32, f"dw[{LINEARS[i]}]")
        if ld != W.ldw[i]:
            raise ValueError(f"dw[{LINEARS[i]}] must share the weight's leading dimension")
        io.dw[i] = p
        io.db[i] = _vec(db[i], g.n_loc, torch.float32, f"db[{LINEARS[i]}]") if db else None
    wsp, wsb = _workspace(workspace)
    _check(load_library().atp_block_bwd(ctypes.byref(m), int(block_mode), int(tokens), int(h),
                                        int(chunks), ctypes.byref(W), ctypes.byref(io), wsp, wsb,
                                        _stream(compute_stream), _stream(comm_stream)))


def atp_profile_enable(on=True):
    """on: False/0 off, True/1 per kernel, 2 per kernel and problem shape."""
    load_library().atp_profile_enable(int(on) if not isinstance(on, bool) else (1 if on else 0))


def atp_profile_collect(max_records: int = 32):
    arr = (atp_kernel_stat * max_records)()
    n = load_library().atp_profile_collect(arr, max_records)
    if n < 0:
        raise AtpError(ATP_ERR_DEVICE, last_error())
    return [dict(name=arr[i].name.decode(), launches=arr[i].launches,
                 total_ms=arr[i].total_ms, flops=arr[i].flops, bytes=arr[i].bytes)
            for i in range(n)]


def atp_transpose_bf16(src, dst, stream=None):
    """dst[c, r] = src[r, c]; src [rows, cols] and dst [cols, rows] bf16 views."""
    rows, cols = src.shape
    sp, lds = _mat(src, rows, cols, torch.bfloat16, "src")
    dp_, ldd = _mat(dst, cols, rows, torch.bfloat16, "dst")
    _check(load_library().atp_transpose_bf16(int(rows), int(cols), sp, lds, dp_, ldd,
                                             _stream(stream)))


def attention_heads(m: atp_mesh, block_mode: int, h: int, heads: int):
    """(first head, number of heads) of the device's run of its QKV block's
    heads (block-local indices), and the block's head count."""
    first, count, per_block = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
    _check(load_library().atp_attention_heads(ctypes.byref(m), int(block_mode), int(h),
                                              int(heads), ctypes.byref(first),
                                              ctypes.byref(count), ctypes.byref(per_block)))
    return first.value, count.value, per_block.value


def _f32_scratch(t, n: int, name: str):
    """A contiguous float32 buffer of at least n values (checked before any
    other argument, so a short buffer never reaches a kernel)."""
    if t is None:
        return
    if t.dtype != torch.float32 or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous float32 tensor")
    if t.numel() < n:
        raise ValueError(f"{name}: {t.numel()} values, the device's heads need {n}")


def atp_attention_fwd(m: atp_mesh, block_mode: int, batch: int, seq: int, h: int, heads: int,
                      qkv, out, lse, stream=None):
    """The device's attention core: qkv [batch*seq, n_loc] bf16 (its reduced
    QKV block), out [batch*seq, >= n_loc/3] bf16 (the gathered out-proj
    input; the device's columns are written), lse [heads_dev, batch*seq] fp32."""
    T = batch * seq
    _, hd, _ = attention_heads(m, block_mode, h, heads)
    _f32_scratch(lse, hd * T, "lse")
    g = block_geometry(m, block_mode, h)[0]
    qp, ldq = _mat(qkv, T, g.n_loc, torch.bfloat16, "qkv")
    op, ldo = _mat(out, T, g.n_loc // 3, torch.bfloat16, "out")
    _check(load_library().atp_attention_fwd(ctypes.byref(m), int(block_mode), int(batch), int(seq),
                                            int(h), int(heads), qp, ldq, op, ldo,
                                            _ptr(lse, "lse"), _stream(stream)))


def atp_attention_bwd(m: atp_mesh, block_mode: int, batch: int, seq: int, h: int, heads: int,
                      qkv, out, lse, d_out, d_qkv, delta, stream=None):
    """Gradient of atp_attention_fwd: d_qkv (the QKV block's shape) receives
    dq, dk, dv of the device's heads; delta is fp32 scratch [heads_dev*T]."""
    T = batch * seq
    _, hd, _ = attention_heads(m, block_mode, h, heads)
    _f32_scratch(lse, hd * T, "lse")
    _f32_scratch(delta, hd * T, "delta")
    g = block_geometry(m, block_mode, h)[0]
    qp, ldq = _mat(qkv, T, g.n_loc, torch.bfloat16, "qkv")
    op, ldo = _mat(out, T, g.n_loc // 3, torch.bfloat16, "out")
    dop, lddo = _mat(d_out, T, g.n_loc // 3, torch.bfloat16, "d_out")
    dqp, lddq = _mat(d_qkv, T, g.n_loc, torch.bfloat16, "d_qkv")
    _check(load_library().atp_attention_bwd(ctypes.byref(m), int(block_mode), int(batch), int(seq),
                                            int(h), int(heads), qp, ldq, op, ldo,
                                            _ptr(lse, "lse"), dop, lddo, dqp, lddq,
                                            _ptr(delta, "delta"), _stream(stream)))


def atp_attention_bwd_noalloc(m: atp_mesh, block_mode: int, batch: int, seq: int, h: int,
                              heads: int, qkv, out, lse, d_out, d_qkv, stream=None):
    """atp_attention_bwd without caller scratch: delta lives in the library's
    own per-GPU array (for callers that cannot allocate)."""
    T = batch * seq
    _, hd, _ = attention_heads(m, block_mode, h, heads)
    _f32_scratch(lse, hd * T, "lse")
    g = block_geometry(m, block_mode, h)[0]
    qp, ldq = _mat(qkv, T, g.n_loc, torch.bfloat16, "qkv")
    op, ldo = _mat(out, T, g.n_loc // 3, torch.bfloat16, "out")
    dop, lddo = _mat(d_out, T, g.n_loc // 3, torch.bfloat16, "d_out")
    dqp, lddq = _mat(d_qkv, T, g.n_loc, torch.bfloat16, "d_qkv")
    _check(load_library().atp_attention_bwd_noalloc(
        ctypes.byref(m), int(block_mode), int(batch), int(seq), int(h), int(heads), qp, ldq, op,
        ldo, _ptr(lse, "lse"), dop, lddo, dqp, lddq, _stream(stream)))


# The calls below are made token by token, so their arguments are looked at once and
# quickly; what does not fit goes to _mat / _vec, which say what is wrong.
def _rows(t, rows: int, cols: int, name: str, dev: int, dtype=torch.bfloat16):
    """(pointer, ld) of a matrix on device dev (None stays NULL)."""
    if t is None:
        return None, 0
    if t.dtype is dtype and t.get_device() == dev and t.dim() == 2:
        r, c = t.shape
        s0, s1 = t.stride()
        if r >= rows and c >= cols and (s1 == 1 or c <= 1):
            return t.data_ptr(), (s0 if r > 1 else max(c, cols))
    return _mat(t, rows, cols, dtype, name)


def _list(t, n: int, name: str, dev: int, dtype=torch.int32):
    """Pointer of a contiguous vector of at least n values (None stays NULL)."""
    if t is None:
        return None
    if t.dtype is dtype and t.get_device() == dev and t.numel() >= n and t.is_contiguous():
        return t.data_ptr()
    return _vec(t, n, dtype, name)


def _bytes(workspace, dev: int):
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace: needs contiguous memory")    # nbytes would count other bytes
    if workspace is not None and workspace.get_device() == dev:
        return workspace.data_ptr(), workspace.nbytes
    return _workspace(workspace)


class _Held:
    """A C struct and the tensors it points into."""

    def _hold(self, struct, **tensors):
        self.c = struct
        self._tensors = [(t, name) for name, t in tensors.items() if t is not None]
        self._ref = ctypes.byref(struct)

    def ref(self, dev: int):
        for t, name in self._tensors:
            if t.get_device() != dev:
                _on_device(t, name)
        return self._ref


class qk_norm_rope(_Held):
    """Parameters of the query/key norms with the position rotation
    (atp_qk_norm_rope in include/atp.h); keeps its tensors alive.  q_weight,
    k_weight: bf16 [128]; inv_freq: float32 [rotary_dims / 2]."""

    def __init__(self, q_weight=None, k_weight=None, eps: float = 1e-6, inv_freq=None,
                 rotary_dims: int = 0, interleaved: bool = False, norm: bool = True):
        rotary_dims = int(rotary_dims)
        if rotary_dims > 0 and inv_freq is None:
            raise ValueError("inv_freq: a rotation needs its frequencies")
        self._hold(atp_qk_norm_rope(
            _vec(q_weight, HEAD_DIM, torch.bfloat16, "q_weight"),
            _vec(k_weight, HEAD_DIM, torch.bfloat16, "k_weight"),
            _vec(inv_freq, max(0, rotary_dims) // 2, torch.float32, "inv_freq"), float(eps),
            int(norm), rotary_dims, int(interleaved)),
            q_weight=q_weight, k_weight=k_weight, inv_freq=inv_freq)


class kv_cache(_Held):
    """One layer's cache: pages, a contiguous bf16 tensor [n_pages, 2, kv_heads,
    page_size, 128] (keys, then values)."""

    def __init__(self, pages: torch.Tensor):
        if pages.dtype != torch.bfloat16:
            raise TypeError(f"pages: expected torch.bfloat16, got {pages.dtype}")
        if (pages.dim() != 5 or pages.size(1) != 2 or pages.size(4) != HEAD_DIM or
                not pages.is_contiguous()):
            raise ValueError("pages: needs a contiguous [n_pages, 2, kv_heads, page_size, "
                             f"{HEAD_DIM}] tensor, got {tuple(pages.shape)}")
        self.n_pages, _, self.kv_heads, self.page_size, _ = pages.shape
        self._hold(atp_kv_cache(_ptr(pages, "pages"), self.n_pages, self.kv_heads,
                                self.page_size), pages=pages)


class kv_batch(_Held):
    """A batch of sequences over a cache: table int32 [n_seqs, max_pages], ctx
    int32 [n_seqs], cu_new int32 [n_seqs + 1] (either may be None for the calls
    that do not read it).  The tensors are read when a call's kernels run."""

    def __init__(self, table: torch.Tensor, ctx=None, cu_new=None):
        if table.dtype != torch.int32:
            raise TypeError(f"table: expected torch.int32, got {table.dtype}")
        if table.dim() != 2 or (table.size(1) > 1 and table.stride(1) != 1):
            raise ValueError("table: needs a 2-D row-major tensor")
        self.n_seqs, self.max_pages = table.shape
        ld = table.stride(0) if self.n_seqs > 1 else self.max_pages
        self._hold(atp_kv_batch(_ptr(table, "table"), ld, self.max_pages, self.n_seqs,
                                _vec(ctx, self.n_seqs, torch.int32, "ctx"),
                                _vec(cu_new, self.n_seqs + 1, torch.int32, "cu_new")),
                   table=table, ctx=ctx, cu_new=cu_new)


def atp_qk_norm_rope_fwd(batch: int, seq: int, kv_heads: int, group: int, params: qk_norm_rope,
                         qkv, out, positions=None, stream=None):
    """qkv, out: bf16 [batch*seq, kv_heads*(group+2)*128] (out may be qkv);
    positions: int32 [batch*seq], or None for t % seq."""
    dev = torch.cuda.current_device()
    T, cols = batch * seq, kv_heads * (group + 2) * HEAD_DIM
    xp, ldx = _rows(qkv, T, cols, "qkv", dev)
    op, ldo = _rows(out, T, cols, "out", dev)
    _check(load_library().atp_qk_norm_rope_fwd(
        int(batch), int(seq), int(kv_heads), int(group), params.ref(dev),
        _list(positions, T, "positions", dev), xp, ldx, op, ldo, _stream(stream, dev)))


def atp_qk_norm_rope_workspace_bytes(tokens: int) -> int:
    return load_library().atp_qk_norm_rope_workspace_bytes(int(tokens))


def atp_qk_norm_rope_bwd(batch: int, seq: int, kv_heads: int, group: int, params: qk_norm_rope,
                         qkv, d_out, d_qkv, dq_weight=None, dk_weight=None, workspace=None,
                         positions=None, stream=None):
    """Gradient of atp_qk_norm_rope_fwd: d_qkv (may be d_out) and, where
    given, the weights' gradients (float32 [128]; they need a workspace of
    atp_qk_norm_rope_workspace_bytes(batch*seq) bytes)."""
    dev = torch.cuda.current_device()
    T, cols = batch * seq, kv_heads * (group + 2) * HEAD_DIM
    xp, ldx = _rows(qkv, T, cols, "qkv", dev)
    gp, ldg = _rows(d_out, T, cols, "d_out", dev)
    dp_, ldd = _rows(d_qkv, T, cols, "d_qkv", dev)
    wsp, wsb = _bytes(workspace, dev)
    _check(load_library().atp_qk_norm_rope_bwd(
        int(batch), int(seq), int(kv_heads), int(group), params.ref(dev),
        _list(positions, T, "positions", dev), xp, ldx, gp, ldg, dp_, ldd,
        _list(dq_weight, HEAD_DIM, "dq_weight", dev, torch.float32),
        _list(dk_weight, HEAD_DIM, "dk_weight", dev, torch.float32), wsp, wsb,
        _stream(stream, dev)))


def atp_qk_norm_rope_cache(cache: kv_cache, batch: kv_batch, tokens: int, group: int,
                           params: qk_norm_rope, qkv, q, positions=None, stream=None):
    """The step's rows qkv [tokens, kv_heads*(group+2)*128]: queries into q
    [tokens, kv_heads*group*128], keys and values into the cache."""
    dev = torch.cuda.current_device()
    xp, ldx = _rows(qkv, tokens, cache.kv_heads * (group + 2) * HEAD_DIM, "qkv", dev)
    qp, ldq = _rows(q, tokens, cache.kv_heads * group * HEAD_DIM, "q", dev)
    _check(load_library().atp_qk_norm_rope_cache(
        cache.ref(dev), batch.ref(dev), int(tokens), int(group), params.ref(dev),
        _list(positions, tokens, "positions", dev), xp, ldx, qp, ldq, _stream(stream, dev)))


def atp_cache_workspace_bytes(n_pages: int, n_seqs: int) -> int:
    return load_library().atp_cache_workspace_bytes(int(n_pages), int(n_seqs))


def _refs(refs, dev: int):
    if refs is None:
        raise ValueError("refs: needs the pages' reference counts")
    return refs.numel(), _list(refs, refs.numel(), "refs", dev)


def atp_cache_reserve(page_size: int, refs, batch: kv_batch, missing, copy_src, copy_dst,
                      copy_rows, workspace, stream=None):
    """Pages for every sequence's new tokens; refs: int32 [n_pages]; missing,
    copy_src, copy_dst, copy_rows: int32 [n_seqs], written."""
    dev = torch.cuda.current_device()
    n, rp = _refs(refs, dev)
    wsp, wsb = _bytes(workspace, dev)
    _check(load_library().atp_cache_reserve(
        n, int(page_size), rp, batch.ref(dev), _list(missing, batch.n_seqs, "missing", dev),
        _list(copy_src, batch.n_seqs, "copy_src", dev),
        _list(copy_dst, batch.n_seqs, "copy_dst", dev),
        _list(copy_rows, batch.n_seqs, "copy_rows", dev), wsp, wsb, _stream(stream, dev)))


def atp_cache_fork(page_size: int, refs, batch: kv_batch, parents, children, done, stream=None):
    """children[f] takes over parents[f]'s pages (int32 lists of one length);
    done: int32, 0 or 1 (refused) per fork."""
    dev = torch.cuda.current_device()
    n, rp = _refs(refs, dev)
    forks = parents.numel()
    _check(load_library().atp_cache_fork(
        n, int(page_size), rp, batch.ref(dev), forks, _list(parents, forks, "parents", dev),
        _list(children, forks, "children", dev), _list(done, forks, "done", dev),
        _stream(stream, dev)))


def atp_cache_release(page_size: int, refs, batch: kv_batch, keep, stream=None):
    """Gives back the pages behind the first keep[s] >= 0 tokens of sequence s."""
    dev = torch.cuda.current_device()
    n, rp = _refs(refs, dev)
    _check(load_library().atp_cache_release(
        n, int(page_size), rp, batch.ref(dev), _list(keep, batch.n_seqs, "keep", dev),
        _stream(stream, dev)))


def atp_cache_copy_pages(cache: kv_cache, src, dst, rows=None, stream=None):
    """The first rows[i] tokens (all for None) of page src[i] to page dst[i]."""
    dev = torch.cuda.current_device()
    n = src.numel()
    _check(load_library().atp_cache_copy_pages(
        cache.ref(dev), n, _list(src, n, "src", dev), _list(dst, n, "dst", dev),
        _list(rows, n, "rows", dev), _stream(stream, dev)))


def atp_cache_compact(cache: kv_cache, batch: kv_batch, cu_keep, keep, moved=None, stream=None):
    """Moves tokens ctx[s] + keep[cu_keep[s] + i] to places ctx[s] + i; moved:
    int32 [n_seqs], rows moved or -1 (refused)."""
    dev = torch.cuda.current_device()
    n = keep.numel()
    _check(load_library().atp_cache_compact(
        cache.ref(dev), batch.ref(dev), _list(cu_keep, batch.n_seqs + 1, "cu_keep", dev),
        _list(keep, n, "keep", dev), n, _list(moved, batch.n_seqs, "moved", dev),
        _stream(stream, dev)))


def atp_attention_cache_workspace_bytes(kv_heads: int, group: int, max_new: int) -> int:
    return load_library().atp_attention_cache_workspace_bytes(int(kv_heads), int(group),
                                                              int(max_new))


def atp_attention_cache_fwd(cache: kv_cache, batch: kv_batch, tokens: int, group: int,
                            max_new: int, q, out, lse=None, tree_mask=None, workspace=None,
                            stream=None):
    """Attention of the step's rows q over the cache into out (both bf16
    [tokens, kv_heads*group*128]); lse: float32 [kv_heads*group, tokens];
    tree_mask: int64 or uint64 [tokens, words], contiguous; workspace:
    atp_attention_cache_workspace_bytes(kv_heads, group, max_new) bytes."""
    dev = torch.cuda.current_device()
    cols = cache.kv_heads * group * HEAD_DIM
    qp, ldq = _rows(q, tokens, cols, "q", dev)
    op, ldo = _rows(out, tokens, cols, "out", dev)
    words, mp = 0, None
    if tree_mask is not None:
        if tree_mask.dtype not in (torch.int64, torch.uint64):
            raise TypeError(f"tree_mask: expected 64-bit words, got {tree_mask.dtype}")
        if tree_mask.dim() != 2 or tree_mask.size(0) < tokens or not tree_mask.is_contiguous():
            raise ValueError(f"tree_mask: needs a contiguous [{tokens}, words] tensor")
        words, mp = tree_mask.size(1), _ptr(tree_mask, "tree_mask")
    wsp, wsb = _bytes(workspace, dev)
    _check(load_library().atp_attention_cache_fwd(
        cache.ref(dev), batch.ref(dev), int(tokens), int(group), int(max_new), qp, ldq, mp, words,
        op, ldo, _list(lse, cache.kv_heads * group * tokens, "lse", dev, torch.float32), wsp, wsb,
        _stream(stream, dev)))


# ------------------------------------------------ around the layers, for training
_FLOATS = {torch.float32: ATP_F32, torch.bfloat16: ATP_BF16}


def _float_code(t, name: str) -> int:
    code = _FLOATS.get(t.dtype)
    if code is None:
        raise TypeError(f"{name}: expected torch.float32 or torch.bfloat16, got {t.dtype}")
    return code


def _width(t, name: str) -> int:
    """Columns of a matrix that gives a call its row width."""
    if t.dim() != 2:
        raise ValueError(f"{name}: needs a 2-D row-major tensor")
    return t.shape[1]


def atp_embedding_fwd(tokens: int, ids, table, out, scale: float = 1.0, vocab_off: int = 0,
                      stream=None):
    """out[t] = scale * table[ids[t] - vocab_off], zeros for tokens of other
    devices.  ids: int32 [tokens]; table: bf16 [vocab_loc, cols]; out: float32 or
    bf16 [tokens, cols]."""
    dev = torch.cuda.current_device()
    cols, vocab = _width(table, "table"), table.shape[0]
    tp, ldt = _rows(table, vocab, cols, "table", dev)
    code = _float_code(out, "out")
    op, ldo = _rows(out, tokens, cols, "out", dev, out.dtype)
    _check(load_library().atp_embedding_fwd(
        int(tokens), _list(ids, tokens, "ids", dev), vocab, int(vocab_off), cols, tp, ldt,
        float(scale), op, code, ldo, _stream(stream, dev)))


def atp_embedding_workspace_bytes(tokens: int, vocab_loc: int, cols: int) -> int:
    return load_library().atp_embedding_workspace_bytes(int(tokens), int(vocab_loc), int(cols))


def atp_embedding_bwd(tokens: int, ids, dy, dtable, workspace, scale: float = 1.0,
                      vocab_off: int = 0, accumulate: bool = False, stream=None):
    """dtable[v] (float32 [vocab_loc, cols]) = or, with accumulate, += scale * the
    sum of dy (bf16 [tokens, cols]) over the tokens with that id; workspace:
    atp_embedding_workspace_bytes(tokens, vocab_loc, cols) bytes."""
    dev = torch.cuda.current_device()
    cols, vocab = _width(dtable, "dtable"), dtable.shape[0]
    yp, ldy = _rows(dy, tokens, cols, "dy", dev)
    tp, ldt = _rows(dtable, vocab, cols, "dtable", dev, torch.float32)
    wsp, wsb = _bytes(workspace, dev)
    _check(load_library().atp_embedding_bwd(
        int(tokens), _list(ids, tokens, "ids", dev), vocab, int(vocab_off), cols, yp, ldy,
        float(scale), tp, ldt, int(accumulate), wsp, wsb, _stream(stream, dev)))


class layer_norm(_Held):
    """Parameters of a layer norm (atp_layer_norm in include/atp.h); keeps its
    tensors alive.  weight, bias: bf16, this device's columns, or None."""

    def __init__(self, weight=None, bias=None, eps: float = 1e-5):
        self.cols = None
        for t, name in ((weight, "weight"), (bias, "bias")):
            if t is None:
                continue
            if self.cols not in (None, t.numel()):
                raise ValueError(f"{name}: {t.numel()} values, weight has {self.cols}")
            self.cols = t.numel()
        self._hold(atp_layer_norm(
            _vec(weight, self.cols or 0, torch.bfloat16, "weight"),
            _vec(bias, self.cols or 0, torch.bfloat16, "bias"), float(eps)),
            weight=weight, bias=bias)

    def of(self, cols: int, dev: int):
        if self.cols not in (None, cols):
            raise ValueError(f"norm: {self.cols} parameters for rows of {cols}")
        return self.ref(dev)


def _row_tables(ts, tokens: int, name: str, dev: int):
    """(red_size, host array) of a group's float32 [tokens, 2] tables."""
    if ts is None:
        return 1, None
    arr = (ctypes.c_void_p * max(1, len(ts)))()
    for j, t in enumerate(ts):
        arr[j] = _list(t, 2 * tokens, f"{name}[{j}]", dev, torch.float32)
    return len(ts), arr


def _summed(tokens: int, x, add, x_out, dev: int):
    """Sizes and arguments of the sum that a norm is of."""
    cols, code = _width(x, "x"), _float_code(x, "x")
    xp, ldx = _rows(x, tokens, cols, "x", dev, x.dtype)
    if add is None and x_out is None:
        return cols, code, (xp, ldx, None, 0, None, 0)
    return cols, code, (xp, ldx, *_rows(add, tokens, cols, "add", dev),
                        *_rows(x_out, tokens, cols, "x_out", dev, x.dtype))


def atp_layer_norm_stats(tokens: int, x, stats, add=None, x_out=None, stream=None):
    """x_out = x + add (both or neither), and the statistics of this device's
    columns of it into stats, float32 [tokens, 2]."""
    dev = torch.cuda.current_device()
    cols, code, args = _summed(tokens, x, add, x_out, dev)
    _check(load_library().atp_layer_norm_stats(
        int(tokens), cols, code, *args, _list(stats, 2 * tokens, "stats", dev, torch.float32),
        _stream(stream, dev)))


def atp_layer_norm_fwd(tokens: int, norm: layer_norm, x, y, mean, rstd, add=None, x_out=None,
                       stats=None, stream=None):
    """y (bf16) = the norm of x (float32 or bf16 [tokens, cols]) or of x_out = x +
    add; mean, rstd: float32 [tokens], written.  stats: the group's statistics
    (a list of float32 [tokens, 2]) where the rows' columns lie on several devices."""
    dev = torch.cuda.current_device()
    cols, code, args = _summed(tokens, x, add, x_out, dev)
    n, tab = _row_tables(stats, tokens, "stats", dev)
    yp, ldy = _rows(y, tokens, cols, "y", dev)
    _check(load_library().atp_layer_norm_fwd(
        int(tokens), cols, code, norm.of(cols, dev), *args, n, tab, yp, ldy,
        _list(mean, tokens, "mean", dev, torch.float32),
        _list(rstd, tokens, "rstd", dev, torch.float32), _stream(stream, dev)))


def _normed(tokens: int, norm, x, mean, rstd, dy, dev: int):
    """Row width and the arguments that both calls of the backward share."""
    cols, code = _width(x, "x"), _float_code(x, "x")
    return cols, (int(tokens), cols, code, norm.of(cols, dev),
                  *_rows(x, tokens, cols, "x", dev, x.dtype),
                  _list(mean, tokens, "mean", dev, torch.float32),
                  _list(rstd, tokens, "rstd", dev, torch.float32),
                  *_rows(dy, tokens, cols, "dy", dev))


def atp_layer_norm_bwd_sums(tokens: int, norm: layer_norm, x, mean, rstd, dy, sums, stream=None):
    """The row sums of this device's columns that the others need, into sums
    (float32 [tokens, 2])."""
    dev = torch.cuda.current_device()
    _, args = _normed(tokens, norm, x, mean, rstd, dy, dev)
    _check(load_library().atp_layer_norm_bwd_sums(
        *args, _list(sums, 2 * tokens, "sums", dev, torch.float32), _stream(stream, dev)))


def atp_layer_norm_workspace_bytes(tokens: int, cols: int) -> int:
    return load_library().atp_layer_norm_workspace_bytes(int(tokens), int(cols))


def atp_layer_norm_bwd(tokens: int, norm: layer_norm, x, mean, rstd, dy, dx, d_res=None,
                       d_add=None, sums=None, dweight=None, dbias=None, workspace=None,
                       stream=None):
    """Gradient of atp_layer_norm_fwd: dx (x's type; may be d_res, the gradient that
    goes past the norm), d_add (bf16 copy of dx), dweight, dbias (float32 [cols]; they
    need a workspace of atp_layer_norm_workspace_bytes(tokens, cols) bytes).  x: the
    normed values; sums: the group's row sums, as stats in the forward."""
    dev = torch.cuda.current_device()
    cols, args = _normed(tokens, norm, x, mean, rstd, dy, dev)
    rp, ldr = _rows(d_res, tokens, cols, "d_res", dev, x.dtype)
    n, tab = _row_tables(sums, tokens, "sums", dev)
    dp_, ldd = _rows(dx, tokens, cols, "dx", dev, x.dtype)
    ap, lda = _rows(d_add, tokens, cols, "d_add", dev)
    wsp, wsb = _bytes(workspace, dev)
    _check(load_library().atp_layer_norm_bwd(
        *args, rp, ldr, n, tab, dp_, ldd, ap, lda,
        _list(dweight, cols, "dweight", dev, torch.float32),
        _list(dbias, cols, "dbias", dev, torch.float32), wsp, wsb, _stream(stream, dev)))


class attention_docs(_Held):
    """Documents of packed rows and what is done to their scores
    (atp_attention_docs in include/atp.h): cu_docs int32 [n_docs + 1], prefix int32
    [n_docs] or None, slopes float32 [query heads] or None, cap (0: none).  The
    tensors are read when a call's kernels run."""

    def __init__(self, cu_docs: torch.Tensor, prefix=None, slopes=None, cap: float = 0.0):
        if cu_docs.numel() < 1:
            raise ValueError("cu_docs: needs n_docs + 1 values")
        self.n_docs = cu_docs.numel() - 1
        self.heads = None if slopes is None else slopes.numel()
        self._hold(atp_attention_docs(
            _vec(cu_docs, self.n_docs + 1, torch.int32, "cu_docs"),
            _vec(prefix, self.n_docs, torch.int32, "prefix"),
            _vec(slopes, self.heads or 0, torch.float32, "slopes"), self.n_docs, float(cap)),
            cu_docs=cu_docs, prefix=prefix, slopes=slopes)

    def of(self, heads: int, dev: int):
        if self.heads is not None and self.heads < heads:
            raise ValueError(f"slopes: {self.heads} for {heads} query heads")
        return self.ref(dev)


def atp_attention_docs_fwd(tokens: int, kv_heads: int, group: int, docs: attention_docs, qkv, out,
                           lse, stream=None):
    """Attention within documents: qkv bf16 [tokens, kv_heads*(group+2)*128], out bf16
    [tokens, kv_heads*group*128], lse float32 [kv_heads*group, tokens]."""
    dev = torch.cuda.current_device()
    heads = kv_heads * group
    qp, ldq = _rows(qkv, tokens, kv_heads * (group + 2) * HEAD_DIM, "qkv", dev)
    op, ldo = _rows(out, tokens, heads * HEAD_DIM, "out", dev)
    _check(load_library().atp_attention_docs_fwd(
        int(tokens), int(kv_heads), int(group), docs.of(heads, dev), qp, ldq, op, ldo,
        _list(lse, heads * tokens, "lse", dev, torch.float32), _stream(stream, dev)))


def atp_attention_docs_workspace_bytes(tokens: int, kv_heads: int, group: int) -> int:
    return load_library().atp_attention_docs_workspace_bytes(int(tokens), int(kv_heads),
                                                             int(group))


def atp_attention_docs_bwd(tokens: int, kv_heads: int, group: int, docs: attention_docs, qkv, out,
                           lse, d_out, d_qkv, workspace, stream=None):
    """Gradient of atp_attention_docs_fwd into d_qkv (qkv's shape); workspace:
    atp_attention_docs_workspace_bytes(tokens, kv_heads, group) bytes."""
    dev = torch.cuda.current_device()
    heads, cols = kv_heads * group, kv_heads * (group + 2) * HEAD_DIM
    qp, ldq = _rows(qkv, tokens, cols, "qkv", dev)
    op, ldo = _rows(out, tokens, heads * HEAD_DIM, "out", dev)
    gp, ldg = _rows(d_out, tokens, heads * HEAD_DIM, "d_out", dev)
    dp_, ldd = _rows(d_qkv, tokens, cols, "d_qkv", dev)
    wsp, wsb = _bytes(workspace, dev)
    _check(load_library().atp_attention_docs_bwd(
        int(tokens), int(kv_heads), int(group), docs.of(heads, dev), qp, ldq, op, ldo,
        _list(lse, heads * tokens, "lse", dev, torch.float32), gp, ldg, dp_, ldd, wsp, wsb,
        _stream(stream, dev)))


# a, b: memory of rows `pitch` bytes apart, (begin, end, rows, pitch, width, ...).
def _meet(a, b) -> bool:
    """Whether a byte belongs to both (columns of one matrix interleave without)."""
    begin, _, rows, pitch, width = a[:5]
    if rows > 1 and b[2] > 1 and pitch != b[3]:
        if rows > b[2]:
            return _meet(b, a)
        return any(_meet((begin + k * pitch, 0, 1, pitch, width), b) for k in range(rows))
    # row k + j of a meets row j of b where k pitch is inside the rows' widths of their distance
    pitch = pitch if rows > 1 else b[3]
    far = b[0] - begin
    least = max((far - width) // pitch + 1, 1 - b[2])
    most = min(-((-far - b[4]) // pitch) - 1, rows - 1)
    return least <= most


class grad_list:
    """Gradients and where their clipped values go (an array of atp_grad; keeps the
    tensors alive).  src: float32 or bf16 tensors, contiguous or 2-D with gaps between
    rows; dst: as many of the same sizes, or None for src itself."""

    def __init__(self, src: Sequence[torch.Tensor], dst: Optional[Sequence] = None):
        dst = list(src) if dst is None else list(dst)
        self._tensors = (list(src), dst)
        if len(dst) != len(self._tensors[0]):
            raise ValueError(f"dst: {len(dst)} tensors for {len(self._tensors[0])} gradients")
        self.n = len(dst)
        self.device = None
        self.c = (atp_grad * max(1, self.n))()
        spans = []
        for i, (s, d) in enumerate(zip(*self._tensors)):
            if s.numel() != d.numel():
                raise ValueError(f"dst[{i}]: {tuple(d.shape)} for {tuple(s.shape)}")
            rows, cols = self._matrix(s, f"src[{i}]")
            if self._matrix(d, f"dst[{i}]") != (rows, cols):
                # one of them has gaps between its rows: both are taken as matrices
                if s.shape != d.shape or s.dim() != 2:
                    raise ValueError(f"dst[{i}]: {tuple(d.shape)} for {tuple(s.shape)}")
                rows, cols = s.shape
            g = self.c[i]
            for t, side in ((s, "src"), (d, "dst")):
                _on_device(t, f"{side}[{i}]")
                setattr(g, side, t.data_ptr())
                gaps = t.dim() == 2 and rows == t.size(0) and rows > 1
                setattr(g, "ld_" + side, t.stride(0) if gaps else cols)
                setattr(g, side + "_dtype", _float_code(t, f"{side}[{i}]"))
                if t.numel():
                    begin, size = t.data_ptr(), t.element_size()
                    pitch, width = getattr(g, "ld_" + side) * size, cols * size
                    spans.append((begin, begin + (rows - 1) * pitch + width, rows, pitch, width,
                                  i, side))
            g.rows, g.cols = rows, cols
            self.device = s.device.index
        # a result must not land in another gradient or result
        spans.sort()
        reach, last = [], 0              # what ends behind the next one's begin
        for span in spans:
            reach = [r for r in reach if r[1] > span[0]] if span[0] < last else []
            for r in reach:
                if r[5] != span[5] and "dst" in (r[6], span[6]) and _meet(r, span):
                    raise ValueError(f"{r[6]}[{r[5]}] and {span[6]}[{span[5]}] overlap")
            reach.append(span)
            last = max(last, span[1])

    @staticmethod
    def _matrix(t: torch.Tensor, name: str):
        if t.is_contiguous():
            return 1, t.numel()
        if t.dim() == 2 and (t.size(1) <= 1 or t.stride(1) == 1) and t.stride(0) >= t.size(1):
            return tuple(t.shape)
        raise ValueError(f"{name}: needs a contiguous tensor or rows with gaps")

    def at(self, dev: int):
        if self.n and self.device != dev:
            raise ValueError(f"gradients: on cuda:{self.device}, but the current device is "
                             f"cuda:{dev}")
        return self.c


def atp_grad_workspace_bytes(grads: grad_list) -> int:
    return load_library().atp_grad_workspace_bytes(grads.n, grads.c)


def atp_grad_sq_sum(grads: grad_list, total, workspace=None, stream=None):
    """total (float64, one value) = the sum of the squares of all gradients;
    workspace: atp_grad_workspace_bytes(grads) bytes."""
    dev = torch.cuda.current_device()
    wsp, wsb = _bytes(workspace, dev)
    _check(load_library().atp_grad_sq_sum(
        grads.n, grads.at(dev), _list(total, 1, "total", dev, torch.float64), wsp, wsb,
        _stream(stream, dev)))


def atp_grad_clip(grads: grad_list, sums, norm, max_norm: float, scale: float = 1.0, stream=None):
    """Scales the gradients into their destinations by scale * min(1, max_norm / norm)
    with norm = scale * sqrt(sum of `sums`), a list of the devices' totals (float64, one
    value each); norm: float32 [2], receives the norm and the factor."""
    dev = torch.cuda.current_device()
    arr = (ctypes.c_void_p * max(1, len(sums)))()
    for j, t in enumerate(sums):
        arr[j] = _list(t, 1, f"sums[{j}]", dev, torch.float64)
    _check(load_library().atp_grad_clip(
        grads.n, grads.at(dev), len(sums), arr, float(scale), float(max_norm),
        _list(norm, 2, "norm", dev, torch.float32), _stream(stream, dev)))


def _attn_weights(G, w, b, layout: int):
    """Weights of QKV and out-proj (entries 0 and 1) for the attention block."""
    W = atp_block_weights()
    W.layout = int(layout)
    for i in range(2):
        g = G[i]
        r, c = (g.k_loc, g.n_loc) if layout == ATP_W_KN else (g.n_loc, g.k_loc)
        W.w[i], W.ldw[i] = _mat(w[i], r, c, torch.bfloat16, f"w[{LINEARS[i]}]")
        W.b[i] = _vec(b[i], g.n_loc, torch.bfloat16, f"b[{LINEARS[i]}]")
    return W


def atp_attention_block_fwd(m: atp_mesh, block_mode: int, batch: int, seq: int, h: int,
                            heads: int, chunks: int, w, b, x_loc, qkv_partials, qkv, attn, lse,
                            o_partials, o, workspace=None, compute_stream=None, comm_stream=None,
                            weight_layout: int = ATP_W_KN):
    """The device's attention block: QKV -> its heads' attention -> out-proj.
    w, b: [qkv, out] weights and biases; qkv_partials / o_partials: the
    groups' buffers (own entry written) or None for a group of one; attn: the
    gathered out-proj input, whose other members' columns must be filled;
    workspace: an optional uint8 device buffer (atp_block_workspace_bytes
    covers it)."""
    T = batch * seq
    G = block_geometry(m, block_mode, h)
    _, hd, _ = attention_heads(m, block_mode, h, heads)
    _f32_scratch(lse, hd * T, "lse")
    W = _attn_weights(G, w, b, weight_layout)
    io = atp_attn_block_fwd_io()
    io.partial_dtype, pdt = _partial_dtype([qkv_partials, o_partials])
    io.x_loc, io.ldx = _mat(x_loc, T, G[0].k_loc, torch.bfloat16, "x_loc")
    keep = []
    for name, parts, g, attr in (("qkv_partials", qkv_partials, G[0], "qkv"),
                                 ("o_partials", o_partials, G[1], "o")):
        if g.red_size > 1:
            if len(parts) != g.red_size:
                raise ValueError(f"{name} needs {g.red_size} buffers")
            tab, arr, ld = _ptr_table(parts, T, g.n_loc, name, pdt)
            setattr(io, name, tab)
            setattr(io, "ldp_" + attr, ld)
            keep.append(arr)
    io.qkv, io.ld_qkv = _mat(qkv, T, G[0].n_loc, torch.bfloat16, "qkv")
    io.attn, io.ld_attn = _mat(attn, T, G[1].k_loc, torch.bfloat16, "attn")
    io.lse = _ptr(lse, "lse")
    io.o, io.ld_o = _mat(o, T, G[1].n_loc, torch.bfloat16, "o")
    wsp, wsb = _workspace(workspace)
    _check(load_library().atp_attention_block_fwd(
        ctypes.byref(m), int(block_mode), int(batch), int(seq), int(h), int(heads), int(chunks),
        ctypes.byref(W), ctypes.byref(io), wsp, wsb, _stream(compute_stream),
        _stream(comm_stream)))


def atp_attention_block_bwd(m: atp_mesh, block_mode: int, batch: int, seq: int, h: int,
                            heads: int, chunks: int, w, b, x_loc, qkv, attn, lse, d_o,
                            d_attn_partials, d_attn, delta, d_qkv, dx_partials, dx, dw, db,
                            workspace=None, compute_stream=None, comm_stream=None,
                            weight_layout: int = ATP_W_KN):
    """Backward of atp_attention_block_fwd.  d_qkv: the QKV block's
    gradient, whose other members' columns must be filled; dw, db: [qkv, out]
    (dw in the weights' layout, db entries may be None); workspace: an
    optional uint8 device buffer (atp_block_workspace_bytes covers it)."""
    T = batch * seq
    G = block_geometry(m, block_mode, h)
    _, hd, _ = attention_heads(m, block_mode, h, heads)
    _f32_scratch(lse, hd * T, "lse")
    _f32_scratch(delta, hd * T, "delta")
    W = _attn_weights(G, w, b, weight_layout)
    io = atp_attn_block_bwd_io()
    io.partial_dtype, pdt = _partial_dtype([d_attn_partials, dx_partials])
    io.x_loc, io.ldx = _mat(x_loc, T, G[0].k_loc, torch.bfloat16, "x_loc")
    io.qkv, io.ld_qkv = _mat(qkv, T, G[0].n_loc, torch.bfloat16, "qkv")
    io.attn, io.ld_attn = _mat(attn, T, G[1].k_loc, torch.bfloat16, "attn")
    io.lse = _ptr(lse, "lse")
    io.d_o, io.ld_do = _mat(d_o, T, G[1].n_loc, torch.bfloat16, "d_o")
    keep = []
    for name, parts, g, ldname in (("d_attn_partials", d_attn_partials, G[1], "ldp_da"),
                                   ("dx_partials", dx_partials, G[0], "ldp_dx")):
        if g.bwd_size > 1:
            if len(parts) != g.bwd_size:
                raise ValueError(f"{name} needs {g.bwd_size} buffers")
            tab, arr, ld = _ptr_table(parts, T, g.k_loc, name, pdt)
            setattr(io, name, tab)
            setattr(io, ldname, ld)
            keep.append(arr)
    io.d_attn, io.ld_d_attn = _mat(d_attn, T, G[1].k_loc, torch.bfloat16, "d_attn")
    io.delta = _ptr(delta, "delta")
    io.d_qkv, io.ld_dqkv = _mat(d_qkv, T, G[0].n_loc, torch.bfloat16, "d_qkv")
    io.dx, io.ld_dx = _mat(dx, T, G[0].k_loc, torch.bfloat16, "dx")
    for i in range(2):
        g = G[i]
        r, c = (g.k_loc, g.n_loc) if weight_layout == ATP_W_KN else (g.n_loc, g.k_loc)
        p, ld = _mat(dw[i], r, c, torch.float32, f"dw[{LINEARS[i]}]")
        if ld != W.ldw[i]:
            raise ValueError(f"dw[{LINEARS[i]}] must share the weight's leading dimension")
        io.dw[i] = p
        io.db[i] = _vec(db[i], g.n_loc, torch.float32, f"db[{LINEARS[i]}]") if db else None
    wsp, wsb = _workspace(workspace)
    _check(load_library().atp_attention_block_bwd(
        ctypes.byref(m), int(block_mode), int(batch), int(seq), int(h), int(heads), int(chunks),
        ctypes.byref(W), ctypes.byref(io), wsp, wsb, _stream(compute_stream),
        _stream(comm_stream)))


# ---------------------------------------------------------------------------
# Mesh planner (host only)
# ---------------------------------------------------------------------------
class Hcm:
    """A hierarchical communication matrix: `layers` is a list of
    (ranks, group_bw, p2p) outermost first, p2p a ranks x ranks nested list of
    GB/s or None (every pair at group_bw)."""

    def __init__(self, layers):
        self._keep = []
        arr = (atp_hcm_layer * len(layers))()
        for j, (ranks, group_bw, p2p) in enumerate(layers):
            arr[j].ranks = int(ranks)
            arr[j].group_bw = float(group_bw)
            if p2p is None:
                arr[j].p2p = None
            else:
                flat = (ctypes.c_double * (int(ranks) * int(ranks)))(
                    *[float(x) for row in p2p for x in row])
                self._keep.append(flat)
                arr[j].p2p = ctypes.cast(flat, ctypes.POINTER(ctypes.c_double))
        self.layers = arr
        self.n = len(layers)


def hcm_mi355x_xgmi(gpus: int = 8, link_gbs: float = 153.0) -> Hcm:
    """One MI355X node: `gpus` GPUs, every pair joined by one xGMI link of
    `link_gbs` GB/s, so a GPU's group bandwidth is (gpus - 1) links."""
    p2p = [[0.0 if u == v else link_gbs for v in range(gpus)] for u in range(gpus)]
    return Hcm([(gpus, (gpus - 1) * link_gbs, p2p)])


def model_dims(layers: int, batch: int, seq: int, hidden: int, elem_bytes: int = 2):
    return atp_model_dims(int(layers), int(batch), int(seq), int(hidden), int(elem_bytes))


def atp_tcomm(dims: atp_model_dims, d1: int, d2: int, b1: float, b2: float) -> float:
    t = ctypes.c_double()
    _check(load_library().atp_tcomm(ctypes.byref(dims), int(d1), int(d2), float(b1), float(b2),
                                    ctypes.byref(t)))
    return t.value


def atp_hcm_mesh_cost(hcm: Hcm, dims: atp_model_dims, d1: int, d2: int) -> dict:
    c = atp_mesh_cost()
    _check(load_library().atp_hcm_mesh_cost(hcm.layers, hcm.n, ctypes.byref(dims), int(d1),
                                            int(d2), ctypes.byref(c)))
    return c.as_dict()


def atp_plan_mesh(hcm: Hcm, dims: atp_model_dims, max_costs: int = 256):
    """(best mesh cost, costs of every candidate mesh, largest d1 first)."""
    best = atp_mesh_cost()
    arr = (atp_mesh_cost * max_costs)()
    n = ctypes.c_int32()
    _check(load_library().atp_plan_mesh(hcm.layers, hcm.n, ctypes.byref(dims), ctypes.byref(best),
                                        arr, int(max_costs), ctypes.byref(n)))
    return best.as_dict(), [arr[i].as_dict() for i in range(n.value)]
