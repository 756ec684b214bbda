"""ctypes binding of libtsfm_spec.so: argument marshalling only.

Every function mirrors the C entry point of the same name in include/tsfm.h.  torch is used
for device memory and streams; no step of the decoding path runs in Python.  There is no
fallback: if the shared library is missing or cannot be loaded, importing this module fails.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, Optional

import numpy as np

from . import build as _build

TSFM_OK = 0
TSFM_ERR_ARG, TSFM_ERR_SHAPE, TSFM_ERR_ARCH, TSFM_ERR_CUDA, TSFM_ERR_TIMEOUT, TSFM_ERR_INTERNAL = -1, -2, -3, -4, -5, -6
TSFM_F32, TSFM_BF16 = 0, 1
TSFM_DRAFT_SEPARATE, TSFM_DRAFT_LAYER_SKIP = 0, 1
TSFM_GEMM_AUTO, TSFM_GEMM_SIMT, TSFM_GEMM_WS = 0, 1, 2
TSFM_EXEC_GRAPH, TSFM_EXEC_STREAM, TSFM_EXEC_NO_PDL, TSFM_EXEC_NO_COMPACT, TSFM_EXEC_CHECK_BOUNDS = 0, 1, 2, 4, 8
TSFM_MAX_K = 32
TSFM_MAX_TREE, TSFM_MAX_TOP = 256, 32
TSFM_PAGES_BAD_ID, TSFM_PAGES_BAD_LEN, TSFM_PAGES_TIMEOUT = 1, 2, 4
TSFM_ROPE_HALF, TSFM_ROPE_INTERLEAVED = 0, 1
TSFM_ROPE_PLAIN, TSFM_ROPE_LINEAR, TSFM_ROPE_BASE, TSFM_ROPE_PARTS = 0, 1, 2, 3

EXPORTS = [
    "tsfm_weights_bytes", "tsfm_weights_offset", "tsfm_weights_bytes_io", "tsfm_weights_offset_io", "tsfm_spec_create", "tsfm_spec_forecast", "tsfm_spec_forecast_variant",
    "tsfm_target_only_forecast", "tsfm_draft_only_forecast", "tsfm_spec_forecast_host", "tsfm_target_only_forecast_host",
    "tsfm_spec_last_trace", "tsfm_accept_round", "tsfm_model_forward", "tsfm_gemm_bf16", "tsfm_gemm_bf16_static",
    "tsfm_rope_init", "tsfm_rope_append", "tsfm_paged_attention", "tsfm_paged_attention_workspace", "tsfm_debug_tile_wait", "tsfm_cache_evict", "tsfm_verify_tokens",
    "tsfm_tree_init", "tsfm_rope_append_tree", "tsfm_tree_attention", "tsfm_tree_attention_workspace", "tsfm_window_attention", "tsfm_token_logprobs",
    "tsfm_verify_tree", "tsfm_cache_commit",
    "tsfm_spec_debug_guard", "tsfm_spec_set_profiling", "tsfm_spec_kernel_profile", "tsfm_advise_block_size", "tsfm_spec_destroy", "tsfm_launch_count", "tsfm_strerror", "tsfm_last_cuda_error",
]


class tsfm_arch(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_heads", C.c_int32), ("d_ff", C.c_int32)]


class tsfm_cfg(C.Structure):
    _fields_ = [("target", tsfm_arch), ("draft", tsfm_arch),
                ("patch_len", C.c_int32), ("dtype", C.c_int32), ("draft_mode", C.c_int32),
                ("max_batch", C.c_int32), ("max_ctx_tokens", C.c_int32),
                ("max_horizon_patches", C.c_int32), ("max_K", C.c_int32), ("gemm_backend", C.c_int32),
                ("rms_eps", C.c_float), ("norm_eps", C.c_float), ("rope_base", C.c_float),
                ("exec_mode", C.c_int32), ("patch_in", C.c_int32), ("stream", C.c_void_p)]


class tsfm_weights(C.Structure):
    _fields_ = [("blob", C.c_void_p), ("bytes", C.c_size_t)]


class tsfm_stats(C.Structure):
    _fields_ = [("rounds", C.c_int64), ("proposals_drafted", C.c_int64), ("proposals_tested", C.c_int64),
                ("proposals_accepted", C.c_int64), ("patches_committed", C.c_int64),
                ("near_margin_decisions", C.c_int64),
                ("tested_by_pos", C.c_int64 * TSFM_MAX_K), ("accepted_by_pos", C.c_int64 * TSFM_MAX_K),
                ("L_hist", C.c_int64 * (TSFM_MAX_K + 2)),
                ("ms_total", C.c_float), ("ms_prefill", C.c_float), ("ms_draft", C.c_float),
                ("ms_verify", C.c_float), ("ms_accept", C.c_float),
                ("device_status", C.c_int32), ("reserved0", C.c_int32)]

    def as_dict(self):
        d = {k: getattr(self, k) for k, _ in self._fields_ if k not in ("tested_by_pos", "accepted_by_pos", "L_hist", "reserved0")}
        d["tested_by_pos"] = list(self.tested_by_pos)
        d["accepted_by_pos"] = list(self.accepted_by_pos)
        d["L_hist"] = list(self.L_hist)
        return d


class tsfm_variant(C.Structure):
    _fields_ = [("sigma_q", C.c_float), ("fallback_noise", C.c_float), ("sample_proposals", C.c_int32),
                ("no_tempering", C.c_int32)]


class tsfm_kernel_stat(C.Structure):
    _fields_ = [("name", C.c_char * 24), ("launches", C.c_int64), ("ms_total", C.c_double),
                ("bytes", C.c_double), ("flops", C.c_double)]


class tsfm_kv_pages(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p),
                ("page_stride", C.c_int64), ("head_stride", C.c_int64), ("slot_stride", C.c_int64),
                ("table", C.c_void_p), ("table_stride", C.c_int32), ("max_pages", C.c_int32), ("n_pages", C.c_int32),
                ("page_size", C.c_int32), ("n_kv_heads", C.c_int32), ("d_head", C.c_int32), ("dtype", C.c_int32),
                ("status", C.c_void_p)]
    device = rows = None                       # of the tensors, where kv_pages has made the description


class tsfm_rope(C.Structure):
    _fields_ = [("layout", C.c_int32), ("rot_dim", C.c_int32), ("mscale", C.c_float), ("reserved0", C.c_int32),
                ("turn", C.c_uint64 * 64)]


def _load() -> C.CDLL:
    path = _build.LIB
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with `python paper_2511_18191_b200/build.py` "
                          "(nvcc, sm_100a); there is no fallback implementation")
    lib = C.CDLL(path)
    i32, f32, u64, vp, sz = C.c_int32, C.c_float, C.c_uint64, C.c_void_p, C.c_size_t
    lib.tsfm_weights_bytes.restype = sz
    lib.tsfm_weights_bytes.argtypes = [C.POINTER(tsfm_arch), i32, i32]
    lib.tsfm_weights_offset.restype = sz
    lib.tsfm_weights_offset.argtypes = [C.POINTER(tsfm_arch), i32, i32, i32, C.c_char_p]
    lib.tsfm_weights_bytes_io.restype = sz
    lib.tsfm_weights_bytes_io.argtypes = [C.POINTER(tsfm_arch), i32, i32, i32]
    lib.tsfm_weights_offset_io.restype = sz
    lib.tsfm_weights_offset_io.argtypes = [C.POINTER(tsfm_arch), i32, i32, i32, i32, C.c_char_p]
    lib.tsfm_spec_create.restype = C.c_int
    lib.tsfm_spec_create.argtypes = [C.POINTER(tsfm_weights), C.POINTER(tsfm_weights), C.POINTER(tsfm_cfg), C.POINTER(vp)]
    for name in ("tsfm_spec_forecast", "tsfm_spec_forecast_host"):
        fn = getattr(lib, name)
        fn.restype = C.c_int
        fn.argtypes = [vp, vp, i32, i32, i32, i32, f32, u64, vp, C.POINTER(tsfm_stats)]
    lib.tsfm_spec_forecast_variant.restype = C.c_int
    lib.tsfm_spec_forecast_variant.argtypes = [vp, vp, i32, i32, i32, i32, f32, u64, C.POINTER(tsfm_variant), vp,
                                               C.POINTER(tsfm_stats)]
    for name in ("tsfm_target_only_forecast", "tsfm_draft_only_forecast", "tsfm_target_only_forecast_host"):
        fn = getattr(lib, name)
        fn.restype = C.c_int
        fn.argtypes = [vp, vp, i32, i32, i32, vp, C.POINTER(tsfm_stats)]
    lib.tsfm_spec_last_trace.restype = C.c_int
    lib.tsfm_spec_last_trace.argtypes = [vp, i32, C.POINTER(i32), vp, vp, vp]
    lib.tsfm_accept_round.restype = C.c_int
    lib.tsfm_accept_round.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, f32, f32, u64, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.tsfm_model_forward.restype = C.c_int
    lib.tsfm_model_forward.argtypes = [vp, i32, vp, i32, i32, vp]
    lib.tsfm_gemm_bf16.restype = C.c_int
    lib.tsfm_gemm_bf16.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32]
    lib.tsfm_gemm_bf16_static.restype = C.c_int
    lib.tsfm_gemm_bf16_static.argtypes = [vp, vp, vp, vp, i32, i32, i32]
    i64, f64, pages = C.c_int64, C.c_double, C.POINTER(tsfm_kv_pages)
    lib.tsfm_rope_init.restype = C.c_int
    lib.tsfm_rope_init.argtypes = [C.POINTER(tsfm_rope), i32, i32, i32, f64, f64, f64, f64, f64, f32]
    lib.tsfm_rope_append.restype = C.c_int
    lib.tsfm_rope_append.argtypes = [vp, C.POINTER(tsfm_rope), pages, vp, i64, vp, i64, vp, vp, vp, i32, i32, i32]
    lib.tsfm_paged_attention.restype = C.c_int
    lib.tsfm_paged_attention.argtypes = [vp, pages, vp, i64, vp, i64, vp, vp, i32, i32, i32, f32, i32, i32, i32, vp, vp, vp, i64, vp, sz]
    lib.tsfm_paged_attention_workspace.restype = sz
    lib.tsfm_paged_attention_workspace.argtypes = [pages, i32, i32, i32, i32, i32]
    lib.tsfm_debug_tile_wait.restype = None
    lib.tsfm_debug_tile_wait.argtypes = [i64, i32]
    lib.tsfm_cache_evict.restype = C.c_int
    lib.tsfm_cache_evict.argtypes = [vp, pages, vp, i32, vp, vp, i64, i32, i32, i32, i32, i32, vp, vp, i64, vp]
    lib.tsfm_verify_tokens.restype = C.c_int
    lib.tsfm_verify_tokens.argtypes = [vp, vp, vp, i64, vp, i64, i32, i32, i32, vp, u64, i32, i32, vp, vp, vp, vp, vp]
    for name, types in (
            ("tsfm_tree_init", [vp, vp, vp, i32, i32, i32, vp, vp]),
            ("tsfm_rope_append_tree", [vp, C.POINTER(tsfm_rope), pages, vp, i64, vp, i64, vp, vp, vp, vp, i32, i32, i32, i32]),
            ("tsfm_tree_attention", [vp, pages, vp, i64, vp, i64, vp, vp, vp, vp, i32, i32, i32, i32, f32, i32, i32, i32, vp, vp, sz]),
            ("tsfm_window_attention", [vp, pages, vp, i64, vp, i64, vp, vp, i32, i32, i32, f32, i32, i32, i32, vp, vp, sz]),
            ("tsfm_token_logprobs", [vp, vp, i64, i32, i32, i32, f32, vp, i32, vp, vp, vp, i32, vp, vp]),
            ("tsfm_verify_tree", [vp, vp, vp, i32, vp, i64, vp, i64, i32, i32, i32, vp, u64, i32, i32, vp, vp, vp, vp, vp, vp]),
            ("tsfm_cache_commit", [vp, pages, vp, vp, i32, i32, i32, i64])):
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = C.c_int, types
    lib.tsfm_tree_attention_workspace.restype = sz
    lib.tsfm_tree_attention_workspace.argtypes = [pages, i32, i32, i32, i32]
    lib.tsfm_spec_debug_guard.restype = C.c_int
    lib.tsfm_spec_debug_guard.argtypes = [vp, i32, i32, C.POINTER(i32)]
    lib.tsfm_spec_set_profiling.restype = C.c_int
    lib.tsfm_spec_set_profiling.argtypes = [vp, i32]
    lib.tsfm_spec_kernel_profile.restype = C.c_int
    lib.tsfm_spec_kernel_profile.argtypes = [vp, i32, C.POINTER(i32), C.POINTER(tsfm_kernel_stat)]
    lib.tsfm_advise_block_size.restype = C.c_int32
    lib.tsfm_advise_block_size.argtypes = [C.c_double, C.c_double, C.c_double, i32, C.POINTER(C.c_double)]
    lib.tsfm_spec_destroy.restype = C.c_int
    lib.tsfm_spec_destroy.argtypes = [vp]
    lib.tsfm_launch_count.restype = C.c_int64
    lib.tsfm_launch_count.argtypes = []
    lib.tsfm_strerror.restype = C.c_char_p
    lib.tsfm_strerror.argtypes = [C.c_int]
    lib.tsfm_last_cuda_error.restype = C.c_char_p
    lib.tsfm_last_cuda_error.argtypes = []
    return lib


lib = _load()


class TsfmError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = lib.tsfm_strerror(code).decode()
        if code in (TSFM_ERR_CUDA, TSFM_ERR_INTERNAL):
            msg += " (" + lib.tsfm_last_cuda_error().decode() + ")"
        super().__init__(f"{where}: {msg} [{code}]")


def _check(code: int, where: str) -> None:
    if code != TSFM_OK:
        raise TsfmError(code, where)


def _ptr(t) -> Optional[int]:
    """Address of a torch tensor / numpy array (None -> NULL)."""
    if t is None:
        return None
    try:
        return t.data_ptr()
    except AttributeError:
        return t.ctypes.data


def _arch(a) -> tsfm_arch:
    return tsfm_arch(a.n_layers, a.d_model, a.n_heads, a.d_ff)


def _dtype_code(dtype: str) -> int:
    return {"f32": TSFM_F32, "bf16": TSFM_BF16}[dtype]


# ---------------------------------------------------------------- weight blobs
def tsfm_weights_bytes(arch, patch_len: int, dtype: str) -> int:
    a = _arch(arch)
    return int(lib.tsfm_weights_bytes(C.byref(a), patch_len, _dtype_code(dtype)))


def tsfm_weights_offset(arch, patch_len: int, dtype: str, layer: int, name: str) -> int:
    a = _arch(arch)
    return int(lib.tsfm_weights_offset(C.byref(a), patch_len, _dtype_code(dtype), layer, name.encode()))


def tsfm_weights_bytes_io(arch, patch_in: int, patch_len: int, dtype: str) -> int:
    a = _arch(arch)
    return int(lib.tsfm_weights_bytes_io(C.byref(a), patch_in, patch_len, _dtype_code(dtype)))


def tsfm_weights_offset_io(arch, patch_in: int, patch_len: int, dtype: str, layer: int, name: str) -> int:
    a = _arch(arch)
    return int(lib.tsfm_weights_offset_io(C.byref(a), patch_in, patch_len, _dtype_code(dtype), layer, name.encode()))


def pack_weights(weights: Dict[str, np.ndarray], arch, patch_len: int, dtype: str, patch_in: int = 0) -> np.ndarray:
    """Serialise a name -> float32 array dict into the blob layout of include/tsfm.h (host bytes)."""
    total = tsfm_weights_bytes_io(arch, patch_in, patch_len, dtype)
    if total == 0:
        raise ValueError("unsupported model shape")
    blob = np.zeros(total, dtype=np.uint8)
    hdr = blob[:36].view(np.int32)
    hdr[:] = [0x4D465354, 1, _dtype_code(dtype), arch.n_layers, arch.d_model, arch.n_heads, arch.d_ff, patch_len,
              patch_in]
    for name, w in weights.items():
        parts = name.split(".")
        layer, short = (int(parts[1]), parts[2]) if parts[0] == "layers" else (-1, name)
        off = tsfm_weights_offset_io(arch, patch_in, patch_len, dtype, layer, short)
        if off == 0:
            raise ValueError(f"no slot for tensor {name}")
        w32 = np.ascontiguousarray(w, dtype=np.float32)
        if w32.ndim == 1 or dtype == "f32":
            raw = w32.view(np.uint8).reshape(-1)
        else:                                   # values are already bf16-representable: keep the top half
            u = w32.view(np.uint32)
            if np.any(u & 0xFFFF):
                raise ValueError(f"tensor {name} is not bf16-representable")
            raw = (u >> 16).astype(np.uint16).view(np.uint8).reshape(-1)
        blob[off:off + raw.size] = raw
    return blob


# ---------------------------------------------------------------- decoder handle
def tsfm_spec_create(target_blob, draft_blob, cfg: tsfm_cfg) -> int:
    """target_blob / draft_blob: torch.uint8 CUDA tensors (kept alive by the caller). Returns the handle."""
    tw = tsfm_weights(_ptr(target_blob), target_blob.numel())
    dw = tsfm_weights(_ptr(draft_blob), draft_blob.numel()) if draft_blob is not None else None
    h = C.c_void_p()
    _check(lib.tsfm_spec_create(C.byref(tw), C.byref(dw) if dw is not None else None, C.byref(cfg), C.byref(h)),
           "tsfm_spec_create")
    return h.value


def tsfm_spec_destroy(h: int) -> None:
    _check(lib.tsfm_spec_destroy(h), "tsfm_spec_destroy")


def tsfm_spec_forecast(h, series, B, ctx_len, H, K, tau, seed, out, stats: Optional[tsfm_stats] = None) -> None:
    _check(lib.tsfm_spec_forecast(h, _ptr(series), B, ctx_len, H, K, tau, seed, _ptr(out),
                                  C.byref(stats) if stats is not None else None), "tsfm_spec_forecast")


def tsfm_spec_forecast_variant(h, series, B, ctx_len, H, K, tau, seed, variant: Optional[tsfm_variant], out,
                               stats: Optional[tsfm_stats] = None) -> None:
    _check(lib.tsfm_spec_forecast_variant(h, _ptr(series), B, ctx_len, H, K, tau, seed,
                                          C.byref(variant) if variant is not None else None, _ptr(out),
                                          C.byref(stats) if stats is not None else None), "tsfm_spec_forecast_variant")


def tsfm_target_only_forecast(h, series, B, ctx_len, H, out, stats: Optional[tsfm_stats] = None) -> None:
    _check(lib.tsfm_target_only_forecast(h, _ptr(series), B, ctx_len, H, _ptr(out),
                                         C.byref(stats) if stats is not None else None), "tsfm_target_only_forecast")


def tsfm_draft_only_forecast(h, series, B, ctx_len, H, out, stats: Optional[tsfm_stats] = None) -> None:
    _check(lib.tsfm_draft_only_forecast(h, _ptr(series), B, ctx_len, H, _ptr(out),
                                        C.byref(stats) if stats is not None else None), "tsfm_draft_only_forecast")


def tsfm_spec_forecast_host(h, series, B, ctx_len, H, K, tau, seed, out, stats: Optional[tsfm_stats] = None) -> None:
    _check(lib.tsfm_spec_forecast_host(h, _ptr(series), B, ctx_len, H, K, tau, seed, _ptr(out),
                                       C.byref(stats) if stats is not None else None), "tsfm_spec_forecast_host")


def tsfm_target_only_forecast_host(h, series, B, ctx_len, H, out, stats: Optional[tsfm_stats] = None) -> None:
    _check(lib.tsfm_target_only_forecast_host(h, _ptr(series), B, ctx_len, H, _ptr(out),
                                              C.byref(stats) if stats is not None else None),
           "tsfm_target_only_forecast_host")


def tsfm_spec_last_trace(h, B: int, K: int, cap_rounds: int):
    """Returns (n_accept [R, B] int32, ell [R, B, K] f32, log_u [R, B, K] f32) as numpy arrays."""
    n_acc = np.empty((cap_rounds, B), dtype=np.int32)
    ell = np.empty((cap_rounds, B, K), dtype=np.float32)
    log_u = np.empty((cap_rounds, B, K), dtype=np.float32)
    r = C.c_int32(0)
    _check(lib.tsfm_spec_last_trace(h, cap_rounds, C.byref(r), _ptr(n_acc), _ptr(ell), _ptr(log_u)),
           "tsfm_spec_last_trace")
    R = r.value
    return n_acc[:R], ell[:R], log_u[:R]


def tsfm_accept_round(stream, x, mu_q, mu_p, B, K, P, T, sigma_p, sigma_q, seed, round_idx, series0,
                      forced_u, done, commit, n_accept, ell, log_u) -> None:
    _check(lib.tsfm_accept_round(stream, _ptr(x), _ptr(mu_q), _ptr(mu_p), B, K, P, T, sigma_p, sigma_q, seed,
                                 round_idx, series0, _ptr(forced_u), _ptr(done), _ptr(commit), _ptr(n_accept),
                                 _ptr(ell), _ptr(log_u)), "tsfm_accept_round")


def tsfm_model_forward(h, which: int, tokens, B: int, n: int, out) -> None:
    _check(lib.tsfm_model_forward(h, which, _ptr(tokens), B, n, _ptr(out)), "tsfm_model_forward")


def tsfm_gemm_bf16(stream, A, W, Cout, M: int, N: int, Kd: int, backend: int) -> None:
    _check(lib.tsfm_gemm_bf16(stream, _ptr(A), _ptr(W), _ptr(Cout), M, N, Kd, backend), "tsfm_gemm_bf16")


TSFM_STATIC_GEMM_MAX_ELEMS = 1 << 20


def tsfm_gemm_bf16_static(stream, A, W, Cout, M: int, N: int, Kd: int) -> None:
    """The contraction of tsfm_gemm_bf16 without any device allocation (scratch is a fixed array inside
    the library; M * N <= TSFM_STATIC_GEMM_MAX_ELEMS; calls on one device must not overlap)."""
    code = lib.tsfm_gemm_bf16_static(stream, _ptr(A), _ptr(W), _ptr(Cout), M, N, Kd)
    if code == TSFM_ERR_SHAPE:
        raise TsfmError(code, "tsfm_gemm_bf16_static: " + lib.tsfm_last_cuda_error().decode())
    _check(code, "tsfm_gemm_bf16_static")


# ---------------------------------------------------------------- serving over a cache of pages
_I32 = _I64 = _F32 = _current_device = None            # torch's, once a tensor has come in
_ELEMENT: Dict[int, object] = {}


def _torch_names() -> None:
    global _I32, _I64, _F32, _current_device
    import torch
    _ELEMENT.update({TSFM_F32: torch.float32, TSFM_BF16: torch.bfloat16})
    _I64, _F32, _current_device = torch.int64, torch.float32, torch._C._cuda_getDevice        # (asked only with a tensor of a GPU at hand)
    _I32 = torch.int32                         # (last: it says that the others are there)


def kv_pages(k, v, table, status=None) -> tsfm_kv_pages:
    """Describe a pool: k, v [n_pages, n_kv_heads, page_size, d_head] tensors of one dtype and the same strides (a pool laid out
    [n_pages, page_size, n_kv_heads, d_head] goes in as k.transpose(1, 2)), table [B, max_pages] int32.  The tensors stay the
    caller's; the description holds their addresses."""
    import torch
    code = {torch.float32: TSFM_F32, torch.bfloat16: TSFM_BF16}.get(k.dtype)
    if (code is None or v.dtype != k.dtype or k.dim() != 4 or v.shape != k.shape or v.stride() != k.stride() or k.stride(3) != 1
            or table.dim() != 2 or table.dtype != torch.int32 or table.stride(1) != 1 or len({k.device, v.device, table.device}) != 1
            or (status is not None and (status.dtype != torch.int32 or status.device != k.device))):
        raise TsfmError(TSFM_ERR_ARG, "kv_pages")
    pages = tsfm_kv_pages(k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(1), k.stride(2), table.data_ptr(), table.stride(0),
                          table.shape[1], k.shape[0], k.shape[2], k.shape[1], k.shape[3], code, _ptr(status))
    pages.device, pages.rows = k.get_device(), table.shape[0]
    return pages


# The calls below take tensors on the current device, of the types that include/tsfm.h names; what would be read as something else is
# TSFM_ERR_ARG: another type, a host tensor or array, another device, a vector that is not contiguous, a table of fewer rows than series.
# (0.2 us a tensor: 0.8 to 1.5 us a call; the library itself takes addresses.)
def _device_of(t, where: str, pages=None, B: int = 0) -> int:
    """The device of the tensor that a call cannot do without."""
    if _I32 is None:
        _torch_names()
    device = -1 if t is None or isinstance(t, np.ndarray) else t.get_device()
    if device < 0 or device != _current_device():
        raise TsfmError(TSFM_ERR_ARG, where)
    if pages is not None and pages.device is not None and (pages.device != device or pages.rows < B):
        raise TsfmError(TSFM_ERR_ARG, where)
    return device


def _rows(t, dtype, device: int, where: str) -> Optional[int]:
    """Address of a tensor whose row stride the caller gives (None -> NULL)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != device:
        raise TsfmError(TSFM_ERR_ARG, where)
    return t.data_ptr()


def _dense(t, dtype, device: int, where: str) -> Optional[int]:
    """Address of a contiguous tensor (None -> NULL)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != device or not t.is_contiguous():
        raise TsfmError(TSFM_ERR_ARG, where)
    return t.data_ptr()


def _bytes(t, device: int, where: str) -> Optional[int]:
    """Address of a contiguous tensor of any type (None -> NULL)."""
    if t is None:
        return None
    if isinstance(t, np.ndarray) or t.get_device() != device or not t.is_contiguous():
        raise TsfmError(TSFM_ERR_ARG, where)
    return t.data_ptr()


def tsfm_rope_init(layout: int, rot_dim: int, scaling: int, base: float, factor: float = 1.0, original_len: float = 0.0,
                   turns_lo: float = 0.0, turns_hi: float = 0.0, mscale: float = 1.0) -> tsfm_rope:
    r = tsfm_rope()
    _check(lib.tsfm_rope_init(C.byref(r), layout, rot_dim, scaling, base, factor, original_len, turns_lo, turns_hi, mscale),
           "tsfm_rope_init")
    return r


def tsfm_rope_append(stream, rope: tsfm_rope, pages: tsfm_kv_pages, qkv, qkv_stride: int, q_out, q_out_stride: int, pos, len, n_new,
                     B: int, M: int, n_heads: int) -> None:
    me = "tsfm_rope_append"
    d = _device_of(len, me, pages, B)
    e = _ELEMENT.get(pages.dtype)
    _check(lib.tsfm_rope_append(stream, rope, pages, _rows(qkv, e, d, me), qkv_stride, _rows(q_out, e, d, me), q_out_stride,
                                _dense(pos, _I32, d, me), _dense(len, _I32, d, me), _dense(n_new, _I32, d, me), B, M, n_heads), me)


def tsfm_paged_attention_workspace(pages: tsfm_kv_pages, B: int, M: int, n_heads: int, max_len: int, with_weights: bool = False) -> int:
    return int(lib.tsfm_paged_attention_workspace(pages, B, M, n_heads, max_len, int(bool(with_weights))))


def tsfm_paged_attention(stream, pages: tsfm_kv_pages, q, q_stride: int, out, out_stride: int, len, n_new, B: int, M: int, n_heads: int,
                         scale: float, causal: bool, window: int, max_len: int, lse, w_in, w_out, w_stride: int, workspace,
                         workspace_bytes: int) -> None:
    me = "tsfm_paged_attention"
    d = _device_of(len, me, pages, B)
    e = _ELEMENT.get(pages.dtype)
    _check(lib.tsfm_paged_attention(stream, pages, _rows(q, e, d, me), q_stride, _rows(out, e, d, me), out_stride, _dense(len, _I32, d, me),
                                    _dense(n_new, _I32, d, me), B, M, n_heads, scale, causal, window, max_len, _dense(lse, _F32, d, me),
                                    _rows(w_in, _F32, d, me), _rows(w_out, _F32, d, me), w_stride,
                                    _bytes(workspace, d, me), workspace_bytes), me)


def tsfm_debug_tile_wait(wait_us: int = 0, miss_from: int = -1) -> None:
    """Tests only: let the attention's wait for a tile run out (no arguments: as it was)."""
    lib.tsfm_debug_tile_wait(wait_us, miss_from)


def tsfm_cache_evict(stream, pages: tsfm_kv_pages, dst_table, dst_stride: int, len, w, w_stride: int, B: int, budget: int, sinks: int,
                     recent: int, max_len: int, kept, w_out, w_out_stride: int, len_out) -> None:
    me = "tsfm_cache_evict"
    d = _device_of(len, me, pages, B)
    _check(lib.tsfm_cache_evict(stream, pages, _rows(dst_table, _I32, d, me), dst_stride, _dense(len, _I32, d, me), _rows(w, _F32, d, me), w_stride,
                                B, budget, sinks, recent, max_len, _dense(kept, _I32, d, me), _rows(w_out, _F32, d, me), w_out_stride,
                                _dense(len_out, _I32, d, me)), me)


def tsfm_verify_tokens(stream, tokens, p, p_stride: int, q, q_stride: int, B: int, K: int, V: int, u, seed: int, round_idx: int,
                       series0: int, n_draft, len, out, n_accept, len_out) -> None:
    me = "tsfm_verify_tokens"
    d = _device_of(p, me)
    _check(lib.tsfm_verify_tokens(stream, _dense(tokens, _I32, d, me), _rows(p, _F32, d, me), p_stride, _rows(q, _F32, d, me), q_stride, B, K, V,
                                  _dense(u, _F32, d, me), seed, round_idx, series0, _dense(n_draft, _I32, d, me), _dense(len, _I32, d, me),
                                  _dense(out, _I32, d, me), _dense(n_accept, _I32, d, me), _dense(len_out, _I32, d, me)), me)


# ---------------------------------------------------------------- trees of drafted tokens, windows with sinks, log probabilities
def _tree(t, dtype, device: int, where: str, shape) -> Optional[int]:
    """Address of a contiguous tensor that describes a tree, of at least as many entries as `shape` has (None -> NULL)."""
    if t is not None and t.numel() < shape:
        raise TsfmError(TSFM_ERR_ARG, where)
    return _dense(t, dtype, device, where)


def tsfm_tree_init(stream, parent, n_new, B: int, M: int, window: int, mask, depth) -> None:
    """mask: int64 (its bits are the library's uint64)."""
    me = "tsfm_tree_init"
    d = _device_of(parent, me)
    _check(lib.tsfm_tree_init(stream, _tree(parent, _I32, d, me, B * M), _dense(n_new, _I32, d, me), B, M, window,
                              _tree(mask, _I64, d, me, B * M * ((M + 63) // 64)), _tree(depth, _I32, d, me, B * M)), me)


def tsfm_rope_append_tree(stream, rope: tsfm_rope, pages: tsfm_kv_pages, qkv, qkv_stride: int, q_out, q_out_stride: int, pos, len, n_new,
                          depth, shared_tree: bool, B: int, M: int, n_heads: int) -> None:
    me = "tsfm_rope_append_tree"
    d = _device_of(len, me, pages, B)
    e = _ELEMENT.get(pages.dtype)
    _check(lib.tsfm_rope_append_tree(stream, rope, pages, _rows(qkv, e, d, me), qkv_stride, _rows(q_out, e, d, me), q_out_stride,
                                     _dense(pos, _I32, d, me), _dense(len, _I32, d, me), _dense(n_new, _I32, d, me),
                                     _tree(depth, _I32, d, me, M if shared_tree else B * M), int(bool(shared_tree)), B, M, n_heads), me)


def tsfm_tree_attention_workspace(pages: tsfm_kv_pages, B: int, M: int, n_heads: int, max_len: int) -> int:
    return int(lib.tsfm_tree_attention_workspace(pages, B, M, n_heads, max_len))


def tsfm_tree_attention(stream, pages: tsfm_kv_pages, q, q_stride: int, out, out_stride: int, len, n_new, mask, depth, shared_tree: bool, B: int,
                        M: int, n_heads: int, scale: float, window: int, sinks: int, max_len: int, lse, workspace, workspace_bytes: int) -> None:
    me = "tsfm_tree_attention"
    d = _device_of(len, me, pages, B)
    e = _ELEMENT.get(pages.dtype)
    nodes = M if shared_tree else B * M
    _check(lib.tsfm_tree_attention(stream, pages, _rows(q, e, d, me), q_stride, _rows(out, e, d, me), out_stride, _dense(len, _I32, d, me),
                                   _dense(n_new, _I32, d, me), _tree(mask, _I64, d, me, nodes * ((M + 63) // 64)), _tree(depth, _I32, d, me, nodes),
                                   int(bool(shared_tree)), B, M, n_heads, scale, window, sinks, max_len, _dense(lse, _F32, d, me),
                                   _bytes(workspace, d, me), workspace_bytes), me)


def tsfm_window_attention(stream, pages: tsfm_kv_pages, q, q_stride: int, out, out_stride: int, len, n_new, B: int, M: int, n_heads: int, scale: float,
                          window: int, sinks: int, max_len: int, lse, workspace, workspace_bytes: int) -> None:
    me = "tsfm_window_attention"
    d = _device_of(len, me, pages, B)
    e = _ELEMENT.get(pages.dtype)
    _check(lib.tsfm_window_attention(stream, pages, _rows(q, e, d, me), q_stride, _rows(out, e, d, me), out_stride, _dense(len, _I32, d, me),
                                     _dense(n_new, _I32, d, me), B, M, n_heads, scale, window, sinks, max_len, _dense(lse, _F32, d, me),
                                     _bytes(workspace, d, me), workspace_bytes), me)


def tsfm_token_logprobs(stream, logits, stride: int, rows: int, V: int, scale: float, tokens, n_tokens: int, logprob, lse, entropy, n_top: int,
                        top_ids, top_logprob) -> None:
    """The library's dtype argument is that of `logits`."""
    me = "tsfm_token_logprobs"
    d = _device_of(logits, me)
    code = next((c for c, e in _ELEMENT.items() if logits.dtype is e), -1) if logits.stride(-1) == 1 else -1
    _check(lib.tsfm_token_logprobs(stream, logits.data_ptr(), stride, code, rows, V, scale, _dense(tokens, _I32, d, me), n_tokens,
                                   _dense(logprob, _F32, d, me), _dense(lse, _F32, d, me), _dense(entropy, _F32, d, me), n_top,
                                   _dense(top_ids, _I32, d, me), _dense(top_logprob, _F32, d, me)), me)


def tsfm_verify_tree(stream, tokens, parent, shared_tree: bool, p, p_stride: int, q, q_stride: int, B: int, M: int, V: int, u, seed: int,
                     round_idx: int, series0: int, n_new, len, out, path, n_accept, len_out) -> None:
    me = "tsfm_verify_tree"
    d = _device_of(p, me)
    _check(lib.tsfm_verify_tree(stream, _dense(tokens, _I32, d, me), _tree(parent, _I32, d, me, M if shared_tree else B * M), int(bool(shared_tree)),
                                _rows(p, _F32, d, me), p_stride, _rows(q, _F32, d, me), q_stride, B, M, V, _dense(u, _F32, d, me), seed, round_idx,
                                series0, _dense(n_new, _I32, d, me), _dense(len, _I32, d, me), _dense(out, _I32, d, me), _dense(path, _I32, d, me),
                                _dense(n_accept, _I32, d, me), _dense(len_out, _I32, d, me)), me)


def tsfm_cache_commit(stream, pages: tsfm_kv_pages, path, len, B: int, M: int, n_layers: int = 1, layer_stride: int = 0) -> None:
    """pages: of the first layer's pool."""
    me = "tsfm_cache_commit"
    d = _device_of(len, me, pages, B)
    _check(lib.tsfm_cache_commit(stream, pages, _dense(path, _I32, d, me), _dense(len, _I32, d, me), B, M, n_layers, layer_stride), me)


def tsfm_spec_debug_guard(h, region: int = -1, damage: bool = False) -> int:
    """Bounds-checking mode: number of guard regions; region >= 0 damages / restores one byte of it."""
    n = C.c_int32(0)
    _check(lib.tsfm_spec_debug_guard(h, region, int(bool(damage)), C.byref(n)), "tsfm_spec_debug_guard")
    return n.value


def tsfm_spec_set_profiling(h, enable: bool) -> None:
    _check(lib.tsfm_spec_set_profiling(h, int(bool(enable))), "tsfm_spec_set_profiling")


def tsfm_spec_kernel_profile(h):
    """Per-kernel {name: dict(launches, ms_total, bytes, flops)} of the launches since profiling was enabled."""
    arr = (tsfm_kernel_stat * 32)()
    n = C.c_int32(0)
    _check(lib.tsfm_spec_kernel_profile(h, 32, C.byref(n), arr), "tsfm_spec_kernel_profile")
    return {arr[i].name.decode(): dict(launches=arr[i].launches, ms_total=arr[i].ms_total, bytes=arr[i].bytes,
                                       flops=arr[i].flops) for i in range(n.value)}


def tsfm_advise_block_size(alpha: float, c: float, v: float, max_K: int):
    """(K, predicted speedup) by the marginal-gain rule; K == 0 on invalid arguments."""
    s = C.c_double(0.0)
    k = int(lib.tsfm_advise_block_size(alpha, c, v, max_K, C.byref(s)))
    return k, s.value


def tsfm_launch_count() -> int:
    return int(lib.tsfm_launch_count())


# ---------------------------------------------------------------- convenience wrapper
class SpecDecoder:
    """Owns device copies of the weight blobs and a decoder handle for one workload shape."""

    def __init__(self, target_w, draft_w, target_arch, draft_arch, patch_len: int, dtype: str,
                 draft_mode: str, max_batch: int, max_ctx_tokens: int, max_horizon_patches: int, max_K: int,
                 gemm_backend: int = TSFM_GEMM_AUTO, exec_mode: int = TSFM_EXEC_GRAPH, device: str = "cuda:0",
                 patch_in: int = 0):
        import torch
        self.torch = torch
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        self.patch_len, self.dtype = patch_len, dtype
        self.target_blob = torch.from_numpy(pack_weights(target_w, target_arch, patch_len, dtype, patch_in)).to(self.device)
        self.draft_blob = None
        if draft_mode != "layer_skip":
            self.draft_blob = torch.from_numpy(pack_weights(draft_w, draft_arch, patch_len, dtype, patch_in)).to(self.device)
        cfg = tsfm_cfg()
        cfg.target, cfg.draft = _arch(target_arch), _arch(draft_arch)
        cfg.patch_len, cfg.dtype = patch_len, _dtype_code(dtype)
        cfg.patch_in = patch_in
        cfg.draft_mode = TSFM_DRAFT_LAYER_SKIP if draft_mode == "layer_skip" else TSFM_DRAFT_SEPARATE
        cfg.max_batch, cfg.max_ctx_tokens = max_batch, max_ctx_tokens
        cfg.max_horizon_patches, cfg.max_K = max_horizon_patches, max_K
        cfg.gemm_backend = gemm_backend
        cfg.exec_mode = exec_mode
        cfg.rms_eps, cfg.norm_eps, cfg.rope_base = 1e-6, 1e-5, 1e4
        cfg.stream = torch.cuda.current_stream(self.device).cuda_stream
        self.cfg = cfg
        self.max_T, self.max_K = max_horizon_patches, max_K
        self.h = tsfm_spec_create(self.target_blob, self.draft_blob, cfg)

    @classmethod
    def for_workload(cls, wl, target_w, draft_w, max_K: Optional[int] = None, batch: Optional[int] = None, **kw):
        ks = max(wl.K_sweep) if wl.K_sweep else wl.K
        return cls(target_w, draft_w, wl.target, wl.draft, wl.patch_len, wl.dtype,
                   "layer_skip" if wl.draft_mode == "layer_skip" else "separate",
                   batch or wl.batch, wl.n_ctx_tokens, wl.n_patches, max_K or ks, patch_in=wl.patch_in, **kw)

    def close(self):
        if getattr(self, "h", None):
            tsfm_spec_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def forecast(self, series, H: int, K: int, tau: float, seed: int, out=None, stats: bool = True,
                 variant: Optional[tsfm_variant] = None):
        """series: CUDA float32 [B, ctx_len]. Returns (out [B, H] CUDA, tsfm_stats | None)."""
        B, ctx_len = series.shape
        if out is None:
            out = self.torch.empty((B, H), dtype=self.torch.float32, device=series.device)
        st = tsfm_stats() if stats else None
        if variant is None:
            tsfm_spec_forecast(self.h, series, B, ctx_len, H, K, tau, seed, out, st)
        else:
            tsfm_spec_forecast_variant(self.h, series, B, ctx_len, H, K, tau, seed, variant, out, st)
        return out, st

    def target_only(self, series, H: int, out=None, stats: bool = True):
        B, ctx_len = series.shape
        if out is None:
            out = self.torch.empty((B, H), dtype=self.torch.float32, device=series.device)
        st = tsfm_stats() if stats else None
        tsfm_target_only_forecast(self.h, series, B, ctx_len, H, out, st)
        return out, st

    def draft_only(self, series, H: int, out=None, stats: bool = True):
        B, ctx_len = series.shape
        if out is None:
            out = self.torch.empty((B, H), dtype=self.torch.float32, device=series.device)
        st = tsfm_stats() if stats else None
        tsfm_draft_only_forecast(self.h, series, B, ctx_len, H, out, st)
        return out, st

    def last_trace(self, B: int, K: int):
        return tsfm_spec_last_trace(self.h, B, K, self.max_T)

    def model_forward(self, which: int, tokens):
        B, n, _ = tokens.shape                                # [B, n, P_in]
        out = self.torch.empty((B, n, self.patch_len), dtype=tokens.dtype, device=tokens.device)
        tsfm_model_forward(self.h, which, tokens, B, n, out)
        return out
