"""Python binding of the ResKV C ABI (include/reskv.h).

Argument marshalling only: every step of construction and decode runs in the
CUDA library ``libreskv.so``.  Tensors are passed by ``data_ptr()``; streams
default to torch's current stream.  Importing this module does not load the
library; the first call does, and fails loudly if it has not been built.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libreskv.so")

RESKV_OK = 0
(RESKV_ERR_INVALID_ARG, RESKV_ERR_UNSUPPORTED, RESKV_ERR_OOM, RESKV_ERR_CUDA,
 RESKV_ERR_DEVICE_STATUS) = 1, 2, 3, 4, 5
STATUS_NAMES = {0: "OK", 1: "INVALID_ARG", 2: "UNSUPPORTED", 3: "OOM", 4: "CUDA",
                5: "DEVICE_STATUS"}
RESKV_SCORE_OBS_POOL, RESKV_SCORE_KEYNORM = 0, 1
RESKV_GATE_DYNAMIC, RESKV_GATE_FIXED = 0, 1
RESKV_DECODE_AUTO, RESKV_DECODE_FMA, RESKV_DECODE_MMA, RESKV_DECODE_CLUSTER = 0, 1, 2, 3
RESKV_DECODE_LSE_MERGE = 4
RESKV_SOFTMAX_SHARED, RESKV_SOFTMAX_SEPARATE = 0, 1
RESKV_DEBUG_SCORES, RESKV_DEBUG_RANKED, RESKV_DEBUG_LOSSES, RESKV_DEBUG_CANDIDATES = 0, 1, 2, 3
RESKV_DEBUG_UNIT_CANDIDATES = 4
RESKV_BUDGET_UNIFORM, RESKV_BUDGET_ADAKV = 0, 1
RESKV_TEST_FAIL_FIRST_WAIT, RESKV_TEST_FAIL_ALLOC = 1, 2
RESKV_APPEND_FAIL, RESKV_APPEND_RING_DROP, RESKV_APPEND_RING_FOLD = 0, 1, 2
RESKV_BF16, RESKV_F16, RESKV_F32 = 0, 1, 2
(RESKV_ROPE_NONE, RESKV_ROPE_LINEAR, RESKV_ROPE_BASE, RESKV_ROPE_WAVELENGTH,
 RESKV_ROPE_YARN) = 0, 1, 2, 3, 4
MAX_GRID = 8


class ReskvError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"reskv status {STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


class reskv_config(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("n_layers", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
        ("group", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("seq_len", ctypes.c_int64),
        ("budget", ctypes.c_int32), ("recent_window", ctypes.c_int32), ("n_obs", ctypes.c_int32),
        ("n_fit", ctypes.c_int32), ("n_val", ctypes.c_int32), ("pool_kernel", ctypes.c_int32),
        ("score_mode", ctypes.c_int32), ("n_grid", ctypes.c_int32),
        ("grid_ratios", ctypes.c_float * MAX_GRID), ("lloyd_iters", ctypes.c_int32),
        ("delta", ctypes.c_float), ("beta", ctypes.c_float),
        ("residual_override", ctypes.POINTER(ctypes.c_int32)),
        ("gate_mode", ctypes.c_int32), ("tau", ctypes.c_float), ("alpha", ctypes.c_float),
        ("g_min", ctypes.c_float), ("g_fixed", ctypes.c_float), ("keep_debug", ctypes.c_int32),
        ("decode_warps", ctypes.c_int32), ("decode_kernel", ctypes.c_int32),
        ("softmax_mode", ctypes.c_int32), ("append_capacity", ctypes.c_int32),
        ("unit_budgets", ctypes.POINTER(ctypes.c_int32)),
        ("budget_mode", ctypes.c_int32), ("adakv_safeguard", ctypes.c_float),
        ("append_policy", ctypes.c_int32),
    ]


class reskv_host_cache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("n_main", "n_res", "kslots", "vslots", "logc", "slot_pos", "counts", "n_app")]


class reskv_cache_info(ctypes.Structure):
    _fields_ = [("n_units", ctypes.c_int64), ("budget", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("slot_bytes", ctypes.c_int64),
                ("cache_bytes", ctypes.c_int64), ("layer_cluster", ctypes.c_int32),
                ("layer_cluster_warps", ctypes.c_int32), ("all_cluster", ctypes.c_int32),
                ("all_cluster_warps", ctypes.c_int32), ("build_ms", ctypes.c_float * 6),
                ("append_capacity", ctypes.c_int32), ("stride", ctypes.c_int32),
                ("max_appended", ctypes.c_int32), ("ragged", ctypes.c_int32),
                ("total_slots", ctypes.c_int64), ("n_candidates", ctypes.c_int32),
                ("ranked_width", ctypes.c_int32), ("all_units_per_warp", ctypes.c_int32),
                ("layer_units_per_warp", ctypes.c_int32), ("kv_copy_rank", ctypes.c_int32),
                ("reserved0", ctypes.c_int32)]


class reskv_device_cache(ctypes.Structure):
    _fields_ = [("kslots", ctypes.c_void_p), ("vslots", ctypes.c_void_p),
                ("logc", ctypes.c_void_p), ("n_main", ctypes.c_void_p), ("n_res", ctypes.c_void_p),
                ("n_units", ctypes.c_int64), ("budget", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("group", ctypes.c_int32),
                ("gate_mode", ctypes.c_int32), ("tau", ctypes.c_float), ("alpha", ctypes.c_float),
                ("g_min", ctypes.c_float), ("g_fixed", ctypes.c_float)]


class reskv_heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64), ("n_heads", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


class reskv_rotation(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("n_positions", ctypes.c_int64),
                ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32)]


class reskv_rope_config(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int32), ("scaling", ctypes.c_int32), ("base", ctypes.c_double),
                ("factor", ctypes.c_double), ("original_positions", ctypes.c_double),
                ("low_freq", ctypes.c_double), ("high_freq", ctypes.c_double),
                ("beta_fast", ctypes.c_double), ("beta_slow", ctypes.c_double),
                ("magnitude", ctypes.c_double)]


class reskv_paged_kv(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_void_p), ("n_pages", ctypes.c_int64),
                ("page_table", ctypes.c_void_p), ("batch", ctypes.c_int32),
                ("table_pages", ctypes.c_int32), ("page_tokens", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("quant_group", ctypes.c_int32), ("status", ctypes.c_void_p)]


class reskv_rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
                ("dtype", ctypes.c_int32)]


class reskv_paged_attn_args(ctypes.Structure):
    _fields_ = [("q", reskv_heads), ("o", reskv_heads), ("lse", ctypes.c_void_p),
                ("q_begin", ctypes.c_void_p), ("lens", ctypes.c_void_p), ("n_tokens", ctypes.c_int64),
                ("scale", ctypes.c_float), ("window", ctypes.c_int32), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t)]


_lib = None


def load_library():
    """Load libreskv.so (built in-tree by ``paper_2607_29591_gb300.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                           "`python -m paper_2607_29591_gb300.build` (there is no fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    cfgp = ctypes.POINTER(reskv_config)
    lib.reskv_config_default.argtypes = [cfgp]
    lib.reskv_config_default.restype = None
    lib.reskv_build_cache.argtypes = [cfgp, ctypes.POINTER(vp), ctypes.POINTER(vp),
                                      ctypes.POINTER(vp), vp, ctypes.POINTER(vp)]
    lib.reskv_build_cache.restype = i32
    lib.reskv_decode_attn.argtypes = [vp, i32, vp, vp, vp]
    lib.reskv_decode_attn.restype = i32
    lib.reskv_decode_attn_layers.argtypes = [vp, i32, i32, vp, vp, vp]
    lib.reskv_decode_attn_layers.restype = i32
    lib.reskv_decode_attn_host.argtypes = [vp, vp, vp, vp]
    lib.reskv_decode_attn_host.restype = i32
    lib.reskv_free.argtypes = [vp]
    lib.reskv_free.restype = None
    lib.reskv_last_error.argtypes = []
    lib.reskv_last_error.restype = ctypes.c_char_p
    lib.reskv_check_status.argtypes = [vp]
    lib.reskv_check_status.restype = i32
    lib.reskv_get_info.argtypes = [vp, ctypes.POINTER(reskv_cache_info)]
    lib.reskv_get_info.restype = i32
    lib.reskv_get_unit_budgets.argtypes = [vp, ctypes.POINTER(ctypes.c_int32), ctypes.c_int64]
    lib.reskv_get_unit_budgets.restype = i32
    lib.reskv_import_cache.argtypes = [cfgp, ctypes.POINTER(reskv_host_cache), vp,
                                       ctypes.POINTER(vp)]
    lib.reskv_import_cache.restype = i32
    lib.reskv_export_cache.argtypes = [vp, ctypes.POINTER(reskv_host_cache), vp]
    lib.reskv_export_cache.restype = i32
    lib.reskv_export_debug.argtypes = [vp, i32, vp, sz]
    lib.reskv_export_debug.restype = i32
    lib.reskv_append.argtypes = [vp, i32, vp, vp, vp]
    lib.reskv_append.restype = i32
    lib.reskv_decode_attn_noalloc.argtypes = [ctypes.POINTER(reskv_device_cache), vp, vp, vp]
    lib.reskv_decode_attn_noalloc.restype = i32
    lib.reskv_noalloc_check_status.argtypes = [vp, ctypes.POINTER(ctypes.c_int32)]
    lib.reskv_noalloc_check_status.restype = i32
    lib.reskv_test_inject.argtypes = [i32, ctypes.c_int64]
    lib.reskv_test_inject.restype = i32
    ropep, headsp = ctypes.POINTER(reskv_rope_config), ctypes.POINTER(reskv_heads)
    rotp, kvp = ctypes.POINTER(reskv_rotation), ctypes.POINTER(reskv_paged_kv)
    rowsp, attnp = ctypes.POINTER(reskv_rows), ctypes.POINTER(reskv_paged_attn_args)
    i64 = ctypes.c_int64
    lib.reskv_rope_config_default.argtypes = [ropep]
    lib.reskv_rope_config_default.restype = None
    lib.reskv_rope_table.argtypes = [ropep, i64, vp, vp]
    lib.reskv_rope_table.restype = i32
    lib.reskv_rope.argtypes = [rotp, vp, i64, i32, i32, headsp, headsp, i32, vp, vp]
    lib.reskv_rope.restype = i32
    lib.reskv_paged_head_bytes.argtypes = [i32, i32, i32]
    lib.reskv_paged_head_bytes.restype = i64
    lib.reskv_paged_append.argtypes = [kvp, i64, vp, vp, rotp, headsp, headsp, headsp, headsp, vp]
    lib.reskv_paged_append.restype = i32
    lib.reskv_paged_gather.argtypes = [kvp, vp, vp, i64, rowsp, rowsp, vp]
    lib.reskv_paged_gather.restype = i32
    lib.reskv_paged_attn_workspace.argtypes = [kvp, attnp]
    lib.reskv_paged_attn_workspace.restype = sz
    lib.reskv_paged_attn.argtypes = [kvp, attnp, vp]
    lib.reskv_paged_attn.restype = i32
    _lib = lib
    return lib


def _check(status: int):
    if status != RESKV_OK:
        raise ReskvError(status, load_library().reskv_last_error().decode())


def _stream(stream):
    if stream is None:
        import torch
        return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    if isinstance(stream, int):
        return ctypes.c_void_p(stream)
    return ctypes.c_void_p(stream.cuda_stream)


def _dptr(t, dtype_name: str, what: str):
    """Device pointer of a contiguous CUDA tensor of the expected dtype."""
    if not t.is_cuda:
        raise ValueError(f"{what} must be a CUDA tensor")
    if str(t.dtype) != dtype_name:
        raise ValueError(f"{what} must be {dtype_name}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


class Cache:
    """Owning wrapper of a reskv_cache* handle (freed with reskv_free)."""

    def __init__(self, handle: ctypes.c_void_p, cfg: reskv_config):
        self.handle = handle
        self.cfg = cfg

    def free(self):
        if self.handle:
            load_library().reskv_free(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


def reskv_config_default(**fields) -> reskv_config:
    """reskv_config with the paper's defaults, then ``fields`` applied.

    ``grid_ratios`` may be a sequence (sets n_grid); ``residual_override`` and
    ``unit_budgets`` numpy int32 arrays per unit (kept alive on the returned
    struct).
    """
    cfg = reskv_config()
    load_library().reskv_config_default(ctypes.byref(cfg))
    for k, v in fields.items():
        if k == "grid_ratios":
            vals = list(v)
            cfg.n_grid = len(vals)
            for i in range(MAX_GRID):
                cfg.grid_ratios[i] = vals[i] if i < len(vals) else 0.0
        elif k in ("residual_override", "unit_budgets"):
            if v is None:
                setattr(cfg, k, None)
                setattr(cfg, f"_{k}_keepalive", None)
            else:
                arr = np.ascontiguousarray(v, dtype=np.int32)
                setattr(cfg, f"_{k}_keepalive", arr)
                setattr(cfg, k, arr.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)))
        else:
            setattr(cfg, k, v)
    return cfg


def reskv_last_error() -> str:
    return load_library().reskv_last_error().decode()


def reskv_build_cache(cfg: reskv_config, K_layers: Sequence, V_layers: Sequence,
                      Qobs_layers: Optional[Sequence] = None, stream=None) -> Cache:
    """Alg. 1 on the GPU.  K_layers[l], V_layers[l]: bf16 [B, H_kv, s, d] CUDA
    tensors; Qobs_layers[l]: bf16 [B, H_kv*G, n_obs, d] or None."""
    L = cfg.n_layers
    if len(K_layers) != L or len(V_layers) != L:
        raise ValueError("one K and one V tensor per layer")
    kp = (ctypes.c_void_p * L)(*[_dptr(k, "torch.bfloat16", "K").value for k in K_layers])
    vp = (ctypes.c_void_p * L)(*[_dptr(v, "torch.bfloat16", "V").value for v in V_layers])
    qp = None
    if Qobs_layers is not None:
        if len(Qobs_layers) != L:
            raise ValueError("one Qobs tensor per layer")
        qp = (ctypes.c_void_p * L)(*[_dptr(q, "torch.bfloat16", "Qobs").value
                                     for q in Qobs_layers])
    out = ctypes.c_void_p()
    _check(load_library().reskv_build_cache(ctypes.byref(cfg), kp, vp, qp, _stream(stream),
                                            ctypes.byref(out)))
    return Cache(out, cfg)


def reskv_decode_attn(cache: Cache, layer: int, Q, O, stream=None) -> None:
    """Alg. 2.  layer >= 0: Q bf16 [B, H_q, d], O fp32 [B, H_q, d]; layer == -1:
    every layer, Q [L, B, H_q, d] and O likewise."""
    c = cache.cfg
    need = (c.n_layers if layer == -1 else 1) * c.batch * c.n_kv_heads * c.group * c.head_dim
    for name, t in (("Q", Q), ("O", O)):
        if t.numel() != need:
            raise ValueError(f"{name} holds {t.numel()} elements; this call needs {need}")
    _check(load_library().reskv_decode_attn(cache.handle, int(layer),
                                            _dptr(Q, "torch.bfloat16", "Q"),
                                            _dptr(O, "torch.float32", "O"), _stream(stream)))


def reskv_decode_attn_layers(cache: Cache, layer0: int, n_layers: int, Q, O, stream=None) -> None:
    """Alg. 2 for layers layer0 .. layer0 + n_layers - 1 in one launch: Q bf16
    [n_layers, B, H_q, d], O fp32 likewise."""
    c = cache.cfg
    need = int(n_layers) * c.batch * c.n_kv_heads * c.group * c.head_dim
    for name, t in (("Q", Q), ("O", O)):
        if t.numel() != need:
            raise ValueError(f"{name} holds {t.numel()} elements; this call needs {need}")
    _check(load_library().reskv_decode_attn_layers(cache.handle, int(layer0), int(n_layers),
                                                   _dptr(Q, "torch.bfloat16", "Q"),
                                                   _dptr(O, "torch.float32", "O"),
                                                   _stream(stream)))


def _hptr(t, dtype_name: str, what: str):
    """Host pointer of a contiguous CPU tensor of the expected dtype."""
    if t.is_cuda:
        raise ValueError(f"{what} must be a host (CPU) tensor")
    if str(t.dtype) != dtype_name:
        raise ValueError(f"{what} must be {dtype_name}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def reskv_decode_attn_host(cache: Cache, Q_host, O_host, stream=None) -> None:
    """Alg. 2 for every layer with host buffers (pinned for overlap): Q_host
    bf16 [L, B, H_q, d], O_host fp32 likewise.  Asynchronous: O_host is
    complete once the stream has passed the call."""
    c = cache.cfg
    need = c.n_layers * c.batch * c.n_kv_heads * c.group * c.head_dim
    for name, t in (("Q_host", Q_host), ("O_host", O_host)):
        if t.numel() != need:
            raise ValueError(f"{name} holds {t.numel()} elements; this call needs {need}")
    _check(load_library().reskv_decode_attn_host(cache.handle,
                                                 _hptr(Q_host, "torch.bfloat16", "Q_host"),
                                                 _hptr(O_host, "torch.float32", "O_host"),
                                                 _stream(stream)))


def reskv_append(cache: Cache, layer: int, K_new, V_new, stream=None) -> None:
    """Append one token per (batch, KV head) unit: layer >= 0: K_new, V_new
    bf16 [B, H_kv, d]; layer == -1: [L, B, H_kv, d]."""
    c = cache.cfg
    need = (c.n_layers if layer == -1 else 1) * c.batch * c.n_kv_heads * c.head_dim
    for name, t in (("K_new", K_new), ("V_new", V_new)):
        if t.numel() != need:
            raise ValueError(f"{name} holds {t.numel()} elements; this call needs {need}")
    _check(load_library().reskv_append(cache.handle, int(layer),
                                       _dptr(K_new, "torch.bfloat16", "K_new"),
                                       _dptr(V_new, "torch.bfloat16", "V_new"), _stream(stream)))


def reskv_test_inject(what: int, n: int) -> None:
    """Testing only: inject a decode wait timeout or an allocation failure
    (see include/reskv.h)."""
    _check(load_library().reskv_test_inject(int(what), int(n)))


def reskv_free(cache: Cache) -> None:
    cache.free()


def reskv_check_status(cache: Cache) -> None:
    _check(load_library().reskv_check_status(cache.handle))


def reskv_get_info(cache: Cache) -> dict:
    info = reskv_cache_info()
    _check(load_library().reskv_get_info(cache.handle, ctypes.byref(info)))
    out = {f: getattr(info, f) for f, _ in info._fields_}
    out["build_ms"] = list(out["build_ms"])
    return out


def reskv_get_unit_budgets(cache: Cache) -> np.ndarray:
    """Budget b_u of every unit of the handle's layout: int32 [U]."""
    c = cache.cfg
    U = c.n_layers * c.batch * c.n_kv_heads
    out = np.zeros(U, np.int32)
    _check(load_library().reskv_get_unit_budgets(
        cache.handle, out.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), U))
    return out


def _host_view(arrs: dict) -> reskv_host_cache:
    h = reskv_host_cache()
    for k, _ in h._fields_:
        a = arrs.get(k)
        setattr(h, k, None if a is None else a.ctypes.data)
    return h


def reskv_import_cache(cfg: reskv_config, n_main, n_res, kslots, vslots, logc,
                       slot_pos=None, counts=None, n_app=None, stream=None) -> Cache:
    """Build a handle from host numpy arrays (layout as in include/reskv.h):
    kslots/vslots uint16 bf16 bits [U, S, d], logc float32 [U, S], with the
    unit stride S = budget + append_capacity."""
    arrs = dict(n_main=np.ascontiguousarray(n_main, np.int32),
                n_res=np.ascontiguousarray(n_res, np.int32),
                kslots=np.ascontiguousarray(kslots, np.uint16),
                vslots=np.ascontiguousarray(vslots, np.uint16),
                logc=np.ascontiguousarray(logc, np.float32),
                slot_pos=None if slot_pos is None else np.ascontiguousarray(slot_pos, np.int32),
                counts=None if counts is None else np.ascontiguousarray(counts, np.int32),
                n_app=None if n_app is None else np.ascontiguousarray(n_app, np.int32))
    U, d = cfg.n_layers * cfg.batch * cfg.n_kv_heads, cfg.head_dim
    N = unit_offsets(cfg)[-1]
    for k in ("kslots", "vslots", "logc", "slot_pos", "counts"):
        if arrs[k] is not None:                  # [U, S, ...] or flat [N, ...]
            arrs[k] = arrs[k].reshape((N, d) if k in ("kslots", "vslots") else (N,))
    for k, shape in (("n_main", (U,)), ("n_res", (U,)), ("kslots", (N, d)),
                     ("vslots", (N, d)), ("logc", (N,)), ("slot_pos", (N,)),
                     ("counts", (N,)), ("n_app", (U,))):
        if arrs[k] is not None and arrs[k].shape != shape:
            raise ValueError(f"{k} must have shape {shape}, got {arrs[k].shape}")
    h = _host_view(arrs)
    out = ctypes.c_void_p()
    _check(load_library().reskv_import_cache(ctypes.byref(cfg), ctypes.byref(h), _stream(stream),
                                             ctypes.byref(out)))
    return Cache(out, cfg)


def reskv_export_cache(cache: Cache, stream=None) -> dict:
    """Copy the cache layout to host numpy arrays."""
    cfg = cache.cfg
    U, d = cfg.n_layers * cfg.batch * cfg.n_kv_heads, cfg.head_dim
    ragged = bool(reskv_get_info(cache)["ragged"])
    off = (np.concatenate([[0], np.cumsum(reskv_get_unit_budgets(cache).astype(np.int64)
                                          + cfg.append_capacity)])
           if ragged else unit_offsets(cfg))
    N = off[-1]
    arrs = dict(n_main=np.zeros(U, np.int32), n_res=np.zeros(U, np.int32),
                kslots=np.zeros((N, d), np.uint16), vslots=np.zeros((N, d), np.uint16),
                logc=np.zeros(N, np.float32), slot_pos=np.zeros(N, np.int32),
                counts=np.zeros(N, np.int32), n_app=np.zeros(U, np.int32))
    h = _host_view(arrs)
    _check(load_library().reskv_export_cache(cache.handle, ctypes.byref(h), _stream(stream)))
    if ragged:                                   # per-unit budgets: flat arrays plus offsets
        arrs["offsets"] = off
    else:                                        # one stride: [U, S, ...]
        S = cfg.budget + cfg.append_capacity
        for k in ("kslots", "vslots"):
            arrs[k] = arrs[k].reshape(U, S, d)
        for k in ("logc", "slot_pos", "counts"):
            arrs[k] = arrs[k].reshape(U, S)
    return arrs


def unit_offsets(cfg: reskv_config) -> np.ndarray:
    """First slot of every unit (and the total) for cfg's layout: [U + 1]."""
    U = cfg.n_layers * cfg.batch * cfg.n_kv_heads
    if cfg.unit_budgets:
        sizes = np.ctypeslib.as_array(cfg.unit_budgets, shape=(U,)).astype(np.int64)
    else:
        sizes = np.full(U, cfg.budget, np.int64)
    return np.concatenate([[0], np.cumsum(sizes + cfg.append_capacity)]).astype(np.int64)


def reskv_export_debug(cache: Cache, what: int, n_cand: Optional[int] = None) -> np.ndarray:
    """Construction intermediates (cfg.keep_debug must have been set, except
    for the candidate tables).  ``n_cand`` defaults to the handle's count."""
    cfg = cache.cfg
    U = cfg.n_layers * cfg.batch * cfg.n_kv_heads
    s = cfg.seq_len
    info = reskv_get_info(cache)
    nc = info["n_candidates"] if n_cand is None else n_cand
    if what == RESKV_DEBUG_CANDIDATES:
        out = np.zeros(nc, np.int32)
    elif what == RESKV_DEBUG_UNIT_CANDIDATES:
        out = np.zeros((U, nc), np.int32)
    elif what == RESKV_DEBUG_SCORES:
        out = np.zeros((U, s), np.float64)
    elif what == RESKV_DEBUG_RANKED:
        out = np.zeros((U, info["ranked_width"]), np.int32)
    elif what == RESKV_DEBUG_LOSSES:
        out = np.zeros((U, 1 + nc), np.float64)
    else:
        raise ValueError("unknown debug array")
    _check(load_library().reskv_export_debug(cache.handle, int(what),
                                             ctypes.c_void_p(out.ctypes.data), out.nbytes))
    return out


def reskv_decode_attn_noalloc(kslots, vslots, logc, n_main, n_res, n_kv_heads: int, group: int,
                              Q, O, gate_mode: int = RESKV_GATE_DYNAMIC, tau: float = 0.25,
                              alpha: float = 12.0, g_min: float = 0.0, g_fixed: float = 1.0,
                              stream=None) -> None:
    """Decode from a cache held in the caller's own device tensors, with no
    device allocation by the library (see include/reskv.h).

    kslots, vslots: bf16 [U, b, 128]; logc: float32 [U, b]; n_main, n_res:
    int32 [U]; Q: bf16 [U / n_kv_heads, n_kv_heads * group, 128]; O: float32,
    Q's shape.  Every shape is checked here, before the call: the kernel reads
    and writes inside these arrays by their sizes alone.
    """
    if kslots.dim() != 3 or int(kslots.shape[2]) != 128:
        raise ValueError(f"kslots must be [U, b, 128], got {tuple(kslots.shape)}")
    U, b = int(kslots.shape[0]), int(kslots.shape[1])
    H, G = int(n_kv_heads), int(group)
    if H < 1 or U % H != 0:
        raise ValueError(f"n_units {U} is not a multiple of n_kv_heads {H}")
    # row-major arrays of these many elements (any leading shape)
    for name, t, n in (("vslots", vslots, U * b * 128), ("logc", logc, U * b),
                       ("n_main", n_main, U), ("n_res", n_res, U),
                       ("Q", Q, U * G * 128), ("O", O, U * G * 128)):
        if t.numel() != n or (name in ("vslots", "Q", "O") and int(t.shape[-1]) != 128):
            raise ValueError(f"{name} must hold {n} elements (rows of 128 for vslots, Q, O), "
                             f"got shape {tuple(t.shape)}")
    d = reskv_device_cache(
        kslots=_dptr(kslots, "torch.bfloat16", "kslots").value,
        vslots=_dptr(vslots, "torch.bfloat16", "vslots").value,
        logc=_dptr(logc, "torch.float32", "logc").value,
        n_main=_dptr(n_main, "torch.int32", "n_main").value,
        n_res=_dptr(n_res, "torch.int32", "n_res").value,
        n_units=U, budget=b, n_kv_heads=H, group=G,
        gate_mode=int(gate_mode), tau=tau, alpha=alpha, g_min=g_min, g_fixed=g_fixed)
    _check(load_library().reskv_decode_attn_noalloc(ctypes.byref(d),
                                                    _dptr(Q, "torch.bfloat16", "Q"),
                                                    _dptr(O, "torch.float32", "O"),
                                                    _stream(stream)))


def reskv_noalloc_check_status(stream=None) -> int:
    """Read and clear the no-allocation decode's device status word; raises
    ReskvError (RESKV_ERR_DEVICE_STATUS) if a kernel fault was recorded.
    Returns the kernel the thread's last call launched (RESKV_DECODE_MMA or
    RESKV_DECODE_FMA, 0 before the first call)."""
    k = ctypes.c_int32(0)
    _check(load_library().reskv_noalloc_check_status(_stream(stream), ctypes.byref(k)))
    return int(k.value)


# ---------------------------------------------------------------------------
# the full cache before compression: rotary positions and 4-bit pages
# ---------------------------------------------------------------------------

# A decode step makes these calls once per layer and token, so their arguments are
# checked in few steps and packed into the C structs' bytes directly.
_pack_heads = struct.Struct("Pqqii").pack            # reskv_heads
_pack_rotation = struct.Struct("Pqii").pack          # reskv_rotation
_pack_rows = struct.Struct("Pqqqi4x").pack           # reskv_rows
_pack_attn = struct.Struct("PqqiiPqqiiPPPqfiPQ").pack  # reskv_paged_attn_args
_dtypes = {}
_kinds = []                 # torch.int32, torch.float32, the current stream's address of a device
_direct = None
_bind = None                # the same calls from plain CUDA tensors, without Python in between


def _calls():
    """The paged calls with every struct passed as an address or packed bytes."""
    global _direct, _bind
    if _direct is None:
        import torch
        load_library()
        _dtypes.update({torch.bfloat16: RESKV_BF16, torch.float16: RESKV_F16, torch.float32: RESKV_F32})
        _kinds.extend((torch.int32, torch.float32, getattr(torch._C, "_cuda_getCurrentRawStream", None)))
        lib = ctypes.CDLL(LIB_PATH)
        vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
        lib.reskv_rope.argtypes = [vp, vp, i64, i32, i32, vp, vp, i32, vp, vp]
        lib.reskv_paged_append.argtypes = [vp, i64, vp, vp, vp, vp, vp, vp, vp, vp]
        lib.reskv_paged_gather.argtypes = [vp, vp, vp, i64, vp, vp, vp]
        lib.reskv_paged_attn.argtypes = [vp, vp, vp]
        lib.reskv_stream_capturing.argtypes = [vp]
        for f in (lib.reskv_rope, lib.reskv_paged_append, lib.reskv_paged_gather, lib.reskv_paged_attn,
                  lib.reskv_stream_capturing):
            f.restype = i32
        if not os.path.exists(os.path.join(os.path.dirname(LIB_PATH), "_bind.so")):
            raise RuntimeError("_bind.so is missing: build it with `python -m paper_2607_29591_gb300.build` "
                               "(there is no fallback)")
        from . import _bind as bind
        if _kinds[2] is not None:
            bind.setup(*(ctypes.cast(f, ctypes.c_void_p).value for f in
                         (lib.reskv_rope, lib.reskv_paged_append, lib.reskv_paged_gather)), _kinds[2])
            _bind = bind
        _direct = lib
    return _direct


def _stream_of(stream, t) -> int:
    """Address of the stream, by default torch's current one on the tensor's device."""
    if stream is None:
        if _kinds[2] is not None:
            return _kinds[2](t.get_device())
        import torch
        return torch.cuda.current_stream(t.device).cuda_stream
    return stream if isinstance(stream, int) else stream.cuda_stream


def _bad_heads(t, what: str, tokens: int, heads: Optional[int], dim: int):
    if not t.is_cuda:
        raise ValueError(f"{what} must be a CUDA tensor")
    if t.dtype not in _dtypes:
        raise ValueError(f"{what} must be bfloat16, float16 or float32, got {t.dtype}")
    if t.dim() == 3 and t.stride(2) != 1 and t.shape[2] == dim:
        raise ValueError(f"{what}: the elements of a row must lie side by side")
    raise ValueError(f"{what} must be [{tokens}, {'heads' if heads is None else heads}, {dim}], "
                     f"got {tuple(t.shape)}")


def _heads(t, what: str, tokens: int, heads: Optional[int], dim: int):
    """The fields of a reskv_heads: a CUDA tensor [tokens, heads, dim] with neighbouring elements in a row."""
    shape, s, code = t.shape, t.stride(), _dtypes.get(t.dtype)
    if (len(s) != 3 or s[2] != 1 or code is None or shape[0] != tokens or shape[2] != dim
            or (heads is not None and shape[1] != heads) or not t.is_cuda):
        _bad_heads(t, what, tokens, heads, dim)
    return t.data_ptr(), s[0], s[1], shape[1], code


def _ints(t, what: str, n: int) -> int:
    """Address of a contiguous int32 CUDA tensor of n elements."""
    if t.numel() != n:
        raise ValueError(f"{what} must hold {n} elements, got {t.numel()}")
    if t.dtype is not _kinds[0] or not t.is_cuda or not t.is_contiguous():
        return _dptr(t, "torch.int32", what).value
    return t.data_ptr()


def _rotation(table, interleaved: bool) -> bytes:
    shape = table.shape
    if len(shape) != 3 or shape[2] != 2:
        raise ValueError(f"table must be [positions, rot_dim / 2, 2], got {tuple(shape)}")
    if table.dtype is not _kinds[1] or not table.is_cuda or not table.is_contiguous():
        _dptr(table, "torch.float32", "table")
    return _pack_rotation(table.data_ptr(), shape[0], 2 * shape[1], 1 if interleaved else 0)


def reskv_rope_config_default(**fields) -> reskv_rope_config:
    """reskv_rope_config with the defaults, then ``fields`` applied."""
    cfg = reskv_rope_config()
    load_library().reskv_rope_config_default(ctypes.byref(cfg))
    for k, v in fields.items():
        setattr(cfg, k, v)
    return cfg


def reskv_rope_table(cfg: reskv_rope_config, n_positions: int, stream=None):
    """float32 [n_positions, rot_dim / 2, 2] cos and sin of every position on the
    current device."""
    import torch
    table = torch.empty((int(n_positions), cfg.rot_dim // 2, 2), dtype=torch.float32, device="cuda")
    _check(load_library().reskv_rope_table(ctypes.byref(cfg), int(n_positions),
                                           ctypes.c_void_p(table.data_ptr()), _stream(stream)))
    return table


def reskv_rope(q, q_out, positions, table, k=None, k_out=None, interleaved: bool = False,
               backward: bool = False, status=None, stream=None) -> None:
    """Rotate q (and k, in the same launch) by their tokens' positions, or with
    ``backward`` their gradients by the transposed map.

    q, q_out: [T, H, d] bf16, f16 or f32, any token and head strides; q_out may be
    q.  k, k_out likewise with their own heads.  positions: int32 [T]; negative
    ones mark padding (rows copied).  table: float32 [positions, rot_dim / 2, 2]
    (reskv_rope_table); rot_dim < d rotates a part of every head.  status: int32
    [1] that a position outside the table sets to 2.
    """
    if _bind is not None:
        st = _bind.rope(q, q_out, positions, table, k, k_out, interleaved, backward, status, stream)
        if st >= 0:
            return _check(st) if st else None
    if (k is None) != (k_out is None):
        raise ValueError("k and k_out go together")
    if q.dim() != 3:
        raise ValueError(f"q must be [tokens, heads, dim], got {tuple(q.shape)}")
    lib = _calls()
    T, H, d = q.shape
    n, x, y = 1, _pack_heads(*_heads(q, "q", T, None, d)), _pack_heads(*_heads(q_out, "q_out", T, H, d))
    if k is not None:
        kh = _heads(k, "k", T, None, d)
        n, x, y = 2, x + _pack_heads(*kh), y + _pack_heads(*_heads(k_out, "k_out", T, kh[3], d))
    st = lib.reskv_rope(_rotation(table, interleaved), _ints(positions, "positions", T), T, d, n, x, y,
                        1 if backward else 0, None if status is None else _ints(status, "status", 1),
                        _stream_of(stream, q))
    if st:
        _check(st)


def reskv_paged_head_bytes(page_tokens: int, head_dim: int, quant_group: int) -> int:
    """Bytes of one KV head of one page."""
    n = load_library().reskv_paged_head_bytes(int(page_tokens), int(head_dim), int(quant_group))
    if n == 0:
        raise ValueError(f"no page of {page_tokens} tokens, head_dim {head_dim}, quant_group {quant_group}")
    return n


def reskv_paged_pages(n_pages: int, n_kv_heads: int, page_tokens: int = 64, head_dim: int = 128,
                      quant_group: int = 32):
    """Zeroed pages on the current device: uint8 [n_pages, n_kv_heads, bytes]."""
    import torch
    return torch.zeros((n_pages, n_kv_heads, reskv_paged_head_bytes(page_tokens, head_dim, quant_group)),
                       dtype=torch.uint8, device="cuda")


class PagedKV:
    """One layer's paged 4-bit cache: the caller's pages and page table, their
    shape, and a status word that device faults are ORed into.

    pages: uint8, n_pages * n_kv_heads * reskv_paged_head_bytes() bytes;
    page_table: int32 [batch, table_pages], read by every call as it then is.
    """

    def __init__(self, pages, page_table, page_tokens: int, n_kv_heads: int, head_dim: int = 128,
                 quant_group: int = 32, status=None):
        import torch
        _calls()
        per = n_kv_heads * reskv_paged_head_bytes(page_tokens, head_dim, quant_group)
        if pages.numel() % per or pages.numel() == 0:
            raise ValueError(f"pages must hold a multiple of {per} bytes, got {pages.numel()}")
        if page_table.dim() != 2:
            raise ValueError(f"page_table must be [batch, pages], got {tuple(page_table.shape)}")
        self.pages, self.page_table = pages, page_table
        self.batch, self.table_pages = page_table.shape
        self.page_tokens, self.n_kv_heads, self.head_dim, self.quant_group = (
            int(page_tokens), int(n_kv_heads), int(head_dim), int(quant_group))
        self.status = torch.zeros(1, dtype=torch.int32, device=pages.device) if status is None else status
        self.struct = reskv_paged_kv(
            pages=_dptr(pages, "torch.uint8", "pages").value, n_pages=pages.numel() // per,
            page_table=_dptr(page_table, "torch.int32", "page_table").value, batch=self.batch,
            table_pages=self.table_pages, page_tokens=self.page_tokens, n_kv_heads=self.n_kv_heads,
            head_dim=self.head_dim, quant_group=self.quant_group,
            status=_ints(self.status, "status", 1))
        self.address = ctypes.addressof(self.struct)
        self.attn_workspace = {}                 # bytes by (query tokens, heads, output type)

    def check_status(self) -> None:
        """Read and clear the status word (synchronises); raises if a fault was recorded."""
        word = int(self.status.item())
        if word:
            self.status.zero_()
            if word & 1:
                _zero_workspaces(self.status.device)     # what such a call leaves is not ready for the next
            raise ReskvError(RESKV_ERR_DEVICE_STATUS, f"paged cache status word {word} (1 = bounded wait "
                                                      "timed out, 2 = index out of range)")


def reskv_paged_append(kv: PagedKV, k, v, seqs, positions, table=None, interleaved: bool = False,
                       q=None, q_out=None, stream=None) -> None:
    """Hold token i's key (rotated by its position, with ``table``) and value at
    positions[i] of sequence seqs[i]; with q, rotate the tokens' queries into
    q_out in the same call.

    k, v: [T, n_kv_heads, d], one of bf16, f16, f32; seqs, positions: int32 [T],
    negative positions mark padding; q, q_out: [T, heads, d].
    """
    if _bind is not None:
        st = _bind.append(kv.address, k, v, seqs, positions, table, interleaved, q, q_out, stream)
        if st >= 0:
            return _check(st) if st else None
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out go together")
    lib = _calls()
    T, heads, d = k.shape[0], kv.n_kv_heads, kv.head_dim
    kh = _pack_heads(*_heads(k, "k", T, heads, d))
    vh = _pack_heads(*_heads(v, "v", T, heads, d))
    qh = qo = None
    if q is not None:
        f = _heads(q, "q", T, None, d)
        qh, qo = _pack_heads(*f), _pack_heads(*_heads(q_out, "q_out", T, f[3], d))
    st = lib.reskv_paged_append(kv.address, T, _ints(seqs, "seqs", T), _ints(positions, "positions", T),
                                None if table is None else _rotation(table, interleaved), kh, vh, qh, qo,
                                _stream_of(stream, k))
    if st:
        _check(st)


def _rows(t, what: str, kv: PagedKV, n: int) -> bytes:
    s, code = t.stride(), _dtypes.get(t.dtype)
    if not t.is_cuda or code is None:
        raise ValueError(f"{what} must be a CUDA tensor of bfloat16, float16 or float32")
    if t.shape != (kv.batch, kv.n_kv_heads, n, kv.head_dim) or s[3] != 1:
        raise ValueError(f"{what} must be [{kv.batch}, {kv.n_kv_heads}, {n}, {kv.head_dim}] with neighbouring "
                         f"elements in a row, got {tuple(t.shape)}")
    return _pack_rows(t.data_ptr(), s[0], s[1], s[2], code)


def reskv_paged_gather(kv: PagedKV, lens, k_out=None, v_out=None, starts=None, stream=None) -> None:
    """The values held at positions starts[b] .. starts[b] + n - 1 (starts None:
    from 0) into k_out, v_out [batch, n_kv_heads, n, d] bf16, f16 or f32; rows at
    positions >= lens[b] are zero.  starts, lens: int32 [batch]."""
    if _bind is not None:
        st = _bind.gather(kv.address, lens, k_out, v_out, starts, stream, kv.pages)
        if st >= 0:
            return _check(st) if st else None
    if k_out is None and v_out is None:
        raise ValueError("k_out or v_out is needed")
    lib = _calls()
    n = (v_out if k_out is None else k_out).shape[2]
    st = lib.reskv_paged_gather(kv.address, None if starts is None else _ints(starts, "starts", kv.batch),
                                _ints(lens, "lens", kv.batch), n,
                                None if k_out is None else _rows(k_out, "k_out", kv, n),
                                None if v_out is None else _rows(v_out, "v_out", kv, n),
                                _stream_of(stream, kv.pages))
    if st:
        _check(st)


_workspaces = {}


def _workspace(device, stream: int, nbytes: int):
    """Zeroed workspaces of a device and stream, the last the largest; what one
    grew from is kept (calls on the stream may still be using it)."""
    import torch
    new = torch.zeros(nbytes, dtype=torch.uint8, device=device)
    torch.cuda.current_stream(device).synchronize()      # zeroed before it is any call's
    held = _workspaces.setdefault((device.index, stream), [])
    held.append(new)
    return held


def _zero_workspaces(device) -> None:
    """Make the kept workspaces of a device ready again, in place: what runs there may hold their addresses."""
    import torch
    torch.cuda.synchronize(device)
    for (index, _), held in list(_workspaces.items()):
        if index == device.index:
            for w in held:
                w.zero_()
    torch.cuda.synchronize(device)


def reskv_paged_attn(kv: PagedKV, q, lens, o, q_begin=None, scale: Optional[float] = None, window: int = 0,
                     lse=None, workspace=None, stream=None) -> None:
    """Attention of every sequence's newest tokens over its cache.

    q: bf16 or f16 [T, heads, d], sequence b's query tokens rows q_begin[b] ..
    q_begin[b + 1] - 1 (int32 [batch + 1]; None: T / batch each), the last of the
    lens[b] tokens it holds; o: [T, heads, d] of q's dtype or float32.  window:
    positions a query sees, itself included (0: all).  scale: of the logits (None
    or 0: 1 / sqrt(d)).  lse: float32 [T, heads]
    for ln sum exp, or None.  workspace: zeroed uint8 tensor of at least
    reskv_paged_attn_workspace() bytes (None: one kept per stream); a call that is
    captured into a graph brings its own.
    """
    lib = _calls()
    T, d, B = q.shape[0], kv.head_dim, kv.batch
    qh = _heads(q, "q", T, None, d)
    oh = _heads(o, "o", T, qh[3], d)
    if lse is not None and lse.numel() != T * qh[3]:
        raise ValueError(f"lse must hold {T * qh[3]} elements, got {lse.numel()}")
    s = _stream_of(stream, q)
    if workspace is None:
        if lib.reskv_stream_capturing(s):
            raise ValueError("a call that is captured into a graph needs workspace=: a zeroed uint8 tensor of "
                             "reskv_paged_attn_workspace() bytes, made before the capture")
        need = kv.attn_workspace.get((T, qh[3], oh[4]))
        if need is None:
            need = kv.attn_workspace[T, qh[3], oh[4]] = reskv_paged_attn_workspace(kv, T, qh[3], o.dtype)
        held = _workspaces.get((q.get_device(), s))
        if held is None or held[-1].numel() < need:
            held = _workspace(q.device, s, need)
        workspace = held[-1]
    elif not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous CUDA tensor")
    st = lib.reskv_paged_attn(kv.address, _pack_attn(
        *qh, *oh, 0 if lse is None else _dptr(lse, "torch.float32", "lse").value,
        0 if q_begin is None else _ints(q_begin, "q_begin", B + 1), _ints(lens, "lens", B), T,
        0.0 if scale is None else scale, window, workspace.data_ptr(),
        workspace.numel() * workspace.element_size()), s)
    if st:
        _check(st)


def reskv_paged_attn_workspace(kv: PagedKV, n_tokens: int, heads: int, out_dtype=None) -> int:
    """Workspace bytes of a reskv_paged_attn call over n_tokens query tokens
    (outputs of out_dtype; None: the most any type needs)."""
    import torch
    _calls()
    a = reskv_paged_attn_args(n_tokens=n_tokens)
    a.q.n_heads = heads
    a.o.dtype = _dtypes[torch.bfloat16 if out_dtype is None else out_dtype]
    return load_library().reskv_paged_attn_workspace(kv.struct, a)
