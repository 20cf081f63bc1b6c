"""Thin binding over the C-ABI library (include/rt.h): argument marshalling only.

Importing this module loads `librt_b200.so` from the package directory and fails loudly
when it is missing or lacks a symbol -- there is no CPU fallback.  Module-level functions
carry the C names (`rt_layer_prefill`, ...) and take raw device pointers; `Layer` and
`Stack` are small conveniences that keep weights, caches and the workspace as torch tensors
(torch is used for device memory and streams only).
"""
from __future__ import annotations

import ctypes as C
import math
import os
from typing import Dict, List, Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "librt_b200.so")

RT_OK, RT_ERR_INVALID_ARG, RT_ERR_UNSUPPORTED, RT_ERR_WORKSPACE, RT_ERR_CUDA, RT_ERR_TIMEOUT = range(6)
RT_F32, RT_BF16, RT_E4M3 = 0, 1, 2
RT_SCHED_TILED, RT_SCHED_NAIVE = 0, 1
RT_NORM_PRE, RT_NORM_QK, RT_NORM_SKIP_Z = 1, 2, 8
RT_FLAG_BACKWARD_STEP_LAUNCHES = 1
RT_PAIRS_HALVES, RT_PAIRS_NEIGHBOURS = 0, 1

EXPORTS = ("rt_workspace_bytes", "rt_layer_prefill", "rt_stack_prefill", "rt_decode_step",
           "rt_layer_decode_step", "rt_get_status", "rt_status_string", "rt_plan_counters", "rt_plan_tiles",
           "rt_profile_enable", "rt_profile_read", "rt_layer_decode_step_static", "rt_update_tile", "rt_selftest_wait_expiry",
           "rt_recompute_workspace_bytes", "rt_layer_recompute", "rt_backward_workspace_bytes", "rt_layer_backward",
           "rt_static_get_status", "rt_cache_write", "rt_cache_read", "rt_paged_attention_workspace_bytes", "rt_paged_attention",
           "rt_qk_rotate", "rt_qk_rotate_backward_workspace_bytes", "rt_qk_rotate_backward")
RT_STATIC_SCRATCH_BYTES = 8 << 20


class RtConfig(C.Structure):
    _fields_ = [("d_model", C.c_int32), ("n_heads", C.c_int32), ("head_dim", C.c_int32), ("d_ff", C.c_int32),
                ("dtype", C.c_int32), ("sched", C.c_int32), ("leaf", C.c_int32), ("norm_flags", C.c_int32),
                ("rms_eps", C.c_float), ("softmax_scale", C.c_float), ("residual_scale", C.c_float),
                ("recur_block", C.c_int32), ("flags", C.c_int32)]


class RtLayerWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("w_q", "w_k", "w_v", "w_o", "w_up", "w_down",
                                           "g_attn", "g_mlp", "g_kv", "g_q", "g_k", "alibi_slopes")]


class RtLayerGrads(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("w_q", "w_k", "w_v", "w_o", "w_up", "w_down",
                                           "g_attn", "g_mlp", "g_kv", "g_q", "g_k")]


class RtCounters(C.Structure):
    _fields_ = [(n, C.c_uint64) for n in ("model_bytes_read", "model_bytes_written", "flops_tile", "flops_leaf",
                                           "flops_gemm", "kv_bytes_read", "leaf_kv_bytes_l2", "n_tiles", "n_leaves")]


class RtProfile(C.Structure):
    _fields_ = [("ms", C.c_double * 4), ("launches", C.c_uint64 * 4)]


class RtPagedCache(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k", "v", "k_exp", "v_exp", "page_table", "status")] + \
               [(n, C.c_int32) for n in ("n_pages", "page_size", "n_kv_heads", "head_dim", "dtype", "n_seqs", "max_pages")]


class RtPagedQuery(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("q", "k_own", "v_own", "lens", "alibi_slopes", "out", "lse")] + \
               [(n, C.c_int64) for n in ("q_stride", "k_own_stride", "v_own_stride", "out_stride")] + \
               [("dtype", C.c_int32), ("n_heads", C.c_int32), ("softmax_scale", C.c_float)]


class RtRotateConfig(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("norm_flags", C.c_int32), ("rms_eps", C.c_float), ("rot_dim", C.c_int32), ("pairs", C.c_int32),
                ("freq", C.POINTER(C.c_double))]


PROFILE_CLASSES = ("prepass", "leaf", "tile", "other")


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python __graft_entry__.py` (needs nvcc); "
                          "this package has no CPU fallback")
    lib = C.CDLL(LIB_PATH)
    for name in EXPORTS:
        if not hasattr(lib, name):
            raise ImportError(f"{LIB_PATH} does not export {name}")
    P, I, Z = C.c_void_p, C.c_int32, C.c_size_t
    lib.rt_workspace_bytes.restype = Z
    lib.rt_workspace_bytes.argtypes = [C.POINTER(RtConfig), I, I, I]
    lib.rt_layer_prefill.restype = C.c_int
    lib.rt_layer_prefill.argtypes = [C.POINTER(RtConfig), C.POINTER(RtLayerWeights), P, I, I, P, P, P, I, P, Z, P]
    lib.rt_layer_decode_step.restype = C.c_int
    lib.rt_layer_decode_step.argtypes = [C.POINTER(RtConfig), C.POINTER(RtLayerWeights), P, I, I, P, P, P, I, P, Z, P]
    lib.rt_layer_decode_step_static.restype = C.c_int
    lib.rt_layer_decode_step_static.argtypes = [C.POINTER(RtConfig), C.POINTER(RtLayerWeights), P, I, I, P, P, P, I, P]
    lib.rt_static_get_status.restype = C.c_int
    lib.rt_static_get_status.argtypes = []
    lib.rt_selftest_wait_expiry.restype = C.c_int
    lib.rt_selftest_wait_expiry.argtypes = [P, P]
    lib.rt_recompute_workspace_bytes.restype = Z
    lib.rt_recompute_workspace_bytes.argtypes = [C.POINTER(RtConfig), I, I]
    lib.rt_layer_recompute.restype = C.c_int
    lib.rt_backward_workspace_bytes.restype = Z
    lib.rt_backward_workspace_bytes.argtypes = [C.POINTER(RtConfig), I, I]
    lib.rt_layer_backward.restype = C.c_int
    lib.rt_layer_backward.argtypes = [C.POINTER(RtConfig), C.POINTER(RtLayerWeights), P, P, P, I, I, P, C.POINTER(RtLayerGrads), P, Z, P]
    lib.rt_layer_recompute.argtypes = [C.POINTER(RtConfig), C.POINTER(RtLayerWeights), P, P, I, I, P, P, P, I, P, Z, P]
    lib.rt_update_tile.restype = C.c_int
    lib.rt_update_tile.argtypes = [C.POINTER(RtConfig), P, P, P, P, P, P, I, I, I, I, I, I, I, P, P, P]
    lib.rt_stack_prefill.restype = C.c_int
    lib.rt_stack_prefill.argtypes = [C.POINTER(RtConfig), I, C.POINTER(RtLayerWeights), P, P, I, P, I, I, P, P,
                                     C.POINTER(P), C.POINTER(P), I, P, Z, P]
    lib.rt_decode_step.restype = C.c_int
    lib.rt_decode_step.argtypes = [C.POINTER(RtConfig), I, C.POINTER(RtLayerWeights), P, P, I, P, I, I, P,
                                   C.POINTER(P), C.POINTER(P), I, P, Z, P]
    L = C.c_int64
    lib.rt_cache_write.restype = lib.rt_cache_read.restype = C.c_int
    lib.rt_cache_write.argtypes = lib.rt_cache_read.argtypes = [C.POINTER(RtPagedCache), I, P, P, L, L, P, P, I, P]
    lib.rt_paged_attention_workspace_bytes.restype = Z
    lib.rt_paged_attention_workspace_bytes.argtypes = [C.POINTER(RtPagedCache), I]
    lib.rt_paged_attention.restype = C.c_int
    lib.rt_paged_attention.argtypes = [C.POINTER(RtPagedCache), C.POINTER(RtPagedQuery), P, Z, P]
    lib.rt_qk_rotate.restype = C.c_int
    lib.rt_qk_rotate.argtypes = [C.POINTER(RtRotateConfig), P, P, L, L, P, P, P, I, P, P, L, L, P]
    lib.rt_qk_rotate_backward_workspace_bytes.restype = Z
    lib.rt_qk_rotate_backward_workspace_bytes.argtypes = [C.POINTER(RtRotateConfig), I]
    lib.rt_qk_rotate_backward.restype = C.c_int
    lib.rt_qk_rotate_backward.argtypes = [C.POINTER(RtRotateConfig), P, P, L, L, P, P, P, I, P, P, P, P, P, P, P, Z, P]
    lib.rt_get_status.restype = C.c_int
    lib.rt_get_status.argtypes = [P]
    lib.rt_status_string.restype = C.c_char_p
    lib.rt_status_string.argtypes = [C.c_int]
    lib.rt_plan_counters.restype = C.c_int
    lib.rt_plan_counters.argtypes = [C.POINTER(RtConfig), I, I, I, I, C.POINTER(RtCounters)]
    lib.rt_plan_tiles.restype = I
    lib.rt_plan_tiles.argtypes = [I, I, C.POINTER(I), I]
    lib.rt_profile_enable.restype = C.c_int
    lib.rt_profile_enable.argtypes = [I]
    lib.rt_profile_read.restype = C.c_int
    lib.rt_profile_read.argtypes = [C.POINTER(RtProfile)]
    return lib


_lib = _load()


class RtError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {rt_status_string(status)} (rt_status {status})")


def _check(status: int, where: str):
    if status != RT_OK:
        raise RtError(status, where)


# ------------------------------------------------------------------ the C names

def rt_status_string(status: int) -> str:
    return _lib.rt_status_string(int(status)).decode()


def rt_workspace_bytes(cfg: RtConfig, B: int, N: int, n_layers: int = 1) -> int:
    return int(_lib.rt_workspace_bytes(C.byref(cfg), B, N, n_layers))


def rt_layer_prefill(cfg, w, x, B, N, z, k_cache, v_cache, N_max, workspace, workspace_bytes, stream) -> int:
    return _lib.rt_layer_prefill(C.byref(cfg), C.byref(w), x, B, N, z, k_cache, v_cache, N_max, workspace,
                                 workspace_bytes, stream)


def rt_layer_decode_step(cfg, w, x, B, pos, z, k_cache, v_cache, N_max, workspace, workspace_bytes, stream) -> int:
    return _lib.rt_layer_decode_step(C.byref(cfg), C.byref(w), x, B, pos, z, k_cache, v_cache, N_max, workspace,
                                     workspace_bytes, stream)


def rt_layer_decode_step_static(cfg, w, x, B, pos, z, k_cache, v_cache, N_max, stream) -> int:
    """Decode step for callers that cannot allocate: no workspace argument, the scratch is a fixed
    array inside the library (see include/rt.h).  Calls on one device must not overlap."""
    return _lib.rt_layer_decode_step_static(C.byref(cfg), C.byref(w), x, B, pos, z, k_cache, v_cache, N_max, stream)


def rt_static_get_status() -> int:
    """Device status word of the last rt_layer_decode_step_static call on the current device (after a synchronise)."""
    return _lib.rt_static_get_status()


def rt_stack_prefill(cfg, n_layers, layers, emb, g_final, vocab, ids, B, N, hidden, logits_last, k_caches, v_caches,
                     N_max, workspace, workspace_bytes, stream) -> int:
    return _lib.rt_stack_prefill(C.byref(cfg), n_layers, layers, emb, g_final, vocab, ids, B, N, hidden, logits_last,
                                 k_caches, v_caches, N_max, workspace, workspace_bytes, stream)


def rt_decode_step(cfg, n_layers, layers, emb, g_final, vocab, ids, B, pos, logits, k_caches, v_caches, N_max,
                   workspace, workspace_bytes, stream) -> int:
    return _lib.rt_decode_step(C.byref(cfg), n_layers, layers, emb, g_final, vocab, ids, B, pos, logits, k_caches,
                               v_caches, N_max, workspace, workspace_bytes, stream)


def rt_update_tile(cfg, q, k_cache, v_cache, st_o, st_m, st_l, B, rows_q, rows_kv, q0, q1, k0, k1, alibi_slopes,
                   workspace, stream) -> int:
    return _lib.rt_update_tile(C.byref(cfg), q, k_cache, v_cache, st_o, st_m, st_l, B, rows_q, rows_kv, q0, q1, k0, k1,
                               alibi_slopes, workspace, stream)


def rt_recompute_workspace_bytes(cfg: RtConfig, B: int, N: int) -> int:
    return int(_lib.rt_recompute_workspace_bytes(C.byref(cfg), B, N))


def rt_backward_workspace_bytes(cfg: RtConfig, B: int, N: int) -> int:
    return int(_lib.rt_backward_workspace_bytes(C.byref(cfg), B, N))


def rt_layer_backward(cfg, w, x, z, dz, B, N, dx, grads, workspace, workspace_bytes, stream) -> int:
    return _lib.rt_layer_backward(C.byref(cfg), C.byref(w), x, z, dz, B, N, dx, C.byref(grads), workspace, workspace_bytes, stream)


def rt_layer_recompute(cfg, w, x, z_claim, B, N, z_out, k_cache, v_cache, N_max, workspace, workspace_bytes, stream) -> int:
    return _lib.rt_layer_recompute(C.byref(cfg), C.byref(w), x, z_claim, B, N, z_out, k_cache, v_cache, N_max, workspace,
                                   workspace_bytes, stream)


def rt_cache_write(cache, dtype, k, v, k_stride, v_stride, seq, pos, rows, stream) -> int:
    return _lib.rt_cache_write(C.byref(cache), dtype, k, v, k_stride, v_stride, seq, pos, rows, stream)


def rt_cache_read(cache, dtype, k, v, k_stride, v_stride, seq, pos, rows, stream) -> int:
    return _lib.rt_cache_read(C.byref(cache), dtype, k, v, k_stride, v_stride, seq, pos, rows, stream)


def rt_paged_attention_workspace_bytes(cache: RtPagedCache, n_heads: int) -> int:
    return int(_lib.rt_paged_attention_workspace_bytes(C.byref(cache), n_heads))


def rt_paged_attention(cache, query, workspace, workspace_bytes, stream) -> int:
    return _lib.rt_paged_attention(C.byref(cache), C.byref(query), workspace, workspace_bytes, stream)


def rt_qk_rotate(cfg, q, k, q_stride, k_stride, g_q, g_k, pos, rows, q_out, k_out, q_out_stride, k_out_stride, stream) -> int:
    return _lib.rt_qk_rotate(C.byref(cfg), q, k, q_stride, k_stride, g_q, g_k, pos, rows, q_out, k_out, q_out_stride, k_out_stride, stream)


def rt_qk_rotate_backward_workspace_bytes(cfg: RtRotateConfig, rows: int) -> int:
    return int(_lib.rt_qk_rotate_backward_workspace_bytes(C.byref(cfg), rows))


def rt_qk_rotate_backward(cfg, q, k, q_stride, k_stride, g_q, g_k, pos, rows, dq_out, dk_out, dq, dk, dg_q, dg_k, workspace, workspace_bytes,
                          stream) -> int:
    return _lib.rt_qk_rotate_backward(C.byref(cfg), q, k, q_stride, k_stride, g_q, g_k, pos, rows, dq_out, dk_out, dq, dk, dg_q, dg_k,
                                      workspace, workspace_bytes, stream)


def rt_selftest_wait_expiry(workspace, stream) -> int:
    return _lib.rt_selftest_wait_expiry(workspace, stream)


def rt_get_status(workspace) -> int:
    return _lib.rt_get_status(workspace)


def rt_plan_counters(cfg: RtConfig, B: int, N: int, n_layers: int = 1, vocab: int = 0) -> Dict[str, int]:
    out = RtCounters()
    _check(_lib.rt_plan_counters(C.byref(cfg), B, N, n_layers, vocab, C.byref(out)), "rt_plan_counters")
    return {n: int(getattr(out, n)) for n, _ in RtCounters._fields_}


def rt_plan_tiles(N: int, leaf: int) -> List[tuple]:
    n = _lib.rt_plan_tiles(N, leaf, None, 0)
    buf = (C.c_int32 * (4 * max(n, 1)))()
    _lib.rt_plan_tiles(N, leaf, buf, n)
    return [tuple(buf[4 * i:4 * i + 4]) for i in range(n)]


def rt_profile_enable(on) -> None:
    """False/0: off; True/1: event spans per kernel class; 2: also the leaf kernels' in-kernel phase timers."""
    _check(_lib.rt_profile_enable(int(on)), "rt_profile_enable")


def rt_profile_read() -> Dict[str, Dict[str, float]]:
    out = RtProfile()
    _check(_lib.rt_profile_read(C.byref(out)), "rt_profile_read")
    return {n: {"ms": float(out.ms[i]), "launches": int(out.launches[i])} for i, n in enumerate(PROFILE_CLASSES)}


def make_config(d_model: int, n_heads: int, d_ff: int, dtype: str = "bf16", sched: str = "tiled", leaf: int = 0,
                norm_flags: int = RT_NORM_PRE | RT_NORM_QK, rms_eps: float = 1e-6,
                softmax_scale: Optional[float] = None, residual_scale: float = 1.0, head_dim: int = 64,
                recur_block: int = 0, flags: int = 0) -> RtConfig:
    return RtConfig(d_model, n_heads, head_dim, d_ff, {"f32": RT_F32, "bf16": RT_BF16}[dtype],
                    {"tiled": RT_SCHED_TILED, "naive": RT_SCHED_NAIVE}[sched], leaf, norm_flags, rms_eps,
                    (1.0 / math.sqrt(head_dim)) if softmax_scale is None else softmax_scale, residual_scale, recur_block, flags)


# ------------------------------------------------------------------ conveniences on torch tensors

_torch_module = _device_now = _stream_now = None


def _torch():
    global _torch_module, _device_now, _stream_now
    if _torch_module is None:
        import torch
        _torch_module = torch
        # the current device, and a device's current stream as a number (torch.cuda.current_stream builds an object for it, 2 us);
        # a torch without CUDA has neither, and the calls that need them refuse its arrays
        _device_now = getattr(torch._C, "_cuda_getDevice", lambda: -1)
        _stream_now = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return _torch_module


def _tdtype(dtype: str):
    torch = _torch()
    return {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]


def _to_dev(a, dtype: str, device):
    torch = _torch()
    if isinstance(a, np.ndarray):
        a = torch.from_numpy(np.ascontiguousarray(a))
    return a.to(device=device, dtype=_tdtype(dtype)).contiguous()


def _require(ok: bool, where: str):
    """What ctypes cannot see of a tensor (its device, type, shape, the order of its dimensions) is refused like a bad argument of the call."""
    if not ok:
        raise RtError(RT_ERR_INVALID_ARG, where)


def _rows(t, heads: int, head_dim: int, n: int, dtype, index: int, where: str) -> tuple:
    """(address, stride) of [n, heads, head_dim] or [n, heads * head_dim] rows on CUDA device `index` whose heads are contiguous."""
    if t.dtype is dtype and t.get_device() == index:
        sh = t.shape
        if t.is_contiguous() and (sh == (n, heads, head_dim) or sh == (n, heads * head_dim)):
            return t.data_ptr(), heads * head_dim
        st = t.stride()
        if (sh == (n, heads, head_dim) and st[2] == 1 and (heads == 1 or st[1] == head_dim)) or (sh == (n, heads * head_dim) and st[1] == 1):
            return t.data_ptr(), st[0]
    raise RtError(RT_ERR_INVALID_ARG, where)


def _vector(t, n: int, dtype, index: int, where: str):
    """Address of a contiguous array of n elements on CUDA device `index`, None for None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != n or t.get_device() != index or not t.is_contiguous():
        raise RtError(RT_ERR_INVALID_ARG, where)
    return t.data_ptr()


_W_NAMES = ("w_q", "w_k", "w_v", "w_o", "w_up", "w_down")
_G_NAMES = ("g_attn", "g_mlp", "g_kv", "g_q", "g_k")


def _pack_weights(wd: dict, dtype: str, device):
    """dict of arrays -> (RtLayerWeights, list of tensors kept alive)"""
    keep, st = [], RtLayerWeights()
    for n in _W_NAMES:
        t = _to_dev(wd[n], dtype, device)
        keep.append(t)
        setattr(st, n, t.data_ptr())
    for n in _G_NAMES:
        if wd.get(n) is not None:
            t = _to_dev(wd[n], dtype, device)
            keep.append(t)
            setattr(st, n, t.data_ptr())
    if wd.get("alibi_slopes") is not None:           # [n_heads], always fp32
        t = _to_dev(np.asarray(wd["alibi_slopes"], dtype=np.float64), "f32", device)
        keep.append(t)
        st.alibi_slopes = t.data_ptr()
    return st, keep


class Layer:
    """One RT layer with its weights, K/V cache and workspace resident on the device."""

    def __init__(self, d_model: int, n_heads: int, d_ff: int, dtype: str = "bf16", device: str = "cuda:0", **cfg_kw):
        torch = _torch()
        self.dtype, self.device = dtype, torch.device(device)
        self.cfg = make_config(d_model, n_heads, d_ff, dtype=dtype, **cfg_kw)
        self.w: Optional[RtLayerWeights] = None
        self._keep: list = []
        self.k_cache = self.v_cache = self.ws = None
        self.N_max = 0

    def set_weights(self, wd: dict):
        self.w, self._keep = _pack_weights(wd, self.dtype, self.device)

    def reserve(self, B: int, N: int, N_max: Optional[int] = None):
        torch = _torch()
        N_max = N if N_max is None else N_max
        d = self.cfg.d_model
        if self.k_cache is None or tuple(self.k_cache.shape) != (N_max, B, d):
            self.k_cache = torch.zeros((N_max, B, d), dtype=_tdtype(self.dtype), device=self.device)
            self.v_cache = torch.zeros_like(self.k_cache)
            self.N_max = N_max
        need = rt_workspace_bytes(self.cfg, B, N, 1)
        if need == 0:
            raise RtError(RT_ERR_INVALID_ARG, "rt_workspace_bytes")
        if self.ws is None or self.ws.numel() < need:
            self.ws = torch.zeros(need, dtype=torch.uint8, device=self.device)

    def prefill_device(self, x_dev, z_dev, stream=None) -> None:
        """x_dev, z_dev: contiguous [B, N, d] device tensors of the storage type (enqueue only)."""
        torch = _torch()
        B, N, _ = x_dev.shape
        s = torch.cuda.current_stream(self.device).cuda_stream if stream is None else stream
        _check(rt_layer_prefill(self.cfg, self.w, x_dev.data_ptr(), B, N, z_dev.data_ptr(), self.k_cache.data_ptr(),
                                self.v_cache.data_ptr(), self.N_max, self.ws.data_ptr(), self.ws.numel(), s),
               "rt_layer_prefill")

    def status(self) -> int:
        return rt_get_status(self.ws.data_ptr())

    def prefill(self, x, N_max: Optional[int] = None):
        """x [B,N,d] (numpy or tensor) -> z, k, v as fp64 numpy arrays, each [B,N,d]."""
        torch = _torch()
        xd = _to_dev(x, self.dtype, self.device)
        B, N, _ = xd.shape
        self.reserve(B, N, N_max)
        zd = torch.empty_like(xd)
        self.prefill_device(xd, zd)
        torch.cuda.synchronize(self.device)
        _check(self.status(), "rt_layer_prefill (device)")
        to_np = lambda t: t.to(torch.float64).cpu().numpy()
        return (to_np(zd), to_np(self.k_cache[:N].permute(1, 0, 2)), to_np(self.v_cache[:N].permute(1, 0, 2)))

    def recompute(self, x, z_claim):
        """One parallel sweep: x, z_claim [B,N,d] -> z', k, v (fp64 numpy, each [B,N,d]); the caches are rebuilt from z_claim."""
        torch = _torch()
        xd = _to_dev(x, self.dtype, self.device)
        zc = _to_dev(z_claim, self.dtype, self.device)
        B, N, _ = xd.shape
        self.reserve(B, N)
        need = rt_recompute_workspace_bytes(self.cfg, B, N)
        if self.ws.numel() < need:
            self.ws = torch.zeros(need, dtype=torch.uint8, device=self.device)
        zo = torch.empty_like(xd)
        s = torch.cuda.current_stream(self.device).cuda_stream
        _check(rt_layer_recompute(self.cfg, self.w, xd.data_ptr(), zc.data_ptr(), B, N, zo.data_ptr(), self.k_cache.data_ptr(),
                                  self.v_cache.data_ptr(), self.N_max, self.ws.data_ptr(), self.ws.numel(), s), "rt_layer_recompute")
        torch.cuda.synchronize(self.device)
        _check(self.status(), "rt_layer_recompute (device)")
        to_np = lambda t: t.to(torch.float64).cpu().numpy()
        return (to_np(zo), to_np(self.k_cache[:N].permute(1, 0, 2)), to_np(self.v_cache[:N].permute(1, 0, 2)))

    def backward_device(self, x_dev, z_dev, dz_dev, dx_dev, grads: "RtLayerGrads", ws, stream=None) -> None:
        """x_dev, z_dev [B,N,d] storage type, dz_dev, dx_dev [B,N,d] fp32, ws a uint8 workspace tensor (enqueue only)."""
        torch = _torch()
        B, N, _ = x_dev.shape
        s = torch.cuda.current_stream(self.device).cuda_stream if stream is None else stream
        _check(rt_layer_backward(self.cfg, self.w, x_dev.data_ptr(), z_dev.data_ptr(), dz_dev.data_ptr(), B, N, dx_dev.data_ptr(),
                                 grads, ws.data_ptr(), ws.numel(), s), "rt_layer_backward")

    def backward(self, x, z, dz):
        """x, z [B,N,d] (z = this layer's outputs), dz = dL/dz [B,N,d] -> dx [B,N,d] and a dict of parameter gradients
        (fp64 numpy; one entry per parameter the layer has)."""
        torch = _torch()
        xd = _to_dev(x, self.dtype, self.device)
        zd = _to_dev(z, self.dtype, self.device)
        dzd = _to_dev(dz, "f32", self.device)
        B, N, d = xd.shape
        need = rt_backward_workspace_bytes(self.cfg, B, N)
        if need == 0:
            raise RtError(RT_ERR_INVALID_ARG, "rt_backward_workspace_bytes")
        ws = torch.zeros(need, dtype=torch.uint8, device=self.device)
        dxd = torch.empty((B, N, d), dtype=torch.float32, device=self.device)
        grads, out = RtLayerGrads(), {}
        shapes = {"w_up": (self.cfg.d_ff, d), "w_down": (d, self.cfg.d_ff)}
        for n in _W_NAMES + _G_NAMES:
            if n in _G_NAMES and not getattr(self.w, n):
                continue
            out[n] = torch.empty(shapes.get(n, (d, d) if n in _W_NAMES else (d,)), dtype=torch.float32, device=self.device)
            setattr(grads, n, out[n].data_ptr())
        self.backward_device(xd, zd, dzd, dxd, grads, ws)
        torch.cuda.synchronize(self.device)
        _check(rt_get_status(ws.data_ptr()), "rt_layer_backward (device)")
        to_np = lambda t: t.to(torch.float64).cpu().numpy()
        return to_np(dxd), {n: to_np(t) for n, t in out.items()}

    def decode(self, x_new, pos: int):
        """x_new [B,d] at position pos (caches must hold pos rows) -> z_new [B,d] fp64 numpy."""
        torch = _torch()
        xd = _to_dev(x_new, self.dtype, self.device)
        B, _ = xd.shape
        zd = torch.empty_like(xd)
        need = rt_workspace_bytes(self.cfg, B, 1, 1)
        if self.ws is None or self.ws.numel() < need:
            self.ws = torch.zeros(need, dtype=torch.uint8, device=self.device)
        s = torch.cuda.current_stream(self.device).cuda_stream
        _check(rt_layer_decode_step(self.cfg, self.w, xd.data_ptr(), B, pos, zd.data_ptr(), self.k_cache.data_ptr(),
                                    self.v_cache.data_ptr(), self.N_max, self.ws.data_ptr(), self.ws.numel(), s),
               "rt_layer_decode_step")
        torch.cuda.synchronize(self.device)
        _check(self.status(), "rt_layer_decode_step (device)")
        return zd.to(torch.float64).cpu().numpy()


class Stack:
    """n_layers RT layers with token embedding and tied head."""

    def __init__(self, n_layers: int, d_model: int, n_heads: int, d_ff: int, vocab: int, dtype: str = "bf16",
                 device: str = "cuda:0", **cfg_kw):
        torch = _torch()
        self.dtype, self.device = dtype, torch.device(device)
        self.n_layers, self.vocab = n_layers, vocab
        self.cfg = make_config(d_model, n_heads, d_ff, dtype=dtype, **cfg_kw)
        self._keep: list = []
        self.layers = (RtLayerWeights * n_layers)()
        self.emb = self.g_final = None
        self.k_caches: List = []
        self.v_caches: List = []
        self.ws = None
        self.N_max = 0

    def set_weights(self, layer_dicts: Sequence[dict], emb, g_final=None):
        assert len(layer_dicts) == self.n_layers
        for i, wd in enumerate(layer_dicts):
            st, keep = _pack_weights(wd, self.dtype, self.device)
            self.layers[i] = st
            self._keep += keep
        self.emb = _to_dev(emb, self.dtype, self.device)
        self.g_final = None if g_final is None else _to_dev(g_final, self.dtype, self.device)

    def reserve(self, B: int, N: int, N_max: Optional[int] = None):
        torch = _torch()
        N_max = N if N_max is None else N_max
        d = self.cfg.d_model
        if not self.k_caches or tuple(self.k_caches[0].shape) != (N_max, B, d):
            self.k_caches = [torch.zeros((N_max, B, d), dtype=_tdtype(self.dtype), device=self.device)
                             for _ in range(self.n_layers)]
            self.v_caches = [torch.zeros_like(t) for t in self.k_caches]
            self.N_max = N_max
            self._kp = (C.c_void_p * self.n_layers)(*[t.data_ptr() for t in self.k_caches])
            self._vp = (C.c_void_p * self.n_layers)(*[t.data_ptr() for t in self.v_caches])
        need = rt_workspace_bytes(self.cfg, B, N, self.n_layers)
        if self.ws is None or self.ws.numel() < need:
            self.ws = torch.zeros(need, dtype=torch.uint8, device=self.device)

    def prefill_device(self, ids_dev, hidden_dev, logits_dev, stream=None) -> None:
        torch = _torch()
        B, N = ids_dev.shape
        s = torch.cuda.current_stream(self.device).cuda_stream if stream is None else stream
        _check(rt_stack_prefill(self.cfg, self.n_layers, self.layers, self.emb.data_ptr(),
                                None if self.g_final is None else self.g_final.data_ptr(), self.vocab,
                                ids_dev.data_ptr(), B, N,
                                None if hidden_dev is None else hidden_dev.data_ptr(),
                                None if logits_dev is None else logits_dev.data_ptr(),
                                self._kp, self._vp, self.N_max, self.ws.data_ptr(), self.ws.numel(), s),
               "rt_stack_prefill")

    def status(self) -> int:
        return rt_get_status(self.ws.data_ptr())

    def prefill(self, ids, N_max: Optional[int] = None):
        """ids [B,N] int -> hidden [B,N,d], logits_last [B,V] (fp64 numpy)."""
        torch = _torch()
        idd = torch.as_tensor(np.asarray(ids), dtype=torch.int32, device=self.device).contiguous()
        B, N = idd.shape
        self.reserve(B, N, N_max)
        hid = torch.empty((B, N, self.cfg.d_model), dtype=_tdtype(self.dtype), device=self.device)
        logits = torch.empty((B, self.vocab), dtype=torch.float32, device=self.device)
        self.prefill_device(idd, hid, logits)
        torch.cuda.synchronize(self.device)
        _check(self.status(), "rt_stack_prefill (device)")
        return hid.to(torch.float64).cpu().numpy(), logits.to(torch.float64).cpu().numpy()

    def decode(self, ids_new, pos: int):
        torch = _torch()
        idd = torch.as_tensor(np.asarray(ids_new), dtype=torch.int32, device=self.device).contiguous()
        B = idd.shape[0]
        logits = torch.empty((B, self.vocab), dtype=torch.float32, device=self.device)
        need = rt_workspace_bytes(self.cfg, B, 1, self.n_layers)
        if self.ws is None or self.ws.numel() < need:
            self.ws = torch.zeros(need, dtype=torch.uint8, device=self.device)
        s = torch.cuda.current_stream(self.device).cuda_stream
        _check(rt_decode_step(self.cfg, self.n_layers, self.layers, self.emb.data_ptr(),
                              None if self.g_final is None else self.g_final.data_ptr(), self.vocab,
                              idd.data_ptr(), B, pos, logits.data_ptr(), self._kp, self._vp, self.N_max,
                              self.ws.data_ptr(), self.ws.numel(), s), "rt_decode_step")
        torch.cuda.synchronize(self.device)
        _check(self.status(), "rt_decode_step (device)")
        return logits.to(torch.float64).cpu().numpy()

    def caches_numpy(self, N: int):
        torch = _torch()
        f = lambda t: t[:N].permute(1, 0, 2).to(torch.float64).cpu().numpy()
        return [(f(k), f(v)) for k, v in zip(self.k_caches, self.v_caches)]


class PagedCache:
    """The pairs of one layer's sequences in pages, over tensors of the caller: k and v [n_pages, n_kv_heads, page_size, head_dim] (float32,
    bfloat16 or float8_e4m3fn, the last with exponents k_exp and v_exp, uint8 [n_pages, n_kv_heads, page_size]) and page_table, int32
    [n_seqs, max_pages].  Which pages a sequence owns is the caller's to say: it writes the page table,
    in place (the object keeps the tensors that it was made with).

    The methods take device tensors, enqueue on the current stream and return; nothing is kept between calls but the status word."""

    def __init__(self, k, v, page_table, k_exp=None, v_exp=None):
        torch = _torch()
        self.device, self.k, self.v, self.page_table, self.k_exp, self.v_exp = k.device, k, v, page_table, k_exp, v_exp
        code = {torch.float32: RT_F32, torch.bfloat16: RT_BF16, torch.float8_e4m3fn: RT_E4M3}.get(k.dtype)
        _require(k.is_cuda and code is not None and k.dim() == 4 and v.shape == k.shape and v.dtype == k.dtype and v.device == k.device and
                 k.is_contiguous() and v.is_contiguous(), "PagedCache: k, v")
        _require(page_table.dim() == 2 and page_table.dtype == torch.int32 and page_table.is_contiguous() and page_table.device == k.device,
                 "PagedCache: page_table")
        n_pages, n_kv, page, hd = k.shape
        _require((k_exp is not None) == (code == RT_E4M3) and (v_exp is not None) == (code == RT_E4M3), "PagedCache: exponents")
        self._status = torch.zeros(1, dtype=torch.int32, device=k.device)
        self._c = RtPagedCache(k.data_ptr(), v.data_ptr(), _vector(k_exp, n_pages * n_kv * page, torch.uint8, k.device.index, "PagedCache: k_exp"),
                               _vector(v_exp, n_pages * n_kv * page, torch.uint8, k.device.index, "PagedCache: v_exp"), page_table.data_ptr(),
                               self._status.data_ptr(), n_pages, page, n_kv, hd, code, page_table.shape[0], page_table.shape[1])
        self._index = k.device.index
        self._ref, self._scale = C.byref(self._c), 1.0 / math.sqrt(hd)
        self._B, self._kv, self._hd = page_table.shape[0], n_kv, hd
        self._codes = {torch.float32: RT_F32, torch.bfloat16: RT_BF16}
        self._ws_like: dict = {}                       # by number of query heads: one word seen as an array of the workspace's size
        _require(rt_paged_attention_workspace_bytes(self._c, n_kv) > 0, "PagedCache: shape")

    @classmethod
    def empty(cls, n_pages: int, page_size: int, n_kv_heads: int, n_seqs: int, max_pages: int, head_dim: int = 64, dtype: str = "bf16",
              device: str = "cuda:0"):
        """A cache with pages of its own; every entry of its page table is -1 (no page)."""
        torch = _torch()
        shape = (n_pages, n_kv_heads, page_size, head_dim)
        t = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}[dtype]
        pool = lambda: torch.zeros(shape, dtype=torch.uint8, device=device).view(t) if dtype == "e4m3" else torch.zeros(shape, dtype=t, device=device)
        exps = lambda: torch.full(shape[:3], 127, dtype=torch.uint8, device=device) if dtype == "e4m3" else None
        return cls(pool(), pool(), torch.full((n_seqs, max_pages), -1, dtype=torch.int32, device=device), exps(), exps())

    # (The methods below are called for every layer and token: checks and arguments are kept to the few microseconds that they need.)

    def write(self, k, v, seq, pos) -> None:
        """Row r of k and v ([rows, n_kv_heads, head_dim], float32 or bfloat16, rows at any stride) becomes position pos[r] of sequence
        seq[r] (int32); a negative position skips the row.  The rows of a call name different places."""
        torch, kv, hd, dev, n, t = _torch(), self._kv, self._hd, self._index, k.shape[0], k.dtype
        if _device_now() != dev:
            with torch.cuda.device(dev):
                return self.write(k, v, seq, pos)
        code = self._codes.get(t)
        _require(code is not None, "PagedCache.write: k")
        kp, ks = _rows(k, kv, hd, n, t, dev, "PagedCache.write: k")
        vp, vs = _rows(v, kv, hd, n, t, dev, "PagedCache.write: v")
        sp, pp = _vector(seq, n, torch.int32, dev, "PagedCache.write: seq"), _vector(pos, n, torch.int32, dev, "PagedCache.write: pos")
        status = _lib.rt_cache_write(self._ref, code, kp, vp, ks, vs, sp, pp, n, _stream_now(dev))
        if status:
            raise RtError(status, "rt_cache_write")

    def read(self, seq, pos, dtype: str = "bf16", k=None, v=None):
        """Rows (seq[r], pos[r]) as `dtype` ("f32", "bf16") -> k, v [rows, n_kv_heads, head_dim]; into k and v where they are given.
        Rows that are skipped stay as they are (in arrays made here: whatever the memory holds)."""
        torch, kv, hd, dev, n = _torch(), self._kv, self._hd, self._index, pos.shape[0]
        if _device_now() != dev:
            with torch.cuda.device(dev):
                return self.read(seq, pos, dtype, k, v)
        t = torch.bfloat16 if dtype == "bf16" else _tdtype(dtype)
        ks = vs = kv * hd
        if k is None:
            k = self.k.new_empty((n, kv, hd), dtype=t)
            kp = k.data_ptr()
        else:
            kp, ks = _rows(k, kv, hd, n, t, dev, "PagedCache.read: k")
        if v is None:
            v = self.k.new_empty((n, kv, hd), dtype=t)
            vp = v.data_ptr()
        else:
            vp, vs = _rows(v, kv, hd, n, t, dev, "PagedCache.read: v")
        sp, pp = _vector(seq, n, torch.int32, dev, "PagedCache.read: seq"), _vector(pos, n, torch.int32, dev, "PagedCache.read: pos")
        status = _lib.rt_cache_read(self._ref, self._codes[t], kp, vp, ks, vs, sp, pp, n, _stream_now(dev))
        if status:
            raise RtError(status, "rt_cache_read")
        return k, v

    def attend(self, q, lens, k_own=None, v_own=None, scale: Optional[float] = None, alibi_slopes=None, out=None, lse=None):
        """One new token of every sequence: q [n_seqs, n_heads, head_dim] attends to its sequence's first lens[b] cached pairs (int32) and,
        if given, to its own pair k_own, v_own [n_seqs, n_kv_heads, head_dim] -> out [n_seqs, n_heads, head_dim].  lse (float32
        [n_seqs, n_heads]) is filled if given; a sequence of negative length keeps its rows of out and lse (a new out:
        whatever the memory holds)."""
        torch, B, kv, hd, dev, t = _torch(), self._B, self._kv, self._hd, self._index, q.dtype
        if _device_now() != dev:
            with torch.cuda.device(dev):
                return self.attend(q, lens, k_own, v_own, scale, alibi_slopes, out, lse)
        code = self._codes.get(t)
        _require(code is not None and q.dim() == 3, "PagedCache.attend: q")
        H = q.shape[1]
        a = RtPagedQuery()
        a.q, a.q_stride = _rows(q, H, hd, B, t, dev, "PagedCache.attend: q")
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
            a.out, a.out_stride = out.data_ptr(), H * hd
        else:
            a.out, a.out_stride = _rows(out, H, hd, B, t, dev, "PagedCache.attend: out")
        if k_own is not None or v_own is not None:
            _require(k_own is not None and v_own is not None, "PagedCache.attend: k_own, v_own")
            a.k_own, a.k_own_stride = _rows(k_own, kv, hd, B, t, dev, "PagedCache.attend: k_own")
            a.v_own, a.v_own_stride = _rows(v_own, kv, hd, B, t, dev, "PagedCache.attend: v_own")
        a.lens = _vector(lens, B, torch.int32, dev, "PagedCache.attend: lens")
        if alibi_slopes is not None:
            a.alibi_slopes = _vector(alibi_slopes, H, torch.float32, dev, "PagedCache.attend: alibi_slopes")
        if lse is not None:
            a.lse = _vector(lse, B * H, torch.float32, dev, "PagedCache.attend: lse")
        a.dtype, a.n_heads, a.softmax_scale = code, H, self._scale if scale is None else scale
        like = self._ws_like.get(H)
        if like is None:
            need = rt_paged_attention_workspace_bytes(self._c, H)
            _require(need > 0, "PagedCache.attend: q")
            like = self._ws_like[H] = self._status.expand(need // 4)
        # a workspace of its own for every call: calls on two streams, or two captured graphs, may overlap
        ws = torch.empty_like(like, memory_format=torch.contiguous_format)
        status = _lib.rt_paged_attention(self._ref, C.byref(a), ws.data_ptr(), 4 * like.shape[0], _stream_now(dev))
        if status:
            raise RtError(status, "rt_paged_attention")
        return out

    def status(self) -> int:
        """RT_OK, or RT_ERR_INVALID_ARG once a call met a sequence, position or page number that does not exist (after a synchronise)."""
        with _torch().cuda.device(self.device):
            return rt_get_status(self._status.data_ptr())

    def clear_status(self) -> None:
        self._status.zero_()


class QkRotate:
    """qkRMS of queries and keys for each head and the rotation by the position, for one layer's shapes.  The angle of pair i at position
    p is p * freq[i], by default base^(-2 i / rot_dim).  The methods take device tensors and enqueue on the current stream."""

    def __init__(self, n_heads: int, n_kv_heads: int, dtype: str = "bf16", head_dim: int = 64, rot_dim: Optional[int] = None,
                 base: float = 10000.0, freq: Optional[Sequence[float]] = None, pairs: str = "halves", norm: bool = True,
                 rms_eps: float = 1e-6):
        self.dtype, self.n_heads, self.n_kv_heads, self.head_dim, self._t = dtype, n_heads, n_kv_heads, head_dim, _tdtype(dtype)
        rot_dim = head_dim if rot_dim is None else rot_dim
        freq = [base ** (-2.0 * i / rot_dim) for i in range(rot_dim // 2)] if freq is None else list(freq)
        _require(len(freq) == rot_dim // 2, "QkRotate: freq")
        self._freq = (C.c_double * max(len(freq), 1))(*freq)
        self.cfg = RtRotateConfig({"f32": RT_F32, "bf16": RT_BF16}[dtype], n_heads, n_kv_heads, head_dim, RT_NORM_QK if norm else 0, rms_eps,
                                  rot_dim, {"halves": RT_PAIRS_HALVES, "neighbours": RT_PAIRS_NEIGHBOURS}[pairs], self._freq)
        self._ref, self._need = C.byref(self.cfg), (-1, 0)      # (rows of the last backward call, bytes of its workspace)
        _require(rt_qk_rotate_backward_workspace_bytes(self.cfg, 1) > 0, "QkRotate: shape")

    def _inputs(self, q, k, pos, g_q, g_k):
        torch, H, kv, hd, n, t, dev = _torch(), self.n_heads, self.n_kv_heads, self.head_dim, q.shape[0], self._t, q.get_device()
        _require(dev >= 0 and (k is not None or kv == 0), "QkRotate: q, k")
        qp, qs = _rows(q, H, hd, n, t, dev, "QkRotate: q")
        kp, ks = _rows(k, kv, hd, n, t, dev, "QkRotate: k") if kv else (None, 0)
        gq = None if g_q is None else _vector(g_q, H * hd, t, dev, "QkRotate: g_q")
        gk = None if g_k is None or not kv else _vector(g_k, kv * hd, t, dev, "QkRotate: g_k")
        return n, t, dev, qp, qs, kp, ks, gq, gk, _vector(pos, n, torch.int32, dev, "QkRotate: pos")

    def forward(self, q, k, pos, g_q=None, g_k=None, q_out=None, k_out=None):
        """q [rows, n_heads, head_dim], k [rows, n_kv_heads, head_dim] at any row stride, pos [rows] int32 -> q_out, k_out (which may be q
        and k).  Rows of negative position stay as they are (in arrays made here: whatever the memory holds)."""
        torch, H, kv, hd = _torch(), self.n_heads, self.n_kv_heads, self.head_dim
        if q.is_cuda and _device_now() != q.get_device():
            with torch.cuda.device(q.get_device()):
                return self.forward(q, k, pos, g_q, g_k, q_out, k_out)
        n, t, dev, qp, qs, kp, ks, gq, gk, pp = self._inputs(q, k, pos, g_q, g_k)
        qos, ko, kos = H * hd, None, kv * hd
        if q_out is None:
            q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
            qo = q_out.data_ptr()
        else:
            qo, qos = _rows(q_out, H, hd, n, t, dev, "QkRotate.forward: q_out")
        if kv and k_out is None:
            k_out = torch.empty_like(k, memory_format=torch.contiguous_format)
            ko = k_out.data_ptr()
        elif kv:
            ko, kos = _rows(k_out, kv, hd, n, t, dev, "QkRotate.forward: k_out")
        status = _lib.rt_qk_rotate(self._ref, qp, kp, qs, ks, gq, gk, pp, n, qo, ko, qos, kos, _stream_now(dev))
        if status:
            raise RtError(status, "rt_qk_rotate")
        return q_out, k_out

    def backward(self, q, k, pos, dq_out, dk_out, g_q=None, g_k=None, dq=None, dk=None):
        """The inputs of forward and the gradients of its outputs (float32, contiguous) -> dq, dk, dg_q, dg_k (float32; dg is None where the
        gain is).  dq and dk may be given, dq_out and dk_out themselves among them; rows of negative position stay as they are."""
        torch, H, kv, hd = _torch(), self.n_heads, self.n_kv_heads, self.head_dim
        if q.is_cuda and _device_now() != q.get_device():
            with torch.cuda.device(q.get_device()):
                return self.backward(q, k, pos, dq_out, dk_out, g_q, g_k, dq, dk)
        f32 = torch.float32
        n, t, dev, qp, qs, kp, ks, gq, gk, pp = self._inputs(q, k, pos, g_q, g_k)
        dqo = _vector(dq_out, n * H * hd, f32, dev, "QkRotate.backward: dq_out")
        if dq is None:
            dq = torch.empty_like(dq_out)
            dqp = dq.data_ptr()
        else:
            dqp = _vector(dq, n * H * hd, f32, dev, "QkRotate.backward: dq")
        dko = dkp = dgk = None
        if kv:
            dko = _vector(dk_out, n * kv * hd, f32, dev, "QkRotate.backward: dk_out")
            if dk is None:
                dk = torch.empty_like(dk_out)
                dkp = dk.data_ptr()
            else:
                dkp = _vector(dk, n * kv * hd, f32, dev, "QkRotate.backward: dk")
            dgk = None if gk is None else torch.empty_like(g_k, dtype=f32)
        dgq = None if gq is None else torch.empty_like(g_q, dtype=f32)
        need = self._need
        if need[0] != n:
            need = self._need = (n, rt_qk_rotate_backward_workspace_bytes(self.cfg, n))
        ws = dq_out.new_empty(need[1] // 4)
        status = _lib.rt_qk_rotate_backward(self._ref, qp, kp, qs, ks, gq, gk, pp, n, dqo, dko, dqp, dkp, None if dgq is None else dgq.data_ptr(),
                                            None if dgk is None else dgk.data_ptr(), ws.data_ptr(), need[1], _stream_now(dev))
        if status:
            raise RtError(status, "rt_qk_rotate_backward")
        return dq, dk, dgq, dgk
