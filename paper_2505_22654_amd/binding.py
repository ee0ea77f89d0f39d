"""Thin ctypes binding of libvscan.so (include/vscan.h).

Argument marshalling only: every step of the reduction runs in the HIP kernels
behind the C ABI.  torch is used for device memory and the current stream.
There is no fallback: if the library is missing the first call raises.
"""
from __future__ import annotations

import array
import ctypes
import os
import sys
from typing import Dict, Optional

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libvscan.so")
_lib = None

VSCAN_F32, VSCAN_BF16 = 0, 1
VSCAN_SCORE_CLS_ROW, VSCAN_SCORE_MEAN_RECEIVED = 0, 1
VSCAN_KEYS_VISUAL_ONLY, VSCAN_KEYS_ALL = 0, 1
VSCAN_ROPE_SECTIONS, VSCAN_ROPE_CYCLED = 0, 1
VSCAN_ROPE_HALVES, VSCAN_ROPE_ADJACENT = 0, 1
ROPE_MAX_AXES = 4
(VSCAN_OK, VSCAN_ERR_NULL, VSCAN_ERR_SHAPE, VSCAN_ERR_BUDGET, VSCAN_ERR_DTYPE, VSCAN_ERR_ALIGN,
 VSCAN_ERR_WORKSPACE, VSCAN_ERR_HIP, VSCAN_ERR_VERSION, VSCAN_ERR_UNSUPPORTED) = (
    0, -1, -2, -3, -4, -5, -6, -7, -8, -9)

EXPORTS = ("vscan_encoder_workspace_size", "vscan_encoder_reduce", "vscan_llm_workspace_size",
           "vscan_llm_prune", "vscan_profile_enable", "vscan_profile_read", "vscan_status_string",
           "vscan_version", "vscan_budget", "vscan_budget_solve_r1", "vscan_flops",
           "vscan_llm_prune_ragged", "vscan_llm_fused_workspace_size", "vscan_llm_prune_fused",
           "vscan_encoder_fused_workspace_size", "vscan_encoder_reduce_fused",
           "vscan_llm_prune_fused_ragged", "vscan_llm_prune_static", "vscan_llm_ragged_workspace_size",
           "vscan_llm_prune_ragged_padded", "vscan_llm_prune_fused_ragged_padded", "vscan_rope",
           "vscan_cache_size", "vscan_cache_plan_workspace_size", "vscan_cache_plan", "vscan_cache_store",
           "vscan_cache_attend_workspace_size", "vscan_cache_attend")
STATIC_SCRATCH_BYTES = 16 << 20


class EncoderDesc(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32),
                ("batch", ctypes.c_int32), ("n_segments", ctypes.c_int32),
                ("grid_h", ctypes.c_int32), ("grid_w", ctypes.c_int32),
                ("has_cls", ctypes.c_int32), ("score_mode", ctypes.c_int32),
                ("softmax_domain", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("feat_dim", ctypes.c_int32),
                ("win_rows", ctypes.c_int32), ("win_cols", ctypes.c_int32),
                ("keep_global", ctypes.c_int32), ("keep_local", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class LlmDesc(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32),
                ("batch", ctypes.c_int32), ("seq_len", ctypes.c_int32),
                ("vis_start", ctypes.c_int32), ("vis_len", ctypes.c_int32),
                ("n_query", ctypes.c_int32), ("q_heads", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("hidden", ctypes.c_int32), ("keep", ctypes.c_int32),
                ("softmax_domain", ctypes.c_int32), ("in_place", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class RopeDesc(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32),
                ("batch", ctypes.c_int32), ("seq_len", ctypes.c_int32),
                ("q_heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("rot_dim", ctypes.c_int32),
                ("n_axes", ctypes.c_int32),
                *[(f"section{i}", ctypes.c_int32) for i in range(ROPE_MAX_AXES)],
                ("order", ctypes.c_int32), ("pairing", ctypes.c_int32),
                ("inverse", ctypes.c_int32),
                *[(f"{t}_stride{i}", ctypes.c_int64) for t in "qk" for i in range(3)]]


class CacheDesc(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32),
                ("batch", ctypes.c_int32), ("q_heads", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("block_size", ctypes.c_int32), ("n_blocks", ctypes.c_int32),
                ("max_blocks", ctypes.c_int32), ("n_new", ctypes.c_int32),
                ("seq_len", ctypes.c_int32), ("max_len", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class KernelTime(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 32), ("launches", ctypes.c_int32),
                ("total_ms", ctypes.c_float)]


class VscanError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


def lib():
    """Load libvscan.so; fails loudly when it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2505_22654_amd.build` (no CPU fallback exists)")
        # torch first: its wheel carries its own HIP runtime, found through the file name
        # libamdhip64.so, while this library asks for the soname libamdhip64.so.7.  Loaded in
        # that order the second request is satisfied by the runtime already in the process;
        # the other way round the process ends up with two runtimes (streams and device
        # pointers of one mean nothing to the other).
        import torch  # noqa: F401
        L = ctypes.CDLL(LIB_PATH)
        vp, i32p, f32p = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p
        L.vscan_encoder_workspace_size.argtypes = [ctypes.POINTER(EncoderDesc), ctypes.c_int,
                                                   ctypes.POINTER(ctypes.c_size_t)]
        L.vscan_encoder_workspace_size.restype = ctypes.c_int
        L.vscan_encoder_reduce.argtypes = [ctypes.POINTER(EncoderDesc), vp, vp, vp, vp, vp, i32p,
                                           vp, i32p, f32p, vp, ctypes.c_size_t, vp]
        L.vscan_encoder_reduce.restype = ctypes.c_int
        L.vscan_llm_workspace_size.argtypes = [ctypes.POINTER(LlmDesc),
                                               ctypes.POINTER(ctypes.c_size_t)]
        L.vscan_llm_workspace_size.restype = ctypes.c_int
        L.vscan_llm_prune.argtypes = [ctypes.POINTER(LlmDesc), vp, vp, vp, vp, i32p, vp, vp, vp,
                                      f32p, vp, ctypes.c_size_t, vp]
        L.vscan_llm_prune.restype = ctypes.c_int
        L.vscan_llm_prune_static.argtypes = [ctypes.POINTER(LlmDesc), vp, vp, vp, vp, i32p, vp, vp,
                                             vp, f32p, vp]
        L.vscan_llm_prune_static.restype = ctypes.c_int
        L.vscan_llm_prune_ragged.argtypes = [ctypes.POINTER(LlmDesc), vp, vp, vp, vp, vp, vp, i32p,
                                             vp, vp, vp, f32p, vp, ctypes.c_size_t, vp]
        L.vscan_llm_prune_ragged.restype = ctypes.c_int
        L.vscan_llm_fused_workspace_size.argtypes = [ctypes.POINTER(LlmDesc),
                                                     ctypes.POINTER(ctypes.c_size_t)]
        L.vscan_llm_fused_workspace_size.restype = ctypes.c_int
        L.vscan_llm_prune_fused.argtypes = [ctypes.POINTER(LlmDesc), vp, vp, vp, i32p, vp, f32p, vp,
                                            ctypes.c_size_t, vp]
        L.vscan_llm_prune_fused.restype = ctypes.c_int
        L.vscan_encoder_fused_workspace_size.argtypes = [ctypes.POINTER(EncoderDesc), ctypes.c_int,
                                                         ctypes.POINTER(ctypes.c_size_t)]
        L.vscan_encoder_fused_workspace_size.restype = ctypes.c_int
        L.vscan_encoder_reduce_fused.argtypes = [ctypes.POINTER(EncoderDesc), vp, vp, vp, vp, vp, vp,
                                                 vp, i32p, vp, i32p, f32p, vp, ctypes.c_size_t, vp]
        L.vscan_encoder_reduce_fused.restype = ctypes.c_int
        L.vscan_llm_prune_fused_ragged.argtypes = [ctypes.POINTER(LlmDesc), vp, vp, vp, vp, vp, i32p,
                                                   vp, f32p, vp, ctypes.c_size_t, vp]
        L.vscan_llm_prune_fused_ragged.restype = ctypes.c_int
        L.vscan_llm_ragged_workspace_size.argtypes = [ctypes.POINTER(LlmDesc), ctypes.c_int,
                                                      ctypes.POINTER(ctypes.c_size_t)]
        L.vscan_llm_ragged_workspace_size.restype = ctypes.c_int
        L.vscan_llm_prune_ragged_padded.argtypes = [ctypes.POINTER(LlmDesc), vp, vp, vp, vp, vp,
                                                    i32p, vp, vp, vp, f32p, vp, ctypes.c_size_t, vp]
        L.vscan_llm_prune_ragged_padded.restype = ctypes.c_int
        L.vscan_llm_prune_fused_ragged_padded.argtypes = [ctypes.POINTER(LlmDesc), vp, vp, vp, vp,
                                                          i32p, vp, f32p, vp, ctypes.c_size_t, vp]
        L.vscan_llm_prune_fused_ragged_padded.restype = ctypes.c_int
        L.vscan_rope.argtypes = [ctypes.POINTER(RopeDesc)] + [vp] * 7
        L.vscan_rope.restype = ctypes.c_int
        L.vscan_cache_size.argtypes = [ctypes.POINTER(CacheDesc)] + [ctypes.POINTER(ctypes.c_size_t)] * 2
        L.vscan_cache_size.restype = ctypes.c_int
        L.vscan_cache_plan_workspace_size.argtypes = [ctypes.POINTER(CacheDesc),
                                                      ctypes.POINTER(ctypes.c_size_t)]
        L.vscan_cache_plan_workspace_size.restype = ctypes.c_int
        L.vscan_cache_plan.argtypes = [ctypes.POINTER(CacheDesc), vp, vp, vp, ctypes.c_int32, vp, vp, vp,
                                       vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.vscan_cache_plan.restype = ctypes.c_int
        L.vscan_cache_store.argtypes = [ctypes.POINTER(CacheDesc)] + [vp] * 8
        L.vscan_cache_store.restype = ctypes.c_int
        L.vscan_cache_attend_workspace_size.argtypes = [ctypes.POINTER(CacheDesc),
                                                        ctypes.POINTER(ctypes.c_size_t)]
        L.vscan_cache_attend_workspace_size.restype = ctypes.c_int
        L.vscan_cache_attend.argtypes = [ctypes.POINTER(CacheDesc)] + [vp] * 10 + [ctypes.c_size_t, vp]
        L.vscan_cache_attend.restype = ctypes.c_int
        L.vscan_profile_enable.argtypes = [ctypes.c_int]
        L.vscan_profile_enable.restype = ctypes.c_int
        L.vscan_profile_read.argtypes = [ctypes.POINTER(KernelTime), ctypes.c_int,
                                         ctypes.POINTER(ctypes.c_int)]
        L.vscan_profile_read.restype = ctypes.c_int
        L.vscan_status_string.argtypes = [ctypes.c_int]
        L.vscan_status_string.restype = ctypes.c_char_p
        L.vscan_version.restype = ctypes.c_uint32
        dp, ip = ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int32)
        L.vscan_budget.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_double,
                                   ctypes.c_double, ip, ip, dp]
        L.vscan_budget.restype = ctypes.c_int
        L.vscan_budget_solve_r1.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_double,
                                            ctypes.c_double, dp]
        L.vscan_budget_solve_r1.restype = ctypes.c_int
        L.vscan_flops.argtypes = [ip, ctypes.c_int32, ctypes.c_int64, ctypes.c_int64, dp]
        L.vscan_flops.restype = ctypes.c_int
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().vscan_status_string(int(status)).decode()


def version() -> int:
    return int(lib().vscan_version())


def profile_enable(on: bool) -> None:
    """Switch per-kernel event timing inside the library on or off."""
    lib().vscan_profile_enable(int(on))


def profile_read() -> Dict[str, Dict[str, float]]:
    """{kernel name: {"launches": n, "total_ms": t}} since the last read."""
    buf = (KernelTime * 32)()
    n = ctypes.c_int(0)
    rc = lib().vscan_profile_read(buf, 32, ctypes.byref(n))
    if rc != VSCAN_OK:
        raise VscanError(rc, "vscan_profile_read")
    return {buf[i].name.decode(): {"launches": int(buf[i].launches),
                                   "total_ms": float(buf[i].total_ms)} for i in range(n.value)}


def budget(n_visual: int, n_layers: int, prune_layer: int, r1: float, r2: float):
    """(keep_encoder, keep_llm, average tokens over the LLM layers) for retention rates r1, r2."""
    n1, n2, avg = ctypes.c_int32(0), ctypes.c_int32(0), ctypes.c_double(0.0)
    rc = lib().vscan_budget(n_visual, n_layers, prune_layer, r1, r2, ctypes.byref(n1),
                            ctypes.byref(n2), ctypes.byref(avg))
    if rc != VSCAN_OK:
        raise VscanError(rc, "vscan_budget")
    return int(n1.value), int(n2.value), float(avg.value)


def budget_solve_r1(n_layers: int, prune_layer: int, avg_rate: float, r2: float) -> float:
    """Stage-1 retention rate that gives the layer-averaged retention `avg_rate` at fixed r2."""
    r1 = ctypes.c_double(0.0)
    rc = lib().vscan_budget_solve_r1(n_layers, prune_layer, avg_rate, r2, ctypes.byref(r1))
    if rc != VSCAN_OK:
        raise VscanError(rc, "vscan_budget_solve_r1")
    return float(r1.value)


def flops(n_per_layer, d: int, m: int) -> float:
    """Eq. 6 for a per-layer list of visual token counts."""
    arr = (ctypes.c_int32 * max(len(n_per_layer), 1))(*[int(n) for n in n_per_layer])
    out = ctypes.c_double(0.0)
    rc = lib().vscan_flops(arr, len(n_per_layer), d, m, ctypes.byref(out))
    if rc != VSCAN_OK:
        raise VscanError(rc, "vscan_flops")
    return float(out.value)


def _ragged_setup(desc, meta, batch: int, from_hidden: bool, device):
    """The host table of a ragged call and a workspace whose first bytes become the device table."""
    import torch
    assert len(meta) == batch
    # rows of another length raise ValueError here, values outside 32 bits OverflowError (ctypes would
    # cut those down)
    host = array.array("i", [int(x) for a, b, c, d in meta for x in (a, b, c, d)])
    n = ctypes.c_size_t(0)
    rc = lib().vscan_llm_ragged_workspace_size(ctypes.byref(desc), int(from_hidden), ctypes.byref(n))
    if rc != VSCAN_OK:
        raise VscanError(rc, "vscan_llm_ragged_workspace_size")
    workspace = torch.empty(n.value, dtype=torch.uint8, device=device)
    table = workspace[:16 * batch].view(torch.int32).view(batch, 4)
    return host, workspace, table


def llm_prune_ragged(shape, meta, q, k, v, hidden, want_scores: bool = False) -> Dict[str, object]:
    """vscan_llm_prune_ragged_padded.  `shape` carries the shared fields and the capacities
    (seq_len, vis_len, keep); `meta` is a list of (seq_len, vis_start, vis_len, keep) per sequence.
    Out-of-place results are tensors shaped like the inputs (rows past a sequence's result are
    zero); `out_len` lists the result lengths."""
    import torch
    desc = llm_desc(shape)
    dev = q.device
    host, workspace, table = _ragged_setup(desc, meta, shape.batch, False, dev)
    out = {"kept_idx": torch.empty((shape.batch, shape.keep), dtype=torch.int32, device=dev)}
    if want_scores:
        out["scores"] = torch.empty((shape.batch, shape.vis_len), dtype=torch.float32, device=dev)
    if shape.in_place:
        ko = vo = ho = None
    else:
        ko, vo, ho = torch.empty_like(k), torch.empty_like(v), torch.empty_like(hidden)
    rc = lib().vscan_llm_prune_ragged_padded(ctypes.byref(desc), host.buffer_info()[0], _ptr(q),
                                             _ptr(k), _ptr(v), _ptr(hidden), _ptr(out["kept_idx"]),
                                             _ptr(ko), _ptr(vo), _ptr(ho), _ptr(out.get("scores")),
                                             _ptr(workspace), workspace.numel(), _stream_handle())
    if rc != VSCAN_OK:
        raise VscanError(rc, "vscan_llm_prune_ragged_padded")
    out["k"], out["v"], out["hidden"] = (k, v, hidden) if shape.in_place else (ko, vo, ho)
    out["out_len"] = [m[0] - m[2] + m[3] for m in meta]
    out["meta_device"], out["workspace"] = table, workspace  # alive until the work has run
    return out


def _dtype_code(dtype: str) -> int:
    return {"f32": VSCAN_F32, "bf16": VSCAN_BF16}[dtype]


def encoder_desc(shape) -> EncoderDesc:
    """Descriptor from an `EncoderShape`-like object."""
    return EncoderDesc(ctypes.sizeof(EncoderDesc), _dtype_code(shape.dtype), shape.batch,
                       shape.n_segments, shape.grid_h, shape.grid_w, shape.has_cls,
                       shape.score_mode, shape.softmax_domain, shape.heads, shape.head_dim,
                       shape.feat_dim, shape.win_rows, shape.win_cols, shape.keep_global,
                       shape.keep_local, shape.scale)


def llm_desc(shape) -> LlmDesc:
    """Descriptor from an `LlmShape`-like object."""
    return LlmDesc(ctypes.sizeof(LlmDesc), _dtype_code(shape.dtype), shape.batch, shape.seq_len,
                   shape.vis_start, shape.vis_len, shape.n_query, shape.q_heads, shape.kv_heads,
                   shape.head_dim, shape.hidden, shape.keep, shape.softmax_domain, shape.in_place,
                   shape.scale)


def encoder_workspace_size(desc: EncoderDesc, with_local_pair: bool = False) -> int:
    n = ctypes.c_size_t(0)
    rc = lib().vscan_encoder_workspace_size(ctypes.byref(desc), int(with_local_pair),
                                            ctypes.byref(n))
    if rc != VSCAN_OK:
        raise VscanError(rc, "vscan_encoder_workspace_size")
    return int(n.value)


def llm_workspace_size(desc: LlmDesc) -> int:
    n = ctypes.c_size_t(0)
    rc = lib().vscan_llm_workspace_size(ctypes.byref(desc), ctypes.byref(n))
    if rc != VSCAN_OK:
        raise VscanError(rc, "vscan_llm_workspace_size")
    return int(n.value)


def llm_fused_workspace_size(desc: LlmDesc) -> int:
    n = ctypes.c_size_t(0)
    rc = lib().vscan_llm_fused_workspace_size(ctypes.byref(desc), ctypes.byref(n))
    if rc != VSCAN_OK:
        raise VscanError(rc, "vscan_llm_fused_workspace_size")
    return int(n.value)


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream_handle():
    import torch
    return torch.cuda.current_stream().cuda_stream


def _torch_dtype(dtype: str):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]


def encoder_reduce(shape, q, k, x, q_local=None, k_local=None, want_assign: bool = False,
                   want_scores: bool = False, workspace=None, out=None) -> Dict[str, object]:
    """vscan_encoder_reduce on CUDA tensors q, k [B,C,H,S,dh], x [B,C*N,D].

    Returns kept_idx [B,K] int32 and merged [B,K,D] (plus assign / scores on request).
    `workspace` (uint8 tensor) and `out` (dict of preallocated outputs) avoid allocation."""
    import torch
    desc = encoder_desc(shape)
    need = encoder_workspace_size(desc, q_local is not None)
    dev = q.device
    for t in (q, k, x, q_local, k_local):
        assert t is None or (t.is_cuda and t.is_contiguous() and t.dtype == _torch_dtype(shape.dtype))
    B, K, T = shape.batch, shape.keep, shape.tokens_per_image
    assert tuple(q.shape) == (B, shape.n_segments, shape.heads, shape.rows, shape.head_dim)
    assert tuple(k.shape) == tuple(q.shape) and tuple(x.shape) == (B, T, shape.feat_dim)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    out = dict(out) if out else {}
    if "kept_idx" not in out:
        out["kept_idx"] = torch.empty((B, K), dtype=torch.int32, device=dev)
    if "merged" not in out:
        out["merged"] = torch.empty((B, K, shape.feat_dim), dtype=x.dtype, device=dev)
    if want_assign and "assign" not in out:
        out["assign"] = torch.empty((B, T), dtype=torch.int32, device=dev)
    if want_scores and "scores" not in out:
        out["scores"] = torch.empty((B, T), dtype=torch.float32, device=dev)
    rc = lib().vscan_encoder_reduce(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(q_local),
                                    _ptr(k_local), _ptr(x), _ptr(out["kept_idx"]),
                                    _ptr(out["merged"]), _ptr(out.get("assign")),
                                    _ptr(out.get("scores")), _ptr(workspace), workspace.numel(),
                                    _stream_handle())
    if rc != VSCAN_OK:
        raise VscanError(rc, "vscan_encoder_reduce")
    out["workspace"] = workspace
    return out


def llm_prune(shape, q, k, v, hidden, want_scores: bool = False, workspace=None,
              out=None, static_scratch: bool = False) -> Dict[str, object]:
    """vscan_llm_prune on CUDA tensors q [B,Hq,Tq,dh], k, v [B,Hkv,S,dh], hidden [B,S,Dh]
    (`static_scratch`: vscan_llm_prune_static, which takes no workspace).

    Out of place it returns k, v, hidden of length S_out; in place (shape.in_place) it
    mutates the inputs and returns views of their first S_out rows."""
    import torch
    desc = llm_desc(shape)
    need = llm_workspace_size(desc)
    dev = q.device
    for t in (q, k, v, hidden):
        assert t.is_cuda and t.is_contiguous() and t.dtype == _torch_dtype(shape.dtype)
    B, S, So = shape.batch, shape.seq_len, shape.seq_out
    assert tuple(q.shape) == (B, shape.q_heads, shape.n_query, shape.head_dim)
    assert tuple(k.shape) == (B, shape.kv_heads, S, shape.head_dim) and k.shape == v.shape
    assert tuple(hidden.shape) == (B, S, shape.hidden)
    if workspace is None and not static_scratch:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    out = dict(out) if out else {}
    if "kept_idx" not in out:
        out["kept_idx"] = torch.empty((B, shape.keep), dtype=torch.int32, device=dev)
    if want_scores and "scores" not in out:
        out["scores"] = torch.empty((B, shape.vis_len), dtype=torch.float32, device=dev)
    if shape.in_place:
        ko = vo = ho = None
    else:
        ko = out.get("k")
        vo = out.get("v")
        ho = out.get("hidden")
        if ko is None:
            ko = torch.empty((B, shape.kv_heads, So, shape.head_dim), dtype=k.dtype, device=dev)
        if vo is None:
            vo = torch.empty_like(ko)
        if ho is None:
            ho = torch.empty((B, So, shape.hidden), dtype=hidden.dtype, device=dev)
    if static_scratch:
        rc = lib().vscan_llm_prune_static(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v),
                                          _ptr(hidden), _ptr(out["kept_idx"]), _ptr(ko), _ptr(vo),
                                          _ptr(ho), _ptr(out.get("scores")), _stream_handle())
    else:
        rc = lib().vscan_llm_prune(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(hidden),
                                   _ptr(out["kept_idx"]), _ptr(ko), _ptr(vo), _ptr(ho),
                                   _ptr(out.get("scores")), _ptr(workspace), workspace.numel(),
                                   _stream_handle())
    if rc != VSCAN_OK:
        raise VscanError(rc, "vscan_llm_prune_static" if static_scratch else "vscan_llm_prune")
    if shape.in_place:
        out["k"], out["v"], out["hidden"] = k[:, :, :So], v[:, :, :So], hidden[:, :So]
    else:
        out["k"], out["v"], out["hidden"] = ko, vo, ho
    out["workspace"] = workspace
    return out


def llm_prune_fused(shape, hidden, w_q, w_k_t, want_scores: bool = False, workspace=None,
                    out=None) -> Dict[str, object]:
    """vscan_llm_prune_fused on CUDA bf16 tensors hidden [B,S,Dh], w_q [Hq*dh, Dh] (rows =
    output features), w_k_t [Dh, Hkv*dh] (rows = input features).  Returns kept_idx, optional
    scores and the compacted hidden states (a view of `hidden` when shape.in_place)."""
    import torch
    desc = llm_desc(shape)
    need = llm_fused_workspace_size(desc)
    dev = hidden.device
    for t in (hidden, w_q, w_k_t):
        assert t.is_cuda and t.is_contiguous() and t.dtype == _torch_dtype(shape.dtype)
    B, S, So = shape.batch, shape.seq_len, shape.seq_out
    assert tuple(hidden.shape) == (B, S, shape.hidden)
    assert tuple(w_q.shape) == (shape.q_heads * shape.head_dim, shape.hidden)
    assert tuple(w_k_t.shape) == (shape.hidden, shape.kv_heads * shape.head_dim)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    out = dict(out) if out else {}
    if "kept_idx" not in out:
        out["kept_idx"] = torch.empty((B, shape.keep), dtype=torch.int32, device=dev)
    if want_scores and "scores" not in out:
        out["scores"] = torch.empty((B, shape.vis_len), dtype=torch.float32, device=dev)
    ho = None
    if not shape.in_place:
        ho = out.get("hidden")
        if ho is None:
            ho = torch.empty((B, So, shape.hidden), dtype=hidden.dtype, device=dev)
    rc = lib().vscan_llm_prune_fused(ctypes.byref(desc), _ptr(hidden), _ptr(w_q), _ptr(w_k_t),
                                     _ptr(out["kept_idx"]), _ptr(ho), _ptr(out.get("scores")),
                                     _ptr(workspace), workspace.numel(), _stream_handle())
    if rc != VSCAN_OK:
        raise VscanError(rc, "vscan_llm_prune_fused")
    out["hidden"] = hidden[:, :So] if shape.in_place else ho
    out["workspace"] = workspace
    return out


def encoder_fused_workspace_size(desc: EncoderDesc, with_local_triple: bool = False) -> int:
    n = ctypes.c_size_t(0)
    rc = lib().vscan_encoder_fused_workspace_size(ctypes.byref(desc), int(with_local_triple),
                                                  ctypes.byref(n))
    if rc != VSCAN_OK:
        raise VscanError(rc, "vscan_encoder_fused_workspace_size")
    return int(n.value)


def encoder_reduce_fused(shape, hidden, w_q, w_k_t, x, local=None, want_assign: bool = False,
                         want_scores: bool = False, workspace=None, out=None) -> Dict[str, object]:
    """vscan_encoder_reduce_fused on CUDA bf16 tensors hidden [B,C,S,D] ([CLS] row first), w_q
    [H*dh, D], w_k_t [D, H*dh], x [B,C*N,D]; `local` is an optional (hidden, w_q, w_k_t) triple
    of the shallow layer."""
    import torch
    desc = encoder_desc(shape)
    need = encoder_fused_workspace_size(desc, local is not None)
    dev = hidden.device
    B, T, D = shape.batch, shape.tokens_per_image, shape.feat_dim
    hd = shape.heads * shape.head_dim
    triples = [(hidden, w_q, w_k_t)] + ([tuple(local)] if local is not None else [])
    for h, a, b in triples:
        for t in (h, a, b):
            assert t.is_cuda and t.is_contiguous() and t.dtype == _torch_dtype(shape.dtype)
        assert tuple(h.shape) == (B, shape.n_segments, shape.rows, D)
        assert tuple(a.shape) == (hd, D) and tuple(b.shape) == (D, hd)
    assert x.is_cuda and x.is_contiguous() and tuple(x.shape) == (B, T, D)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    out = dict(out) if out else {}
    if "kept_idx" not in out:
        out["kept_idx"] = torch.empty((B, shape.keep), dtype=torch.int32, device=dev)
    if "merged" not in out:
        out["merged"] = torch.empty((B, shape.keep, D), dtype=x.dtype, device=dev)
    if want_assign and "assign" not in out:
        out["assign"] = torch.empty((B, T), dtype=torch.int32, device=dev)
    if want_scores and "scores" not in out:
        out["scores"] = torch.empty((B, T), dtype=torch.float32, device=dev)
    loc = triples[1] if local is not None else (None, None, None)
    rc = lib().vscan_encoder_reduce_fused(ctypes.byref(desc), _ptr(hidden), _ptr(w_q), _ptr(w_k_t),
                                          _ptr(loc[0]), _ptr(loc[1]), _ptr(loc[2]), _ptr(x),
                                          _ptr(out["kept_idx"]), _ptr(out["merged"]),
                                          _ptr(out.get("assign")), _ptr(out.get("scores")),
                                          _ptr(workspace), workspace.numel(), _stream_handle())
    if rc != VSCAN_OK:
        raise VscanError(rc, "vscan_encoder_reduce_fused")
    out["workspace"] = workspace
    return out


def llm_prune_fused_ragged(shape, meta, hidden, w_q, w_k_t, want_scores: bool = False) -> Dict[str, object]:
    """vscan_llm_prune_fused_ragged_padded.  `shape` carries the shared fields and the capacities;
    `meta` lists (seq_len, vis_start, vis_len, keep) per sequence.  The out-of-place result is
    shaped like `hidden` (rows past a sequence's result are zero); `out_len` lists the result
    lengths."""
    import torch
    desc = llm_desc(shape)
    dev = hidden.device
    host, workspace, table = _ragged_setup(desc, meta, shape.batch, True, dev)
    out = {"kept_idx": torch.empty((shape.batch, shape.keep), dtype=torch.int32, device=dev)}
    if want_scores:
        out["scores"] = torch.empty((shape.batch, shape.vis_len), dtype=torch.float32, device=dev)
    ho = None if shape.in_place else torch.empty_like(hidden)
    rc = lib().vscan_llm_prune_fused_ragged_padded(ctypes.byref(desc), host.buffer_info()[0],
                                                   _ptr(hidden), _ptr(w_q), _ptr(w_k_t),
                                                   _ptr(out["kept_idx"]), _ptr(ho),
                                                   _ptr(out.get("scores")), _ptr(workspace),
                                                   workspace.numel(), _stream_handle())
    if rc != VSCAN_OK:
        raise VscanError(rc, "vscan_llm_prune_fused_ragged_padded")
    out["hidden"] = hidden if shape.in_place else ho
    out["out_len"] = [m[0] - m[2] + m[3] for m in meta]
    out["meta_device"], out["workspace"] = table, workspace  # alive until the work has run
    return out


# ---- around the pruned prefill: rotary positions and the paged 8-bit cache -----------------------
_ROPE_BYTES, _CACHE_BYTES = ctypes.sizeof(RopeDesc), ctypes.sizeof(CacheDesc)


def _check(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _check_tensor(name: str, t, dtype, shape, index: int) -> None:
    """`t` on CUDA device `index`, contiguous, of this dtype and shape."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name}: expected contiguous {dtype} {shape} on cuda:{index}, got {t.dtype} "
                         f"{tuple(t.shape)}, strides {tuple(t.stride())}, on {t.device}")


def _workspace(workspace, need: int, device):
    """The caller's workspace as it is, or a new one where one is needed."""
    torch = _torch()
    if workspace is None:
        return torch.empty(need, dtype=torch.uint8, device=device) if need else None
    _check(workspace.device == device and workspace.dtype == torch.uint8 and workspace.is_contiguous(),
           f"workspace: expected contiguous uint8 on {device}")
    return workspace


def _call(entry: str, index: int, *args) -> None:
    """Calls `entry` on the current stream of CUDA device `index`, with that device the current one.
    (The stream's handle is taken without the object that torch.cuda.current_stream makes around it:
    4 of the 19 us that a small call took.)"""
    fn, C = getattr(_lib or lib(), entry), _torch()._C
    if index == C._cuda_getDevice():  # (the tensors are there, so CUDA is initialised)
        rc = fn(*args, C._cuda_getCurrentRawStream(index))
    else:
        with _torch().cuda.device(index):
            rc = fn(*args, C._cuda_getCurrentRawStream(index))
    if rc != VSCAN_OK:
        raise VscanError(rc, entry)


def _torch(modules=sys.modules):
    """torch, which lib() imports first (an import statement in every small call costs 0.3 us)."""
    torch = modules.get("torch")
    if torch is None:
        import torch
    return torch


def _dtype_of(torch, dtype: str):
    return torch.bfloat16 if dtype == "bf16" else torch.float32 if dtype == "f32" else _torch_dtype(dtype)


def rope_desc(shape, q_stride=(0, 0, 0), k_stride=(0, 0, 0)) -> RopeDesc:
    """Descriptor from a `RopeShape`-like object."""
    n = len(shape.sections)
    _check(1 <= n <= ROPE_MAX_AXES, f"sections: 1 to {ROPE_MAX_AXES} axes, got {n}")
    return RopeDesc(_ROPE_BYTES, _dtype_code(shape.dtype), shape.batch, shape.seq_len,
                    shape.q_heads, shape.kv_heads, shape.head_dim, shape.rot_dim, n, *shape.sections,
                    *(0,) * (ROPE_MAX_AXES - n), shape.order, shape.pairing, shape.inverse, *q_stride, *k_stride)


def rope_frequencies(rot_dim: int, theta: float = 10000.0, device="cuda"):
    """Radians per position of the rot_dim/2 pairs, theta^(-2i/rot_dim), in 64 bits."""
    import torch
    i = torch.arange(rot_dim // 2, dtype=torch.float64, device=device)
    return torch.pow(torch.tensor(float(theta), dtype=torch.float64, device=device), -2.0 * i / rot_dim)


def rope(shape, positions, inv_freq, q=None, k=None, in_place: bool = False,
         out=None) -> Dict[str, object]:
    """vscan_rope on CUDA tensors q [B,Hq,S,dh], k [B,Hkv,S,dh] (None where the head count is 0), of any
    strides over sequences, heads and tokens (multiples of 16 bytes), positions [axes,B,S] int32 and
    inv_freq [rot_dim/2] float64.

    Returns q and k turned: new contiguous tensors, those of `out`, or (`in_place`) the inputs."""
    torch = _torch()
    dt, B, S = _dtype_of(torch, shape.dtype), shape.batch, shape.seq_len
    index, src, dst, strides = positions.get_device(), [None, None], [None, None], [(0, 0, 0), (0, 0, 0)]
    _check(positions.is_cuda, "positions: expected a CUDA tensor")
    _check_tensor("positions", positions, torch.int32, (len(shape.sections), B, S), index)
    _check_tensor("inv_freq", inv_freq, torch.float64, (shape.rot_dim // 2,), index)
    for i, (name, t, heads) in enumerate((("q", q, shape.q_heads), ("k", k, shape.kv_heads))):
        if heads == 0:
            _check(t is None, f"{name}: the shape has no heads for it")
            continue
        size = (B, heads, S, shape.head_dim)
        if t is None or t.dtype is not dt or t.shape != size or t.get_device() != index:
            raise ValueError(f"{name}: expected {dt} {size} on cuda:{index}")
        if not t.is_contiguous():
            *strides[i], entry = t.stride()
            if entry != 1 or not any(strides[i]):  # three zeros would mean a contiguous tensor
                raise ValueError(f"{name}: the entries of a row must be adjacent, and rows apart")
        src[i] = t
        if in_place:
            dst[i] = t
        else:
            dst[i] = out.get(name) if out else None
            if dst[i] is None:
                dst[i] = t.new_empty(size)
            else:
                _check_tensor(f"out[{name!r}]", dst[i], dt, size, index)
    desc = rope_desc(shape, *strides)
    outs = (None, None) if in_place else (_ptr(dst[0]), _ptr(dst[1]))
    _call("vscan_rope", index, ctypes.byref(desc), _ptr(src[0]), _ptr(src[1]), positions.data_ptr(),
          inv_freq.data_ptr(), *outs)
    return {n: t for n, t in zip("qk", dst) if t is not None}


def cache_desc(shape, seq_len: int = 0) -> CacheDesc:
    """Descriptor from a `CacheShape`-like object."""
    return CacheDesc(_CACHE_BYTES, _dtype_code(shape.dtype), shape.batch, shape.q_heads,
                     shape.kv_heads, shape.head_dim, shape.block_size, shape.n_blocks, shape.max_blocks,
                     shape.n_new, seq_len, shape.max_len, shape.scale)


def _cache_shapes(shape):
    """(name, dtype name, tensor shape) of the parts of a cache."""
    groups, dp = shape.block_size // 16, (shape.head_dim + 63) // 64 * 64
    at = (shape.n_blocks, shape.kv_heads)
    return (("k", "uint8", at + (groups, dp // 16, 16, 16)),
            ("v", "uint8", at + (groups, dp // 64, 4, 16, 4, 4)),
            ("k_scale", "float32", at), ("v_scale", "float32", at))


def cache_alloc(shape, device="cuda") -> Dict[str, object]:
    """Memory of a cache: k, v (uint8, e4m3 values in operand order) and k_scale, v_scale (fp32)."""
    import torch
    nc, ns = ctypes.c_size_t(0), ctypes.c_size_t(0)
    rc = lib().vscan_cache_size(ctypes.byref(cache_desc(shape)), ctypes.byref(nc), ctypes.byref(ns))
    if rc != VSCAN_OK:
        raise VscanError(rc, "vscan_cache_size")
    cache = {n: torch.empty(s, dtype=getattr(torch, d), device=device) for n, d, s in _cache_shapes(shape)}
    assert cache["k"].numel() == cache["v"].numel() == nc.value
    assert 4 * cache["k_scale"].numel() == 4 * cache["v_scale"].numel() == ns.value
    return cache


def _check_cache(shape, cache, index: int) -> None:
    torch = _torch()
    groups, dp = shape.block_size // 16, (shape.head_dim + 63) // 64 * 64
    n, h, u8, f32 = shape.n_blocks, shape.kv_heads, torch.uint8, torch.float32
    _check_tensor("k", cache["k"], u8, (n, h, groups, dp // 16, 16, 16), index)
    _check_tensor("v", cache["v"], u8, (n, h, groups, dp // 64, 4, 16, 4, 4), index)
    _check_tensor("k_scale", cache["k_scale"], f32, (n, h), index)
    _check_tensor("v_scale", cache["v_scale"], f32, (n, h), index)


def cache_plan_workspace_size(desc: CacheDesc) -> int:
    n = ctypes.c_size_t(0)
    rc = lib().vscan_cache_plan_workspace_size(ctypes.byref(desc), ctypes.byref(n))
    if rc != VSCAN_OK:
        raise VscanError(rc, "vscan_cache_plan_workspace_size")
    return int(n.value)


def cache_plan(shape, cached_len, new_len, free_blocks, free_head, block_table, workspace=None,
               out=None) -> Dict[str, object]:
    """vscan_cache_plan on int32 CUDA tensors cached_len, new_len [B], free_blocks [n_free], free_head
    [1] and block_table [B,max_blocks] (written in place).

    Returns slot_map [B,n_new], kv_len [B], free_head and missing [1], and block_table.  `out` may hold
    any of the results; its kv_len may be cached_len and its free_head the one passed."""
    torch = _torch()
    i32, dev, index, B = torch.int32, block_table.device, block_table.get_device(), shape.batch
    desc = cache_desc(shape)
    need = cache_plan_workspace_size(desc) if workspace is None else 0
    _check(block_table.is_cuda, "block_table: expected a CUDA tensor")
    _check_tensor("cached_len", cached_len, i32, (B,), index)
    _check_tensor("new_len", new_len, i32, (B,), index)
    _check_tensor("free_blocks", free_blocks, i32, (free_blocks.numel(),), index)
    _check_tensor("free_head", free_head, i32, (1,), index)
    _check_tensor("block_table", block_table, i32, (B, shape.max_blocks), index)
    out = dict(out) if out else {}
    new = dict(zip(("kv_len", "free_head", "missing"), block_table.new_empty(B + 2).split_with_sizes((B, 1, 1))))
    for name, size in (("slot_map", (B, shape.n_new)), ("kv_len", (B,)), ("free_head", (1,)), ("missing", (1,))):
        if name in out:
            _check_tensor(f"out[{name!r}]", out[name], i32, size, index)
        else:
            out[name] = new[name] if name in new else block_table.new_empty(size)
    workspace = _workspace(workspace, need, dev)
    _call("vscan_cache_plan", index, ctypes.byref(desc), cached_len.data_ptr(), new_len.data_ptr(),
          free_blocks.data_ptr(), free_blocks.numel(), free_head.data_ptr(), block_table.data_ptr(),
          out["slot_map"].data_ptr(), out["kv_len"].data_ptr(), out["free_head"].data_ptr(),
          out["missing"].data_ptr(), _ptr(workspace), 0 if workspace is None else workspace.numel())
    out["block_table"], out["workspace"] = block_table, workspace
    return out


def cache_store(shape, k, v, slot_map, cache) -> Dict[str, object]:
    """vscan_cache_store on CUDA tensors k, v [B,Hkv,n_new,dh], slot_map [B,n_new] int32 and a cache of
    `cache_alloc`, which is written in place and returned.  k and v may be the first n_new rows of longer
    slabs (what an in-place prune returns)."""
    torch = _torch()
    dt, dev, index = _dtype_of(torch, shape.dtype), slot_map.device, slot_map.get_device()
    T, dh = shape.n_new, shape.head_dim
    size, rows = (shape.batch, shape.kv_heads, T, dh), T
    _check(slot_map.is_cuda, "slot_map: expected a CUDA tensor")
    for name, t in (("k", k), ("v", v)):
        if t.dtype is not dt or t.shape != size or t.get_device() != index:
            raise ValueError(f"{name}: expected {dt} {size} on {dev}")
    if not (k.is_contiguous() and v.is_contiguous()):
        _check(k.stride() == v.stride() and k.stride(3) == 1 and k.stride(2) == dh and k.stride(1) % dh == 0
               and k.stride(1) >= T * dh
               and (shape.batch == 1 or k.stride(0) == shape.kv_heads * k.stride(1)),
               f"k, v: expected rows of equal slabs, got strides {k.stride()} and {v.stride()}")
        rows = k.stride(1) // dh
        _check(rows < 1 << 31, f"k, v: slabs of {rows} rows, which the descriptor does not hold")
    _check_tensor("slot_map", slot_map, torch.int32, (shape.batch, T), index)
    _check_cache(shape, cache, index)
    desc = cache_desc(shape, rows)
    _call("vscan_cache_store", index, ctypes.byref(desc), k.data_ptr(), v.data_ptr(), slot_map.data_ptr(),
          cache["k"].data_ptr(), cache["v"].data_ptr(), cache["k_scale"].data_ptr(), cache["v_scale"].data_ptr())
    return cache


def cache_attend_workspace_size(desc: CacheDesc) -> int:
    n = ctypes.c_size_t(0)
    rc = lib().vscan_cache_attend_workspace_size(ctypes.byref(desc), ctypes.byref(n))
    if rc != VSCAN_OK:
        raise VscanError(rc, "vscan_cache_attend_workspace_size")
    return int(n.value)


def cache_attend(shape, q, cache, block_table, kv_len, new_len=None, workspace=None,
                 out=None) -> Dict[str, object]:
    """vscan_cache_attend on CUDA tensors q [B,Hq,n_new,dh], a cache of `cache_alloc`, block_table
    [B,max_blocks], kv_len [B] and new_len [B] int32 (None: n_new everywhere).

    Returns out [B,Hq,n_new,dh] and the workspace; both may be passed in."""
    torch = _torch()
    i32, dt, dev, index, B = torch.int32, _dtype_of(torch, shape.dtype), q.device, q.get_device(), shape.batch
    desc = cache_desc(shape)
    size = (B, shape.q_heads, shape.n_new, shape.head_dim)
    _check(q.is_cuda, "q: expected a CUDA tensor")
    _check_tensor("q", q, dt, size, index)
    _check_tensor("block_table", block_table, i32, (B, shape.max_blocks), index)
    _check_tensor("kv_len", kv_len, i32, (B,), index)
    if new_len is not None:
        _check_tensor("new_len", new_len, i32, (B,), index)
    _check_cache(shape, cache, index)
    need = cache_attend_workspace_size(desc) if workspace is None else 0
    workspace = _workspace(workspace, need, dev)
    res = out.get("out") if out else None
    if res is None:
        res = q.new_empty(size)
    else:
        _check_tensor("out", res, dt, size, index)
    _call("vscan_cache_attend", index, ctypes.byref(desc), q.data_ptr(), cache["k"].data_ptr(), cache["v"].data_ptr(),
          cache["k_scale"].data_ptr(), cache["v_scale"].data_ptr(), block_table.data_ptr(), kv_len.data_ptr(),
          _ptr(new_len), res.data_ptr(), _ptr(workspace), 0 if workspace is None else workspace.numel())
    return {"out": res, "workspace": workspace}
