"""ctypes binding of libveda.so: argument marshalling only.

Every function below maps one-to-one onto the C entry point of the same name in
include/veda.h and does nothing but turn torch tensors into pointers, sizes and the current
HIP stream.  PyTorch provides device memory and streams; all arithmetic runs in the HIP
kernels.  There is no fallback: if the library is missing or a call fails, this raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import math
import operator
from pathlib import Path
from typing import Optional, Sequence, Tuple

import numpy as np
import torch

_PKG = Path(__file__).resolve().parent
LIB_PATH = _PKG / "libveda.so"

VEDA_OK, VEDA_ERR_INVALID_ARG, VEDA_ERR_UNSUPPORTED, VEDA_ERR_WORKSPACE, VEDA_ERR_HIP = range(5)
VEDA_F32, VEDA_BF16 = 0, 1
VEDA_ACT_IDENTITY, VEDA_ACT_RELU = 0, 1
VEDA_TOKEN_MAJOR, VEDA_CHANNEL_MAJOR = 0, 1
VEDA_OPT_EXACT_LOGIT_SCALE = 0
VEDA_OPT_ATTN_LIST_WALK = 1
VEDA_OPT_FP32_CHAIN_UNIT = 2
VEDA_OPT_FP32_PRODUCTS = 3
VEDA_PRODUCTS_FP32, VEDA_PRODUCTS_SPLIT = 1, 2
VEDA_CHAINS_MATRIX, VEDA_CHAINS_VECTOR = 1, 2
VEDA_ROPE_INTERLEAVED, VEDA_ROPE_HALVES = 0, 1
VEDA_ROPE_PLAIN, VEDA_ROPE_LINEAR, VEDA_ROPE_NTK, VEDA_ROPE_BY_PARTS = range(4)
VEDA_STEP_SERVED, VEDA_STEP_REFUSED, VEDA_STEP_NO_ROOM = range(3)

EXPORTS = (
    "veda_plan_create", "veda_plan_destroy", "veda_plan_set_option", "veda_plan_chain_unit", "veda_plan_tiles", "veda_plan_tile_offset",
    "veda_plan_score_offset", "veda_plan_total_tiles", "veda_plan_score_elems",
    "veda_plan_workspace_bytes", "veda_plan_workspace_layout", "veda_tile_layout", "veda_tile_score", "veda_tile_layout_stats",
    "veda_tile_layout_path",
    "veda_tile_score_stats", "veda_tile_score_closed_form", "veda_tile_select", "veda_plan_fused_workspace_bytes",
    "veda_tile_score_select", "veda_tile_score_select_stats", "veda_tile_score_select_stats_noalloc",
    "veda_sparse_attn_fwd", "veda_sparse_attn_fwd_q_tokens",
    "veda_sparse_attn_fwd_qk_tokens", "veda_tile_heatmap", "veda_tile_heatmap_rows",
    "veda_tile_heatmap_ws", "veda_plan_heatmap_workspace_bytes",
    "veda_tile_recall", "veda_output_sqerr",
    "veda_rope_create", "veda_rope_destroy", "veda_rope_frequencies", "veda_rope_apply",
    "veda_cache_append", "veda_cache_attn_workspace_bytes", "veda_cache_attn_fwd", "veda_cache_copy_pages",
    "veda_packed_append", "veda_packed_attn_workspace_bytes", "veda_packed_attn_fwd", "veda_packed_copy_pages",
    "veda_pages_create", "veda_pages_destroy", "veda_pages_table", "veda_pages_length", "veda_pages_free_count", "veda_pages_extend",
    "veda_pages_fork", "veda_pages_truncate", "veda_pages_evict", "veda_pages_compact", "veda_pages_step",
    "veda_status_string", "veda_last_error",
)


class VedaError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str = ""):
        self.status = status
        super().__init__(f"{where}: status {status}" + (f" ({detail})" if detail else ""))


class veda_problem(C.Structure):
    _fields_ = [("batch", C.c_int32), ("heads", C.c_int32), ("head_dim", C.c_int32),
                ("T", C.c_int32), ("H", C.c_int32), ("W", C.c_int32), ("tile_tokens", C.c_int32),
                ("tile_shape", C.POINTER(C.c_int32)), ("dtype", C.c_int)]


class veda_strides(C.Structure):
    _fields_ = [("b", C.c_int64), ("h", C.c_int64), ("n", C.c_int64)]


_NO_ROWS = veda_strides(0, 0, 0)


class veda_mlp(C.Structure):
    _fields_ = [("in_dim", C.c_int32), ("hidden", C.c_int32), ("out_dim", C.c_int32), ("act", C.c_int),
                ("w1", C.c_void_p), ("b1", C.c_void_p), ("w2", C.c_void_p), ("b2", C.c_void_p)]


class veda_workspace_layout(C.Structure):
    _fields_ = [("stats_q", C.c_int64), ("stats_k", C.c_int64), ("latent_q", C.c_int64), ("latent_k", C.c_int64)]


class veda_rope_config(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("axes", C.c_int32), ("axis_dim", C.c_int32 * 3), ("pairs", C.c_int), ("scaling", C.c_int),
                ("base", C.c_double), ("factor", C.c_double), ("trained_len", C.c_double), ("beta_fast", C.c_double),
                ("beta_slow", C.c_double), ("amplitude", C.c_double)]


class veda_cache(C.Structure):
    _fields_ = [("pages", C.c_int32), ("page_tokens", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int),
                ("page_stride", C.c_int64), ("k", C.c_void_p), ("v", C.c_void_p)]


class veda_packed_cache(C.Structure):
    _fields_ = veda_cache._fields_


class veda_device_pages(C.Structure):
    _fields_ = [("pages", C.c_int32), ("page_tokens", C.c_int32), ("max_seqs", C.c_int32), ("max_pages", C.c_int32),
                ("table", C.c_void_p), ("length", C.c_void_p), ("used", C.c_void_p)]


class veda_step(C.Structure):
    _fields_ = [("seqs", C.c_int32), ("rows", C.c_int32), ("max_new", C.c_int32), ("axes", C.c_int32), ("frame_h", C.c_int32),
                ("frame_w", C.c_int32), ("seq", C.c_void_p), ("keep", C.c_void_p), ("evict", C.c_void_p), ("grow", C.c_void_p)]


class veda_step_tables(C.Structure):
    _fields_ = [("table_stride", C.c_int64)] + [(n, C.c_void_p) for n in ("page_table", "kv_len", "q_start", "status", "positions", "row_seq", "slots")]


class veda_cache_batch(C.Structure):
    _fields_ = [("seqs", C.c_int32), ("rows", C.c_int32), ("max_new", C.c_int32), ("max_pages", C.c_int32), ("table_stride", C.c_int64),
                ("page_table", C.c_void_p), ("kv_len", C.c_void_p), ("q_start", C.c_void_p)]


class veda_visible(C.Structure):
    _fields_ = [("block", C.c_int32), ("window", C.c_int32), ("sinks", C.c_int32)]


_lib = None


def load():
    """Load libveda.so (built in-tree by paper_2605_30325_amd.build).  Raises if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not LIB_PATH.exists():
        raise FileNotFoundError(f"{LIB_PATH} is not built; run `python -m paper_2605_30325_amd.build`")
    L = C.CDLL(str(LIB_PATH))
    vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
    L.veda_plan_create.argtypes = [C.POINTER(veda_problem), C.POINTER(vp)]
    L.veda_plan_create.restype = C.c_int
    L.veda_plan_destroy.argtypes = [vp]
    L.veda_plan_destroy.restype = None
    L.veda_plan_set_option.argtypes = [vp, C.c_int, i32]
    L.veda_plan_set_option.restype = C.c_int
    L.veda_plan_chain_unit.argtypes = [vp]
    L.veda_plan_chain_unit.restype = i32
    L.veda_plan_tiles.argtypes = [vp, i32]
    L.veda_plan_tiles.restype = i32
    for name in ("veda_plan_tile_offset", "veda_plan_score_offset"):
        getattr(L, name).argtypes = [vp, i32]
        getattr(L, name).restype = i64
    for name in ("veda_plan_total_tiles", "veda_plan_score_elems"):
        getattr(L, name).argtypes = [vp]
        getattr(L, name).restype = i64
    L.veda_plan_workspace_bytes.argtypes = [vp, C.POINTER(veda_mlp), C.POINTER(veda_mlp)]
    L.veda_plan_workspace_bytes.restype = C.c_size_t
    L.veda_plan_workspace_layout.argtypes = [vp, C.POINTER(veda_mlp), C.POINTER(veda_mlp), C.POINTER(veda_workspace_layout)]
    L.veda_plan_workspace_layout.restype = C.c_int
    L.veda_tile_layout.argtypes = [vp, vp, veda_strides, C.c_int, vp, vp, vp, vp]
    L.veda_tile_layout.restype = C.c_int
    L.veda_tile_score.argtypes = [vp, vp, vp, vp, C.POINTER(veda_mlp), C.POINTER(veda_mlp), C.c_float,
                                  vp, vp, C.c_size_t, vp]
    L.veda_tile_score.restype = C.c_int
    L.veda_tile_layout_stats.argtypes = [vp, vp, veda_strides, vp, vp, vp, vp, vp]
    L.veda_tile_layout_stats.restype = C.c_int
    L.veda_tile_layout_path.argtypes = [vp, vp, veda_strides, vp, veda_strides, vp, veda_strides] + [vp] * 8
    L.veda_tile_layout_path.restype = C.c_int
    L.veda_tile_score_stats.argtypes = [vp, vp, vp, C.POINTER(veda_mlp), C.POINTER(veda_mlp), C.c_float, vp, vp,
                                        C.c_size_t, vp]
    L.veda_tile_score_stats.restype = C.c_int
    L.veda_tile_score_closed_form.argtypes = [vp, vp, vp, vp, C.c_float, vp, vp, C.c_size_t, vp]
    L.veda_tile_score_closed_form.restype = C.c_int
    L.veda_tile_select.argtypes = [vp, vp, C.POINTER(i32), vp, vp, vp]
    L.veda_tile_select.restype = C.c_int
    L.veda_plan_fused_workspace_bytes.argtypes = [vp, C.POINTER(veda_mlp), C.POINTER(veda_mlp)]
    L.veda_plan_fused_workspace_bytes.restype = C.c_size_t
    L.veda_tile_score_select.argtypes = [vp, vp, vp, vp, C.POINTER(veda_mlp), C.POINTER(veda_mlp), C.c_float,
                                         C.POINTER(i32), vp, vp, vp, C.c_size_t, vp]
    L.veda_tile_score_select.restype = C.c_int
    L.veda_tile_score_select_stats.argtypes = [vp, vp, vp, C.POINTER(veda_mlp), C.POINTER(veda_mlp), C.c_float,
                                               C.POINTER(i32), vp, vp, vp, C.c_size_t, vp]
    L.veda_tile_score_select_stats.restype = C.c_int
    L.veda_tile_score_select_stats_noalloc.argtypes = [vp, vp, vp, C.POINTER(veda_mlp), C.POINTER(veda_mlp), C.c_float,
                                                       C.POINTER(i32), vp, vp, vp]
    L.veda_tile_score_select_stats_noalloc.restype = C.c_int
    L.veda_sparse_attn_fwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, C.c_float, vp, veda_strides, vp, vp]
    L.veda_sparse_attn_fwd.restype = C.c_int
    L.veda_sparse_attn_fwd_q_tokens.argtypes = [vp, vp, veda_strides, vp, vp, vp, vp, vp, C.c_float, vp, veda_strides,
                                                vp, vp]
    L.veda_sparse_attn_fwd_q_tokens.restype = C.c_int
    L.veda_sparse_attn_fwd_qk_tokens.argtypes = [vp, vp, veda_strides, vp, veda_strides, vp, vp, vp, vp, C.c_float, vp,
                                                 veda_strides, vp, vp]
    L.veda_sparse_attn_fwd_qk_tokens.restype = C.c_int
    L.veda_tile_heatmap.argtypes = [vp, vp, vp, vp, C.c_float, vp, i64, vp, vp]
    L.veda_tile_heatmap.restype = C.c_int
    L.veda_tile_heatmap_rows.argtypes = [vp, vp, vp, vp, C.c_float, vp, i32, vp, vp]
    L.veda_tile_heatmap_rows.restype = C.c_int
    L.veda_plan_heatmap_workspace_bytes.argtypes = [vp, i64]
    L.veda_plan_heatmap_workspace_bytes.restype = C.c_size_t
    L.veda_tile_heatmap_ws.argtypes = [vp, vp, vp, vp, C.c_float, vp, i64, vp, vp, vp, C.c_size_t, vp]
    L.veda_tile_heatmap_ws.restype = C.c_int
    L.veda_tile_recall.argtypes = [vp, C.POINTER(i32), vp, vp, vp, vp, C.c_size_t, vp]
    L.veda_tile_recall.restype = C.c_int
    L.veda_output_sqerr.argtypes = [vp, vp, veda_strides, vp, veda_strides, vp, vp, C.c_size_t, vp]
    L.veda_output_sqerr.restype = C.c_int
    L.veda_rope_create.argtypes = [C.POINTER(veda_rope_config), C.POINTER(vp)]
    L.veda_rope_create.restype = C.c_int
    L.veda_rope_destroy.argtypes = [vp]
    L.veda_rope_destroy.restype = None
    L.veda_rope_frequencies.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_double)]
    L.veda_rope_frequencies.restype = C.c_int
    L.veda_rope_apply.argtypes = [vp, C.c_int, i32, i32, i32, vp, veda_strides, vp, i64, i32, vp, veda_strides, vp]
    L.veda_rope_apply.restype = C.c_int
    cache, batch = C.POINTER(veda_cache), C.POINTER(veda_cache_batch)
    L.veda_cache_append.argtypes = [cache, batch, vp, veda_strides, vp, veda_strides, i32, vp, veda_strides, vp, veda_strides, vp, vp, vp]
    L.veda_cache_append.restype = C.c_int
    L.veda_cache_attn_workspace_bytes.argtypes = [cache, batch, i32]
    L.veda_cache_attn_workspace_bytes.restype = C.c_size_t
    L.veda_cache_attn_fwd.argtypes = [cache, batch, i32, vp, veda_strides, C.c_float, veda_visible, vp, veda_strides, vp, vp, C.c_size_t, vp]
    L.veda_cache_attn_fwd.restype = C.c_int
    L.veda_cache_copy_pages.argtypes = [cache, vp, i64, vp]
    L.veda_cache_copy_pages.restype = C.c_int
    packed = C.POINTER(veda_packed_cache)
    L.veda_packed_append.argtypes = [packed, *L.veda_cache_append.argtypes[1:-1], vp, veda_strides, vp, veda_strides, vp]
    L.veda_packed_append.restype = C.c_int
    L.veda_packed_attn_workspace_bytes.argtypes = [packed, batch, i32]
    L.veda_packed_attn_workspace_bytes.restype = C.c_size_t
    L.veda_packed_attn_fwd.argtypes = [packed, *L.veda_cache_attn_fwd.argtypes[1:]]
    L.veda_packed_attn_fwd.restype = C.c_int
    L.veda_packed_copy_pages.argtypes = [packed, vp, i64, vp]
    L.veda_packed_copy_pages.restype = C.c_int
    L.veda_pages_step.argtypes = [C.POINTER(veda_device_pages), C.POINTER(veda_step), C.POINTER(veda_step_tables), vp]
    L.veda_pages_step.restype = C.c_int
    L.veda_pages_create.argtypes = [i32, i32, i32, i32, C.POINTER(vp)]
    L.veda_pages_create.restype = C.c_int
    L.veda_pages_destroy.argtypes = [vp]
    L.veda_pages_destroy.restype = None
    L.veda_pages_table.argtypes = [vp]
    L.veda_pages_table.restype = C.POINTER(i32)
    L.veda_pages_length.argtypes = [vp, i32]
    L.veda_pages_free_count.argtypes = [vp]
    for name in ("veda_pages_length", "veda_pages_free_count"):
        getattr(L, name).restype = i32
    L.veda_pages_extend.argtypes = [vp, i32, i32, vp, i32, C.POINTER(i32)]
    L.veda_pages_fork.argtypes = [vp, i32, i32]
    L.veda_pages_truncate.argtypes = [vp, i32, i32]
    L.veda_pages_evict.argtypes = [vp, i32, i32, i32]
    L.veda_pages_compact.argtypes = [vp, vp, i32, C.POINTER(i32)]
    for name in ("extend", "fork", "truncate", "evict", "compact"):
        getattr(L, "veda_pages_" + name).restype = C.c_int
    L.veda_status_string.argtypes = [C.c_int]
    L.veda_status_string.restype = C.c_char_p
    L.veda_last_error.argtypes = []
    L.veda_last_error.restype = C.c_char_p
    _lib = L
    return L


def _check(status: int, where: str):
    if status != VEDA_OK:
        L = load()
        detail = L.veda_status_string(status).decode()
        if status == VEDA_ERR_HIP:
            detail += ": " + L.veda_last_error().decode()
        raise VedaError(status, where, detail)


def _stream() -> int:
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())   # current_stream() makes an object first: 2 us of a call's 12


def _stream_of(dev: torch.device) -> int:
    return torch._C._cuda_getCurrentRawStream(dev.index)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _strides(t: torch.Tensor) -> veda_strides:
    assert t.dim() == 4 and t.stride(3) == 1, "expected [batch, heads, N, d] with unit channel stride"
    return veda_strides(t.stride(0), t.stride(1), t.stride(2))


def _dtype_code(dt: torch.dtype) -> int:
    if dt == torch.float32:
        return VEDA_F32
    if dt == torch.bfloat16:
        return VEDA_BF16
    raise TypeError(f"unsupported dtype {dt}")


class Mlp:
    """Device-resident projection weights as the veda_mlp struct expects them."""

    def __init__(self, w1, b1, w2=None, b2=None, relu: bool = True, device="cuda"):
        def dev(a):
            return None if a is None else torch.as_tensor(np.ascontiguousarray(a, np.float32)).to(device).contiguous()
        self.w1, self.b1, self.w2, self.b2 = dev(w1), dev(b1), dev(w2), dev(b2)
        self.in_dim = int(self.w1.shape[1])
        self.hidden = 0 if self.w2 is None else int(self.w1.shape[2])
        self.out_dim = int(self.w1.shape[2] if self.w2 is None else self.w2.shape[2])
        self.act = VEDA_ACT_RELU if relu else VEDA_ACT_IDENTITY

    def struct(self) -> veda_mlp:
        return veda_mlp(self.in_dim, self.hidden, self.out_dim, self.act,
                        _ptr(self.w1), _ptr(self.b1), _ptr(self.w2), _ptr(self.b2))


class Plan:
    """veda_plan handle plus the sizes callers need to allocate buffers."""

    def __init__(self, batch: int, heads: int, head_dim: int, grid: Sequence[int],
                 tile_shape: np.ndarray, dtype: torch.dtype, tile_tokens: int = 64):
        L = load()
        self._shape = np.ascontiguousarray(tile_shape, np.int32).reshape(-1)
        if self._shape.size != 3 * heads:
            raise VedaError(VEDA_ERR_INVALID_ARG, "Plan", "tile_shape must be [heads, 3]")
        prob = veda_problem(batch, heads, head_dim, int(grid[0]), int(grid[1]), int(grid[2]), tile_tokens,
                            self._shape.ctypes.data_as(C.POINTER(C.c_int32)), _dtype_code(dtype))
        h = C.c_void_p()
        self.handle = None
        _check(L.veda_plan_create(C.byref(prob), C.byref(h)), "veda_plan_create")
        self.handle = h
        self.batch, self.heads, self.head_dim, self.grid, self.dtype = batch, heads, head_dim, tuple(grid), dtype
        self.tile_tokens = int(tile_tokens)        # 64, or 128 (two 64-slot halves per tile)
        self.mask_words = self.tile_tokens // 64   # u64 words of valid_mask per tile
        self.tokens = int(grid[0]) * int(grid[1]) * int(grid[2])
        self.tiles = [int(L.veda_plan_tiles(h, i)) for i in range(heads)]
        self.tile_offset = [int(L.veda_plan_tile_offset(h, i)) for i in range(heads)]
        self.score_offset = [int(L.veda_plan_score_offset(h, i)) for i in range(heads)]
        self.total_tiles = int(L.veda_plan_total_tiles(h))
        self.score_elems = int(L.veda_plan_score_elems(h))

    def set_option(self, option: int, value: int):
        _check(load().veda_plan_set_option(self.handle, option, int(value)), "veda_plan_set_option")

    def chain_unit(self) -> int:
        """VEDA_CHAINS_MATRIX or VEDA_CHAINS_VECTOR: where the plan's next stage-2 call runs its fp32 chains."""
        return int(load().veda_plan_chain_unit(self.handle))

    def workspace_bytes(self, phi_q: Mlp, phi_k: Mlp) -> int:
        return int(load().veda_plan_workspace_bytes(self.handle, C.byref(phi_q.struct()), C.byref(phi_k.struct())))

    def workspace_layout(self, phi_q: Mlp, phi_k: Mlp) -> veda_workspace_layout:
        """Float offsets of the intermediates veda_tile_score leaves in its workspace."""
        lay = veda_workspace_layout()
        _check(load().veda_plan_workspace_layout(self.handle, C.byref(phi_q.struct()), C.byref(phi_k.struct()),
                                                 C.byref(lay)), "veda_plan_workspace_layout")
        return lay

    def close(self):
        if self.handle is not None:
            load().veda_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def veda_tile_layout(plan: Plan, x: torch.Tensor, order: int = VEDA_TOKEN_MAJOR,
                     x_tiled: Optional[torch.Tensor] = None, valid_mask: Optional[torch.Tensor] = None,
                     valid_cnt: Optional[torch.Tensor] = None, want_mask: bool = True):
    """Stage 1.  Returns (x_tiled [batch, total_tiles, tile_tokens*d], valid_mask i64-as-u64
    [total_tiles * tile_tokens/64], valid_cnt i32 [total_tiles])."""
    dev = x.device
    if x_tiled is None:
        x_tiled = torch.empty((plan.batch, plan.total_tiles, plan.tile_tokens * plan.head_dim), dtype=x.dtype,
                              device=dev)
    if want_mask and valid_mask is None:
        valid_mask = torch.empty(plan.total_tiles * plan.mask_words, dtype=torch.int64, device=dev)
    if want_mask and valid_cnt is None:
        valid_cnt = torch.empty(plan.total_tiles, dtype=torch.int32, device=dev)
    _check(load().veda_tile_layout(plan.handle, _ptr(x), _strides(x), order, _ptr(x_tiled), _ptr(valid_mask),
                                   _ptr(valid_cnt), _stream()), "veda_tile_layout")
    return x_tiled, valid_mask, valid_cnt


def veda_tile_score(plan: Plan, q_tiled, k_tiled, valid_mask, phi_q: Mlp, phi_k: Mlp, scale: float,
                    scores: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Stage 2.  Returns (scores fp32 [batch, score_elems], workspace)."""
    dev = q_tiled.device
    if scores is None:
        scores = torch.empty((plan.batch, plan.score_elems), dtype=torch.float32, device=dev)
    need = plan.workspace_bytes(phi_q, phi_k)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    sq, sk = phi_q.struct(), phi_k.struct()
    _check(load().veda_tile_score(plan.handle, _ptr(q_tiled), _ptr(k_tiled), _ptr(valid_mask), C.byref(sq),
                                  C.byref(sk), C.c_float(scale), _ptr(scores), _ptr(workspace),
                                  workspace.numel() * workspace.element_size(), _stream()), "veda_tile_score")
    return scores, workspace


def veda_tile_layout_stats(plan: Plan, x: torch.Tensor, x_tiled: Optional[torch.Tensor] = None,
                           valid_mask: Optional[torch.Tensor] = None, valid_cnt: Optional[torch.Tensor] = None,
                           stats: Optional[torch.Tensor] = None, want_mask: bool = True, want_tiles: bool = True):
    """Stage 1 (token-major) with the TripPool descriptors taken during the gather.
    Returns (x_tiled, valid_mask, valid_cnt, stats fp32 [batch, total_tiles, 3*d]).
    want_tiles=False: descriptors (and masks) only, x_tiled is returned as None."""
    dev = x.device
    if x_tiled is None and want_tiles:
        x_tiled = torch.empty((plan.batch, plan.total_tiles, plan.tile_tokens * plan.head_dim), dtype=x.dtype,
                              device=dev)
    if want_mask and valid_mask is None:
        valid_mask = torch.empty(plan.total_tiles * plan.mask_words, dtype=torch.int64, device=dev)
    if want_mask and valid_cnt is None:
        valid_cnt = torch.empty(plan.total_tiles, dtype=torch.int32, device=dev)
    if stats is None:
        stats = torch.empty((plan.batch, plan.total_tiles, 3 * plan.head_dim), dtype=torch.float32, device=dev)
    _check(load().veda_tile_layout_stats(plan.handle, _ptr(x), _strides(x), _ptr(x_tiled), _ptr(valid_mask),
                                         _ptr(valid_cnt), _ptr(stats), _stream()), "veda_tile_layout_stats")
    return x_tiled, valid_mask, valid_cnt, stats


def veda_tile_layout_path(plan: Plan, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, buffers: Optional[dict] = None,
                          want_tiles: bool = True) -> dict:
    """Stage 1 of a whole call in one launch: q and k as veda_tile_layout_stats takes them, v channel-major.  Returns
    {qt, kt, vt, vm, vc, zq, zk} (qt, kt None with want_tiles=False), from `buffers` where it has them."""
    b, dev = {} if buffers is None else buffers, q.device
    tiles = (plan.batch, plan.total_tiles, plan.tile_tokens * plan.head_dim)

    def take(name, shape, dtype):
        t = b.get(name)
        return torch.empty(shape, dtype=dtype, device=dev) if t is None else t

    r = {"qt": take("qt", tiles, q.dtype) if want_tiles else None, "kt": take("kt", tiles, k.dtype) if want_tiles else None,
         "vt": take("vt", tiles, v.dtype), "vm": take("vm", plan.total_tiles * plan.mask_words, torch.int64),
         "vc": take("vc", plan.total_tiles, torch.int32),
         "zq": take("zq", (plan.batch, plan.total_tiles, 3 * plan.head_dim), torch.float32),
         "zk": take("zk", (plan.batch, plan.total_tiles, 3 * plan.head_dim), torch.float32)}
    _check(load().veda_tile_layout_path(plan.handle, _ptr(q), _strides(q), _ptr(k), _strides(k), _ptr(v), _strides(v), _ptr(r["qt"]),
                                        _ptr(r["kt"]), _ptr(r["vt"]), _ptr(r["vm"]), _ptr(r["vc"]), _ptr(r["zq"]), _ptr(r["zk"]),
                                        _stream()), "veda_tile_layout_path")
    return r


def veda_tile_score_stats(plan: Plan, stats_q, stats_k, phi_q: Mlp, phi_k: Mlp, scale: float,
                          scores: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Stage 2 from descriptors.  Returns (scores fp32 [batch, score_elems], workspace holding the latents)."""
    dev = stats_q.device
    if scores is None:
        scores = torch.empty((plan.batch, plan.score_elems), dtype=torch.float32, device=dev)
    sq, sk = phi_q.struct(), phi_k.struct()
    if workspace is None:   # room for the hidden layers too: the faster route of the projections
        need = int(load().veda_plan_workspace_bytes(plan.handle, C.byref(sq), C.byref(sk)))
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    _check(load().veda_tile_score_stats(plan.handle, _ptr(stats_q), _ptr(stats_k), C.byref(sq), C.byref(sk),
                                        C.c_float(scale), _ptr(scores), _ptr(workspace),
                                        workspace.numel() * workspace.element_size(), _stream()),
           "veda_tile_score_stats")
    return scores, workspace


def veda_tile_score_closed_form(plan: Plan, q_tiled, k_tiled, valid_mask, lam: float,
                                scores: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Stage 2 with the weight-free scorer.  Returns (scores fp32 [batch, score_elems], workspace)."""
    dev = q_tiled.device
    if scores is None:
        scores = torch.empty((plan.batch, plan.score_elems), dtype=torch.float32, device=dev)
    if workspace is None:
        workspace = torch.empty(plan.batch * plan.total_tiles * 10 * plan.head_dim * 4, dtype=torch.uint8, device=dev)
    _check(load().veda_tile_score_closed_form(plan.handle, _ptr(q_tiled), _ptr(k_tiled), _ptr(valid_mask),
                                              C.c_float(lam), _ptr(scores), _ptr(workspace),
                                              workspace.numel() * workspace.element_size(), _stream()),
           "veda_tile_score_closed_form")
    return scores, workspace


def veda_tile_select(plan: Plan, scores, k_per_head: Sequence[int], row_ptr: Optional[torch.Tensor] = None,
                     col_idx: Optional[torch.Tensor] = None):
    """Stage 3.  Returns (row_ptr i32 [batch*total_tiles+1], col_idx i32 [batch*nnz])."""
    k = np.ascontiguousarray(k_per_head, np.int32)
    if k.size != plan.heads:
        raise VedaError(VEDA_ERR_INVALID_ARG, "veda_tile_select", "k_per_head must have one entry per head")
    nnz = int(sum(int(n) * int(kk) for n, kk in zip(plan.tiles, k)))
    dev = scores.device
    if row_ptr is None:
        row_ptr = torch.empty(plan.batch * plan.total_tiles + 1, dtype=torch.int32, device=dev)
    if col_idx is None:
        col_idx = torch.empty(max(1, plan.batch * max(nnz, 0)), dtype=torch.int32, device=dev)
    _check(load().veda_tile_select(plan.handle, _ptr(scores), k.ctypes.data_as(C.POINTER(C.c_int32)),
                                   _ptr(row_ptr), _ptr(col_idx), _stream()), "veda_tile_select")
    return row_ptr, col_idx


def veda_tile_score_select(plan: Plan, phi_q: Mlp, phi_k: Mlp, scale: float, k_per_head: Sequence[int],
                           q_tiled=None, k_tiled=None, valid_mask=None, stats_q=None, stats_k=None,
                           row_ptr: Optional[torch.Tensor] = None, col_idx: Optional[torch.Tensor] = None,
                           workspace: Optional[torch.Tensor] = None):
    """Stages 2 + 3 in one call, from the tiled Q, K (q_tiled, k_tiled, valid_mask) or from their
    descriptors (stats_q, stats_k).  Returns (row_ptr, col_idx, workspace)."""
    k = np.ascontiguousarray(k_per_head, np.int32)
    if k.size != plan.heads:
        raise VedaError(VEDA_ERR_INVALID_ARG, "veda_tile_score_select", "k_per_head must have one entry per head")
    from_stats = stats_q is not None
    dev = (stats_q if from_stats else q_tiled).device
    nnz = int(sum(int(n) * int(kk) for n, kk in zip(plan.tiles, k)))
    if row_ptr is None:
        row_ptr = torch.empty(plan.batch * plan.total_tiles + 1, dtype=torch.int32, device=dev)
    if col_idx is None:
        col_idx = torch.empty(max(1, plan.batch * max(nnz, 0)), dtype=torch.int32, device=dev)
    sq, sk = phi_q.struct(), phi_k.struct()
    if workspace is None:
        need = int(load().veda_plan_fused_workspace_bytes(plan.handle, C.byref(sq), C.byref(sk)))
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    kp = k.ctypes.data_as(C.POINTER(C.c_int32))
    nbytes = workspace.numel() * workspace.element_size()
    if from_stats:
        _check(load().veda_tile_score_select_stats(plan.handle, _ptr(stats_q), _ptr(stats_k), C.byref(sq), C.byref(sk),
                                                   C.c_float(scale), kp, _ptr(row_ptr), _ptr(col_idx), _ptr(workspace),
                                                   nbytes, _stream()), "veda_tile_score_select_stats")
    else:
        _check(load().veda_tile_score_select(plan.handle, _ptr(q_tiled), _ptr(k_tiled), _ptr(valid_mask), C.byref(sq),
                                             C.byref(sk), C.c_float(scale), kp, _ptr(row_ptr), _ptr(col_idx),
                                             _ptr(workspace), nbytes, _stream()), "veda_tile_score_select")
    return row_ptr, col_idx, workspace


NOALLOC_SCRATCH_BYTES = 128 << 20


def veda_tile_score_select_stats_noalloc(plan: Plan, phi_q: Mlp, phi_k: Mlp, scale: float, k_per_head: Sequence[int],
                                         stats_q: torch.Tensor, stats_k: torch.Tensor, row_ptr: torch.Tensor,
                                         col_idx: torch.Tensor):
    """Stages 2 + 3 from descriptors with the library's fixed scratch array: the caller passes every
    input and output, nothing is allocated here or in the library."""
    k = np.ascontiguousarray(k_per_head, np.int32)
    if k.size != plan.heads:
        raise VedaError(VEDA_ERR_INVALID_ARG, "veda_tile_score_select_stats_noalloc",
                        "k_per_head must have one entry per head")
    sq, sk = phi_q.struct(), phi_k.struct()
    status = load().veda_tile_score_select_stats_noalloc(
        plan.handle, _ptr(stats_q), _ptr(stats_k), C.byref(sq), C.byref(sk), C.c_float(scale),
        k.ctypes.data_as(C.POINTER(C.c_int32)), _ptr(row_ptr), _ptr(col_idx), _stream())
    if status == VEDA_ERR_WORKSPACE:
        raise VedaError(status, "veda_tile_score_select_stats_noalloc", load().veda_last_error().decode())
    _check(status, "veda_tile_score_select_stats_noalloc")
    return row_ptr, col_idx


def veda_sparse_attn_fwd(plan: Plan, q_tiled, k_tiled, v_tiled, valid_mask, row_ptr, col_idx,
                         softmax_scale: float, out: Optional[torch.Tensor] = None,
                         lse: Optional[torch.Tensor] = None, want_lse: bool = False,
                         q_tokens: Optional[torch.Tensor] = None, k_tokens: Optional[torch.Tensor] = None):
    """Stage 4.  Returns (out [batch, heads, N, d] in token order, lse or None).
    q_tokens (with q_tiled None): Q in token order [batch, heads, N, d], gathered by the kernel;
    k_tokens (with q_tokens, k_tiled None): K in token order as well."""
    dev = v_tiled.device
    if out is None:
        out = torch.empty((plan.batch, plan.heads, plan.tokens, plan.head_dim), dtype=plan.dtype, device=dev)
    if want_lse and lse is None:
        lse = torch.empty((plan.batch, plan.heads, plan.tokens), dtype=torch.float32, device=dev)
    if q_tokens is not None and k_tokens is not None and q_tiled is None and k_tiled is None:
        _check(load().veda_sparse_attn_fwd_qk_tokens(plan.handle, _ptr(q_tokens), _strides(q_tokens), _ptr(k_tokens),
                                                     _strides(k_tokens), _ptr(v_tiled), _ptr(valid_mask),
                                                     _ptr(row_ptr), _ptr(col_idx), C.c_float(softmax_scale), _ptr(out),
                                                     _strides(out), _ptr(lse), _stream()),
               "veda_sparse_attn_fwd_qk_tokens")
        return out, lse
    if q_tokens is not None and q_tiled is None:
        _check(load().veda_sparse_attn_fwd_q_tokens(plan.handle, _ptr(q_tokens), _strides(q_tokens), _ptr(k_tiled),
                                                    _ptr(v_tiled), _ptr(valid_mask), _ptr(row_ptr), _ptr(col_idx),
                                                    C.c_float(softmax_scale), _ptr(out), _strides(out), _ptr(lse),
                                                    _stream()), "veda_sparse_attn_fwd_q_tokens")
        return out, lse
    _check(load().veda_sparse_attn_fwd(plan.handle, _ptr(q_tiled), _ptr(k_tiled), _ptr(v_tiled),
                                       _ptr(valid_mask), _ptr(row_ptr), _ptr(col_idx), C.c_float(softmax_scale),
                                       _ptr(out), _strides(out), _ptr(lse), _stream()), "veda_sparse_attn_fwd")
    return out, lse


def veda_tile_heatmap(plan: Plan, q_tiled, k_tiled, valid_mask, softmax_scale: float,
                      query_tiles: Optional[torch.Tensor] = None, heat: Optional[torch.Tensor] = None):
    """Target tile scores of full attention: heat fp32 [batch, score_elems] (rows of unlisted query
    tiles are left as they were)."""
    dev = q_tiled.device
    if heat is None:
        heat = torch.zeros((plan.batch, plan.score_elems), dtype=torch.float32, device=dev)
    n_qt = 0 if query_tiles is None else int(query_tiles.numel())
    _heatmap_ws(plan, q_tiled, k_tiled, valid_mask, softmax_scale, query_tiles, n_qt, None, heat, "veda_tile_heatmap")
    return heat


HEATMAP_SCRATCH_BYTES = 2 << 30   # what veda_plan_heatmap_workspace_bytes asks for up to about 8000 tiles a head


def _heatmap_ws(plan, q_tiled, k_tiled, valid_mask, softmax_scale, query_tiles, n_qt, row_sums, heat, what):
    """One walk over the keys, with scratch from torch's allocator (taken on every call: no state that calls on other
    streams or threads could share); two walks without scratch, the same bits in about 1.6 times the time, where that
    would be more than HEATMAP_SCRATCH_BYTES or there is no memory left for it."""
    args = (plan.handle, _ptr(q_tiled), _ptr(k_tiled), _ptr(valid_mask), C.c_float(softmax_scale))
    need = int(load().veda_plan_heatmap_workspace_bytes(plan.handle, n_qt))
    ws = None
    if need <= HEATMAP_SCRATCH_BYTES:
        try:
            ws = torch.empty(need, dtype=torch.uint8, device=q_tiled.device)
        except torch.cuda.OutOfMemoryError:
            pass
    if ws is not None:
        status = load().veda_tile_heatmap_ws(*args, _ptr(query_tiles), n_qt, _ptr(row_sums), _ptr(heat), _ptr(ws), need, _stream())
    elif row_sums is None:
        status = load().veda_tile_heatmap(*args, _ptr(query_tiles), n_qt, _ptr(heat), _stream())
    else:
        status = load().veda_tile_heatmap_rows(*args, _ptr(row_sums), 0, _ptr(heat), _stream())
    _check(status, what)


def veda_tile_heatmap_rows(plan: Plan, q_tiled, k_tiled, valid_mask, softmax_scale: float, row_sums: Optional[torch.Tensor] = None,
                           heat: Optional[torch.Tensor] = None):
    """veda_tile_heatmap of all query tiles with the rows' softmax sums: given (as an earlier call on the same
    Q, K and scale returned them, under whatever tiling), only the second pass over the keys runs.  Sums of another
    tiling are the same up to fp32 rounding, not bit for bit.
    Returns (heat, row_sums fp32 [batch, heads, tokens, 2])."""
    dev = q_tiled.device
    if heat is None:
        heat = torch.empty((plan.batch, plan.score_elems), dtype=torch.float32, device=dev)
    have = row_sums is not None
    shape = (plan.batch, plan.heads, plan.tokens, 2)
    if not have:
        row_sums = torch.empty(shape, dtype=torch.float32, device=dev)
    elif tuple(row_sums.shape) != shape or row_sums.dtype != torch.float32 or row_sums.device != dev or not row_sums.is_contiguous():
        # the kernel reads one pair per row: a buffer of another problem would be read past its end
        raise VedaError(VEDA_ERR_INVALID_ARG, "veda_tile_heatmap_rows",
                        f"row_sums must be contiguous fp32 {list(shape)} on {dev}, as an earlier call returned them")
    if not have:
        _heatmap_ws(plan, q_tiled, k_tiled, valid_mask, softmax_scale, None, 0, row_sums, heat, "veda_tile_heatmap_rows")
        return heat, row_sums
    _check(load().veda_tile_heatmap_rows(plan.handle, _ptr(q_tiled), _ptr(k_tiled), _ptr(valid_mask), C.c_float(softmax_scale),
                                         _ptr(row_sums), 1, _ptr(heat), _stream()), "veda_tile_heatmap_rows")
    return heat, row_sums


def veda_tile_recall(plan: Plan, k_per_head: Sequence[int], col_idx_a, col_idx_b,
                     recall: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Recall@k of selection a against selection b: fp32 [batch, heads]."""
    k = np.ascontiguousarray(k_per_head, np.int32)
    if k.size != plan.heads:
        raise VedaError(VEDA_ERR_INVALID_ARG, "veda_tile_recall", "k_per_head must have one entry per head")
    dev = col_idx_a.device
    if recall is None:
        recall = torch.empty((plan.batch, plan.heads), dtype=torch.float32, device=dev)
    if workspace is None:
        workspace = torch.empty(plan.batch * plan.heads, dtype=torch.int64, device=dev)
    _check(load().veda_tile_recall(plan.handle, k.ctypes.data_as(C.POINTER(C.c_int32)), _ptr(col_idx_a), _ptr(col_idx_b),
                                   _ptr(recall), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                   _stream()), "veda_tile_recall")
    return recall


def veda_output_sqerr(plan: Plan, a: torch.Tensor, b: torch.Tensor, err: Optional[torch.Tensor] = None,
                      workspace: Optional[torch.Tensor] = None):
    """Squared Frobenius distance of two [batch, heads, N, d] tensors per (batch, head): fp64 [batch, heads]."""
    dev = a.device
    if err is None:
        err = torch.empty((plan.batch, plan.heads), dtype=torch.float64, device=dev)
    if workspace is None:
        workspace = torch.empty(plan.batch * plan.heads * 64, dtype=torch.float64, device=dev)
    _check(load().veda_output_sqerr(plan.handle, _ptr(a), _strides(a), _ptr(b), _strides(b), _ptr(err),
                                    _ptr(workspace), workspace.numel() * workspace.element_size(), _stream()),
           "veda_output_sqerr")
    return err


def veda_attention(plan: Plan, q, k, v, phi_q: Mlp, phi_k: Mlp, k_per_head, score_scale: float,
                   softmax_scale: float, buffers: Optional[dict] = None, fused: bool = False,
                   one_call: bool = False, from_tokens: bool = False):
    """The whole path in call order: layout x3 -> score -> select -> sparse attention.
    fused=True takes the descriptors during the Q and K gathers (veda_tile_layout_stats +
    veda_tile_score_stats); one_call=True runs stages 2 and 3 through veda_tile_score_select*,
    which never writes the score matrix; from_tokens=True (with fused, bf16) writes no
    tiled copy of Q and K: the gathers only take descriptors and masks, and the attention kernel
    gathers the rows of both from token order.  The results are bit-identical whichever way.
    `buffers` (optional dict) is filled on the first call and reused afterwards so that a
    steady-state step allocates nothing."""
    bufs = {} if buffers is None else buffers
    if from_tokens and not fused:
        raise ValueError("from_tokens needs fused=True (the descriptors must come from the gathers)")
    if fused:
        r = veda_tile_layout_path(plan, q, k, v, bufs, want_tiles=not from_tokens)
        qt, kt, vt, vm, vc, zq, zk = (r[x] for x in ("qt", "kt", "vt", "vm", "vc", "zq", "zk"))
        bufs.update(zq=zq, zk=zk)
    else:
        qt, vm, vc = veda_tile_layout(plan, q, VEDA_TOKEN_MAJOR, bufs.get("qt"), bufs.get("vm"), bufs.get("vc"))
        kt, _, _ = veda_tile_layout(plan, k, VEDA_TOKEN_MAJOR, bufs.get("kt"), want_mask=False)
        vt, _, _ = veda_tile_layout(plan, v, VEDA_CHANNEL_MAJOR, bufs.get("vt"), want_mask=False)
    if one_call:
        s = None
        if fused:
            rp, ci, ws = veda_tile_score_select(plan, phi_q, phi_k, score_scale, k_per_head, stats_q=zq, stats_k=zk,
                                                row_ptr=bufs.get("rp"), col_idx=bufs.get("ci"), workspace=bufs.get("ws"))
        else:
            rp, ci, ws = veda_tile_score_select(plan, phi_q, phi_k, score_scale, k_per_head, q_tiled=qt, k_tiled=kt,
                                                valid_mask=vm, row_ptr=bufs.get("rp"), col_idx=bufs.get("ci"),
                                                workspace=bufs.get("ws"))
    else:
        if fused:
            s, ws = veda_tile_score_stats(plan, zq, zk, phi_q, phi_k, score_scale, bufs.get("s"), bufs.get("ws"))
        else:
            s, ws = veda_tile_score(plan, qt, kt, vm, phi_q, phi_k, score_scale, bufs.get("s"), bufs.get("ws"))
        rp, ci = veda_tile_select(plan, s, k_per_head, bufs.get("rp"), bufs.get("ci"))
    out, _ = veda_sparse_attn_fwd(plan, qt, kt, vt, vm, rp, ci, softmax_scale, bufs.get("out"),
                                  q_tokens=q if from_tokens else None, k_tokens=k if from_tokens else None)
    bufs.update(qt=qt, kt=kt, vt=vt, vm=vm, vc=vc, s=s, ws=ws, rp=rp, ci=ci, out=out)
    return out, bufs


# ---- streaming generation: rotary positions, a paged cache and the attention over it -------------------------------------
# As everywhere in this binding no graph is formed (generation needs no gradients), with the exception of veda_rope_apply, whose gradient
# the library has.

class Rope:
    """veda_rope handle: the frequencies of one rotary scheme, on the current device.
    axis_dim: channels of every axis (one number or up to three), the first sum(axis_dim) channels of a row rotate."""

    def __init__(self, head_dim: int, axis_dim, base: float = 10000.0, pairs: int = VEDA_ROPE_INTERLEAVED, scaling: int = VEDA_ROPE_PLAIN,
                 factor: float = 1.0, trained_len: float = 0.0, beta_fast: float = 32.0, beta_slow: float = 1.0, amplitude: float = 0.0):
        dims = [int(axis_dim)] if isinstance(axis_dim, int) else [int(x) for x in axis_dim]
        self.handle = None
        if not 1 <= len(dims) <= 3:
            raise VedaError(VEDA_ERR_INVALID_ARG, "Rope", "axis_dim must name 1 to 3 axes")
        _ints("Rope", head_dim, *dims, pairs, scaling)
        cfg = veda_rope_config(head_dim, len(dims), (C.c_int32 * 3)(*dims), pairs, scaling, base, factor, trained_len, beta_fast, beta_slow,
                               amplitude)
        h = C.c_void_p()
        _check(load().veda_rope_create(C.byref(cfg), C.byref(h)), "veda_rope_create")
        self.handle = h
        self.head_dim, self.axes, self.rot_dim = int(head_dim), len(dims), sum(dims)
        self.device = torch.device("cuda", torch.cuda.current_device())

    def frequencies(self):
        """(radians per position of every pair, float64 [rot_dim / 2]; the amplitude)"""
        f, a = np.empty(self.rot_dim // 2, np.float64), C.c_double()
        _check(load().veda_rope_frequencies(self.handle, f.ctypes.data_as(C.POINTER(C.c_double)), C.byref(a)), "veda_rope_frequencies")
        return f, a.value

    def close(self):
        if self.handle is not None:
            load().veda_rope_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _refuse(where: str, what: str):
    raise VedaError(VEDA_ERR_INVALID_ARG, where, what)


def _need(ok: bool, where: str, what: str):
    if not ok:
        _refuse(where, what)


def _ints(where: str, *values: int):
    """ctypes cuts numbers off at 32 bits without a word."""
    for x in values:
        if not -(1 << 31) <= x < 1 << 31:
            _refuse(where, f"{x} does not fit 32 bits")


def _on(dev: torch.device, where: str):
    """The kernels run on the current device, so that is where the tensors have to be."""
    if dev.type != "cuda" or dev.index != torch._C._cuda_getDevice():
        _refuse(where, f"tensors on {dev}, which is not the current device")


def veda_rope_apply(rope: Rope, x: torch.Tensor, positions: torch.Tensor, y: Optional[torch.Tensor] = None, transpose: bool = False):
    """Rotates x [batch, heads, N, d] by positions i32 [batch or 1, N, axes] (or [N], one axis) into y (x itself: in place).
    transpose=True turns the gradient of the result into the gradient of x.  Where x requires a gradient the result carries one (and its
    backward pass makes that call); a y that is given is then refused, as no graph leads through it."""
    w, dev = "veda_rope_apply", x.device
    if (x.requires_grad or (y is not None and y.requires_grad)) and torch.is_grad_enabled():
        _need(y is None, w, "y is given and a gradient is required: leave y out, or call under torch.no_grad()")
        return _Turn.apply(x, rope, positions, transpose)
    if rope.handle is None:
        _refuse(w, "the rope is closed")
    if x.dim() != 4 or x.shape[3] != rope.head_dim or (x.stride(3) != 1 and x.numel()):
        _refuse(w, "x must be [batch, heads, N, head_dim] with unit channel stride")
    _on(dev, w)
    b, h, n, _ = x.shape
    if rope.axes == 1 and positions.dim() == 1:
        positions = positions.reshape(1, -1, 1)
    if (positions.dim() != 3 or positions.shape[0] not in (1, b) or positions.shape[1] != n or positions.shape[2] != rope.axes or
            positions.dtype != torch.int32 or positions.device != dev or not positions.is_contiguous()):
        _refuse(w, f"positions must be contiguous i32 [{b} or 1, {n}, {rope.axes}] on {dev}")
    if y is None:
        y = torch.empty_like(x)
        if y.stride(3) != 1:
            y = torch.empty(x.shape, dtype=x.dtype, device=dev)
    elif y.shape != x.shape or y.dtype != x.dtype or y.device != dev or (y.stride(3) != 1 and y.numel()):
        _refuse(w, "y must be as x, with unit channel stride")
    sx, sy = x.stride(), y.stride()
    _check(load().veda_rope_apply(rope.handle, _dtype_code(x.dtype), b, h, n, x.data_ptr(), veda_strides(sx[0], sx[1], sx[2]),
                                  positions.data_ptr(), 0 if positions.shape[0] == 1 else n * rope.axes, int(transpose), y.data_ptr(),
                                  veda_strides(sy[0], sy[1], sy[2]), _stream_of(dev)), w)
    return y


class _Turn(torch.autograd.Function):
    """The rotation is linear, so its gradient is the transposed rotation of the result's; and the other way round."""

    @staticmethod
    def forward(ctx, x, rope, positions, transpose):
        ctx.rope, ctx.transpose = rope, transpose
        ctx.save_for_backward(positions)
        return veda_rope_apply(rope, x, positions, transpose=transpose)

    @staticmethod
    def backward(ctx, g):
        es = g.element_size()
        if g.stride(3) != 1 or g.data_ptr() % 16 or any(n > 1 and s * es % 16 for n, s in zip(g.shape[:3], g.stride())):
            g = g.clone(memory_format=torch.contiguous_format)     # a sum's gradient has no strides at all
        return veda_rope_apply(ctx.rope, g, ctx.saved_tensors[0], transpose=not ctx.transpose), None, None, None


class Cache:
    """One layer's paged cache: pools k, v [pages, kv_heads, page_tokens, d], made here unless given (views with a larger page
    stride are fine)."""

    def __init__(self, pages: int, page_tokens: int, kv_heads: int, head_dim: int, dtype: torch.dtype, device="cuda",
                 k: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None):
        shape = (pages, kv_heads, page_tokens, head_dim)
        if k is None and v is None:
            k, v = (torch.empty(shape, dtype=dtype, device=device) for _ in range(2))
        inner = (page_tokens * head_dim, head_dim, 1)
        for t in (k, v):
            _need(t is not None and tuple(t.shape) == shape and t.dtype == dtype and t.device == k.device and
                  all(a == b or n == 1 for n, a, b in zip(shape[1:], t.stride()[1:], inner)) and
                  (pages == 1 or t.stride(0) == k.stride(0) >= kv_heads * page_tokens * head_dim),
                  "Cache", f"k and v must be {dtype} {list(shape)} with close rows, heads and tokens, and pages apart")
        self.k, self.v = k, v
        self.pages, self.page_tokens, self.kv_heads, self.head_dim, self.dtype = int(pages), int(page_tokens), int(kv_heads), int(head_dim), dtype
        stride = k.stride(0) if pages > 1 else 0
        self.device = k.device
        self._struct = veda_cache(self.pages, self.page_tokens, self.kv_heads, self.head_dim, _dtype_code(dtype), stride, _ptr(k), _ptr(v))
        self._ref = C.byref(self._struct)


class PackedCache:
    """One layer's paged cache in 4 bits: pools k, v u8 [pages, kv_heads, page_tokens * (d / 2 + d / 32)], made here unless given (views
    with a larger page stride are fine).  dtype: of the rows that go in, of queries and of results."""

    def __init__(self, pages: int, page_tokens: int, kv_heads: int, head_dim: int, dtype: torch.dtype, device="cuda",
                 k: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None):
        _ints("PackedCache", pages, page_tokens, kv_heads, head_dim)
        run = page_tokens * (head_dim // 2 + head_dim // 32)
        shape = (pages, kv_heads, run)
        if k is None and v is None:
            k, v = (torch.zeros(shape, dtype=torch.uint8, device=device) for _ in range(2))
        for t in (k, v):
            _need(t is not None and tuple(t.shape) == shape and t.dtype == torch.uint8 and t.device == k.device and
                  all(a == b or n == 1 for n, a, b in zip(shape[1:], t.stride()[1:], (run, 1))) and
                  (pages == 1 or t.stride(0) == k.stride(0) >= kv_heads * run),
                  "PackedCache", f"k and v must be uint8 {list(shape)} with close bytes and heads, and pages apart")
        self.k, self.v = k, v
        self.pages, self.page_tokens, self.kv_heads, self.head_dim, self.dtype = int(pages), int(page_tokens), int(kv_heads), int(head_dim), dtype
        stride = k.stride(0) if pages > 1 else 0
        self.device = k.device
        self._struct = veda_packed_cache(self.pages, self.page_tokens, self.kv_heads, self.head_dim, _dtype_code(dtype), stride, _ptr(k), _ptr(v))
        self._ref = C.byref(self._struct)

    def codes(self, pool: torch.Tensor) -> torch.Tensor:
        """The codes of k or v, a view u8 [pages, kv_heads, page_tokens, d / 2]: channel 2i in the low, 2i + 1 in the high half of a byte."""
        return pool[:, :, :self.page_tokens * (self.head_dim // 2)].unflatten(2, (self.page_tokens, self.head_dim // 2))

    def scales(self, pool: torch.Tensor) -> torch.Tensor:
        """The bytes s of k or v, a view u8 [pages, kv_heads, page_tokens, d / 32]: 32 channels are their codes times 2^(s - 127)."""
        return pool[:, :, self.page_tokens * (self.head_dim // 2):].unflatten(2, (self.page_tokens, self.head_dim // 32))


class CacheBatch:
    """The sequences of a call: page_table i32 [seqs, max_pages], kv_len i32 [seqs], q_start i32 [seqs + 1] on the GPU (read when the
    kernels run), max_new: the most new tokens of any sequence."""

    def __init__(self, page_table: torch.Tensor, kv_len: torch.Tensor, q_start: torch.Tensor, max_new: int):
        seqs = page_table.shape[0]
        _need(page_table.dim() == 2 and page_table.dtype == torch.int32 and (page_table.stride(1) == 1 or page_table.shape[1] == 1) and
              (seqs < 2 or page_table.stride(0) >= page_table.shape[1]), "CacheBatch", "page_table must be i32 [seqs, max_pages], a row for each sequence")
        _ints("CacheBatch", max_new)
        for t, n in ((kv_len, seqs), (q_start, seqs + 1)):
            _need(tuple(t.shape) == (n,) and t.dtype == torch.int32 and t.is_contiguous() and t.device == page_table.device, "CacheBatch",
                  "kv_len and q_start must be contiguous i32 [seqs] and [seqs + 1] where the page table is")
        self.page_table, self.kv_len, self.q_start, self.max_new, self.seqs = page_table, kv_len, q_start, int(max_new), int(seqs)

    def struct(self, rows: int) -> veda_cache_batch:
        t = self.page_table
        width, stride = t.shape[1], t.stride(0)
        return veda_cache_batch(self.seqs, rows, self.max_new, width, stride if stride > width else width, t.data_ptr(), self.kv_len.data_ptr(),
                                self.q_start.data_ptr())


@functools.lru_cache(maxsize=1024)
def _row_strides(h: int, n: int) -> veda_strides:
    """Passed by value and never written; making one is a quarter of a microsecond of a call's ten."""
    return veda_strides(0, h, n)


@functools.lru_cache(maxsize=1024)
def _visible(block: int, window: int, sinks: int) -> veda_visible:
    """For ints alone: 7.0 equals 7, and a tensor stays itself when its number changes."""
    return veda_visible(block, window, sinks)


def _rows(cache: Cache, t: torch.Tensor, rows: int, where: str, name: str, heads: Optional[int] = None) -> veda_strides:
    shape, stride = t.shape, t.stride()
    if (len(shape) != 3 or shape[0] != rows or shape[2] != cache.head_dim or t.dtype != cache.dtype or t.device != cache.device or
            (stride[2] != 1 and t.numel())):
        _refuse(where, f"{name} must be {cache.dtype} [{rows}, heads, {cache.head_dim}] beside the cache")
    if heads is not None and shape[1] != heads:
        _refuse(where, f"{name} must have {heads} heads")
    return _row_strides(stride[1], stride[0])


def veda_cache_append(cache: Cache, batch: CacheBatch, k: torch.Tensor, v: torch.Tensor, rope: Optional[Rope] = None,
                      positions: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None):
    """Writes the new rows' k (rotated) and v [rows, kv_heads, d] into the cache; with q [rows, q_heads, d], returns q rotated (q_out).
    positions i32 [rows, axes]; without them the position in the sequence (ropes of one axis)."""
    w, rows = "veda_cache_append", k.shape[0]
    _on(cache.device, w)
    if rope is not None and rope.handle is None:    # which the library would take for no rope
        _refuse(w, "the rope is closed")
    sk, sv = _rows(cache, k, rows, w, "k"), _rows(cache, v, rows, w, "v")
    if k.shape[1] != cache.kv_heads or v.shape[1] != cache.kv_heads:
        _refuse(w, "k and v must have the cache's heads")
    if batch.page_table.device != cache.device:
        _refuse(w, "the batch must be where the cache is")
    if q is not None:
        if q_out is None:
            q_out = torch.empty((rows, q.shape[1], cache.head_dim), dtype=cache.dtype, device=cache.device)
        sq, so = _rows(cache, q, rows, w, "q"), _rows(cache, q_out, rows, w, "q_out")
        if q.shape[1] != q_out.shape[1]:
            _refuse(w, "q and q_out must have the same heads")
    else:
        sq = so = veda_strides(0, 0, 0)
        _need(q_out is None, w, "q_out without q")
    if positions is not None and (rope is None or tuple(positions.shape) != (rows, rope.axes) or positions.dtype != torch.int32 or
                                  positions.device != cache.device or not positions.is_contiguous()):
        _refuse(w, "positions must be contiguous i32 [rows, axes of rope]")
    bs = batch.struct(rows)
    _check(load().veda_cache_append(cache._ref, C.byref(bs), k.data_ptr(), sk, v.data_ptr(), sv, 0 if q is None else q.shape[1], _ptr(q), sq,
                                    _ptr(q_out), so, None if rope is None else rope.handle, _ptr(positions), _stream_of(cache.device)), w)
    return q_out


def veda_cache_attn_workspace_bytes(cache: Cache, batch: CacheBatch, q_heads: int, rows: int) -> int:
    """Bytes of scratch for veda_cache_attn_fwd on buffers of `rows` rows."""
    _ints("veda_cache_attn_workspace_bytes", q_heads, rows)
    bs = batch.struct(rows)
    return int(load().veda_cache_attn_workspace_bytes(cache._ref, C.byref(bs), q_heads))


def veda_packed_attn_workspace_bytes(cache: PackedCache, batch: CacheBatch, q_heads: int, rows: int) -> int:
    """Bytes of scratch for veda_packed_attn_fwd on buffers of `rows` rows."""
    _ints("veda_packed_attn_workspace_bytes", q_heads, rows)
    bs = batch.struct(rows)
    return int(load().veda_packed_attn_workspace_bytes(cache._ref, C.byref(bs), q_heads))


def _attn_fits(cache: Cache, batch: CacheBatch, q: torch.Tensor, softmax_scale: float, block: int, window: int, sinks: int,
               w: str) -> Tuple[veda_strides, veda_visible]:
    """Refuses what the library would refuse, of everything but the buffers; q's strides and the masks."""
    _on(cache.device, w)
    block, window, sinks = operator.index(block), operator.index(window), operator.index(sinks)
    if not (0 <= block <= 1 << 30 and 0 <= window <= 1 << 30 and 0 <= sinks <= 1 << 30):
        _refuse(w, "block, window and sinks must be 0 .. 2^30")
    if not 0.0 < softmax_scale < math.inf:
        _refuse(w, "softmax_scale must be positive and finite")
    sq, heads = _rows(cache, q, q.shape[0], w, "q"), q.shape[1]
    if heads < 1 or heads % cache.kv_heads:
        _refuse(w, f"{heads} query heads on {cache.kv_heads} key heads")
    if heads > 32 * cache.kv_heads:
        raise VedaError(VEDA_ERR_UNSUPPORTED, w, "more than 32 query heads to a key head")
    if batch.page_table.device != cache.device:
        _refuse(w, "the batch must be where the cache is")
    return sq, _visible(block, window, sinks)


def _attn_fwd(kind: str, cache, batch: CacheBatch, q: torch.Tensor, softmax_scale: float, block: int, window: int, sinks: int,
              out: Optional[torch.Tensor], lse: Optional[torch.Tensor], want_lse: bool, workspace: Optional[torch.Tensor]):
    w = kind + "_fwd"
    sq, visible = _attn_fits(cache, batch, q, softmax_scale, block, window, sinks, w)
    rows, heads = q.shape[0], q.shape[1]
    if out is None:
        out = torch.empty((rows, heads, cache.head_dim), dtype=cache.dtype, device=cache.device)
    so = _rows(cache, out, rows, w, "out")
    if out.shape[1] != heads:
        _refuse(w, "out must have q's heads")
    if want_lse and lse is None:
        lse = torch.empty((heads, rows), dtype=torch.float32, device=cache.device)
    if lse is not None and (tuple(lse.shape) != (heads, rows) or lse.dtype != torch.float32 or lse.device != cache.device or not lse.is_contiguous()):
        _refuse(w, "lse must be contiguous fp32 [q_heads, rows]")
    bs = batch.struct(rows)
    lib, ref = load(), C.byref(bs)
    if workspace is None:
        need = int(getattr(lib, kind + "_workspace_bytes")(cache._ref, ref, heads))
        workspace = torch.empty(need, dtype=torch.uint8, device=cache.device) if need else None
    elif workspace.device != cache.device or not workspace.is_contiguous():
        _refuse(w, "the workspace must be contiguous and where the cache is")
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(getattr(lib, w)(cache._ref, ref, heads, q.data_ptr(), sq, softmax_scale, visible, out.data_ptr(), so,
                           _ptr(lse), _ptr(workspace) or None, nbytes, _stream_of(cache.device)), w)
    return out, lse


def veda_cache_attn_fwd(cache: Cache, batch: CacheBatch, q: torch.Tensor, softmax_scale: float, block: int = 1, window: int = 0, sinks: int = 0,
                        out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, want_lse: bool = False,
                        workspace: Optional[torch.Tensor] = None):
    """Attention of the new rows q [rows, q_heads, d] over the cache.  block, window, sinks: which keys a row sees (veda_visible: block 1
    causal, 0 everything).  Returns (out [rows, q_heads, d], lse fp32 [q_heads, rows] or None); rows of no sequence are left as they are
    in buffers given, and undefined in buffers made here."""
    return _attn_fwd("veda_cache_attn", cache, batch, q, softmax_scale, block, window, sinks, out, lse, want_lse, workspace)


def veda_packed_append(cache: PackedCache, batch: CacheBatch, k: torch.Tensor, v: torch.Tensor, rope: Optional[Rope] = None,
                       positions: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                       k_out: Optional[torch.Tensor] = None, v_out: Optional[torch.Tensor] = None):
    """veda_cache_append into a cache held in 4 bits.  k_out, v_out [rows, kv_heads, d]: the rows as the cache then stands for them."""
    w, rows = "veda_packed_append", k.shape[0]
    _on(cache.device, w)
    _need(isinstance(cache, PackedCache), w, "the cache is not held in 4 bits")
    if rope is not None and rope.handle is None:    # which the library would take for no rope
        _refuse(w, "the rope is closed")
    kv, sq, so, sko, svo = cache.kv_heads, _NO_ROWS, _NO_ROWS, _NO_ROWS, _NO_ROWS
    sk, sv = _rows(cache, k, rows, w, "k", kv), _rows(cache, v, rows, w, "v", kv)
    if k_out is not None:
        sko = _rows(cache, k_out, rows, w, "k_out", kv)
    if v_out is not None:
        svo = _rows(cache, v_out, rows, w, "v_out", kv)
    if batch.page_table.device != cache.device:
        _refuse(w, "the batch must be where the cache is")
    heads = 0
    if q is not None:
        sq = _rows(cache, q, rows, w, "q")
        heads = q.shape[1]
        if q_out is None:
            q_out = torch.empty((rows, heads, cache.head_dim), dtype=cache.dtype, device=cache.device)
        so = _rows(cache, q_out, rows, w, "q_out", heads)
    else:
        _need(q_out is None, w, "q_out without q")
    if positions is not None and (rope is None or positions.shape != (rows, rope.axes) or positions.dtype != torch.int32 or
                                  positions.device != cache.device or not positions.is_contiguous()):
        _refuse(w, "positions must be contiguous i32 [rows, axes of rope]")
    bs = batch.struct(rows)
    _check(load().veda_packed_append(cache._ref, C.byref(bs), k.data_ptr(), sk, v.data_ptr(), sv, heads, _ptr(q), sq,
                                     _ptr(q_out), so, None if rope is None else rope.handle, _ptr(positions), _ptr(k_out), sko, _ptr(v_out), svo,
                                     _stream_of(cache.device)), w)
    return q_out


def veda_packed_attn_fwd(cache: PackedCache, batch: CacheBatch, q: torch.Tensor, softmax_scale: float, block: int = 1, window: int = 0, sinks: int = 0,
                         out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, want_lse: bool = False,
                         workspace: Optional[torch.Tensor] = None):
    """veda_cache_attn_fwd over a cache held in 4 bits: the same arguments and results."""
    _need(isinstance(cache, PackedCache), "veda_packed_attn_fwd", "the cache is not held in 4 bits")
    return _attn_fwd("veda_packed_attn", cache, batch, q, softmax_scale, block, window, sinks, out, lse, want_lse, workspace)


_I32 = np.dtype(np.int32)


def _pairs(pairs, w: str) -> Tuple[bytes, int]:
    """The numbers as bytes, whose place ctypes knows (a numpy array takes 2 us to tell its own), and how many pairs they are."""
    p = np.asarray(pairs)
    if p.size and not (p.shape[1] == 2 if p.ndim == 2 else p.ndim == 1 and p.size % 2 == 0):     # sources and targets as two rows, say
        _refuse(w, "pairs must be page numbers [n, 2]")
    if p.dtype != _I32:
        _need(p.size == 0 or (p.dtype.kind in "iu" and 0 <= p.min() and p.max() < 1 << 31), w, "pairs must be page numbers [n, 2]")
        p = p.astype(_I32)
    return p.tobytes(), p.size // 2


def veda_cache_copy_pages(cache: Cache, pairs):
    """Copies pages (from, to) [n, 2] inside both pools, as if one after the other."""
    w = "veda_cache_copy_pages"
    _on(cache.device, w)
    p, n = _pairs(pairs, w)
    _check(load().veda_cache_copy_pages(cache._ref, p, n, _stream_of(cache.device)), w)


def veda_packed_copy_pages(cache: PackedCache, pairs):
    """veda_cache_copy_pages for a cache held in 4 bits."""
    w = "veda_packed_copy_pages"
    _on(cache.device, w)
    _need(isinstance(cache, PackedCache), w, "the cache is not held in 4 bits")
    p, n = _pairs(pairs, w)
    _check(load().veda_packed_copy_pages(cache._ref, p, n, _stream_of(cache.device)), w)


class Pages:
    """veda_pages: which page belongs to which sequence (host).  extend and compact return the pairs [n, 2] for
    veda_cache_copy_pages, which has to run before the pages are used."""

    def __init__(self, pages: int, page_tokens: int, max_seqs: int, max_pages: int):
        h = C.c_void_p()
        self.handle = None
        _ints("Pages", pages, page_tokens, max_seqs, max_pages)
        _check(load().veda_pages_create(pages, page_tokens, max_seqs, max_pages, C.byref(h)), "veda_pages_create")
        self.handle, self.pages, self.page_tokens, self.max_seqs, self.max_pages = h, pages, page_tokens, max_seqs, max_pages

    def _copies(self, name: str, capacity: int, *args):
        _ints(name, *args)
        buf, n = np.empty((capacity, 2), np.int32), C.c_int32()
        _book(getattr(load(), name)(self.handle, *args, buf.ctypes.data_as(C.c_void_p), capacity, C.byref(n)), name)
        return buf[:n.value]

    def table(self) -> np.ndarray:
        """A copy of the table, i32 [max_seqs, max_pages], -1 where there is no page."""
        t = load().veda_pages_table(self.handle)
        _need(bool(t), "veda_pages_table", "the book is closed")
        return np.ctypeslib.as_array(t, (self.max_seqs, self.max_pages)).copy()

    def length(self, seq: int) -> int:
        _ints("veda_pages_length", seq)
        n = int(load().veda_pages_length(self.handle, seq))
        _need(n >= 0, "veda_pages_length", f"no sequence {seq}")
        return n

    def free_count(self) -> int:
        n = int(load().veda_pages_free_count(self.handle))
        _need(n >= 0, "veda_pages_free_count", "the book is closed")
        return n

    def extend(self, seq: int, tokens: int) -> np.ndarray:
        return self._copies("veda_pages_extend", 1, seq, tokens)

    def fork(self, source: int, target: int):
        _ints("veda_pages_fork", source, target)
        _book(load().veda_pages_fork(self.handle, source, target), "veda_pages_fork")

    def truncate(self, seq: int, tokens: int = 0):
        _ints("veda_pages_truncate", seq, tokens)
        _book(load().veda_pages_truncate(self.handle, seq, tokens), "veda_pages_truncate")

    def evict(self, seq: int, first: int, last: int):
        _ints("veda_pages_evict", seq, first, last)
        _book(load().veda_pages_evict(self.handle, seq, first, last), "veda_pages_evict")

    def compact(self) -> np.ndarray:
        return self._copies("veda_pages_compact", self.pages)

    def close(self):
        if self.handle is not None:
            load().veda_pages_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _book(status: int, where: str):
    if status == VEDA_ERR_WORKSPACE:
        raise VedaError(status, where, load().veda_last_error().decode())
    _check(status, where)


class DevicePages:
    """A page book on the GPU (veda_device_pages): table i32 [max_seqs, max_pages], length i32 [max_seqs], used i32 [(pages + 31) / 32],
    made here (empty) unless given."""

    def __init__(self, pages: int, page_tokens: int, max_seqs: int, max_pages: int, device="cuda", table: Optional[torch.Tensor] = None,
                 length: Optional[torch.Tensor] = None, used: Optional[torch.Tensor] = None):
        _ints("DevicePages", pages, page_tokens, max_seqs, max_pages)
        _need(min(pages, page_tokens, max_seqs, max_pages) >= 1, "DevicePages", "a book has pages, tokens to a page, sequences and pages of one")
        shapes = ((max_seqs, max_pages), (max_seqs,), ((pages + 31) // 32,))
        self.table, self.length, self.used = (torch.zeros(n, dtype=torch.int32, device=device) if t is None else t
                                              for t, n in zip((table, length, used), shapes))
        self.device = self.table.device
        for t, n in zip((self.table, self.length, self.used), shapes):
            _need(tuple(t.shape) == n and t.dtype == torch.int32 and t.device == self.device and t.is_contiguous(), "DevicePages",
                  f"table, length and used must be contiguous i32 {list(shapes[0])}, {list(shapes[1])}, {list(shapes[2])}")
        self.pages, self.page_tokens, self.max_seqs, self.max_pages = int(pages), int(page_tokens), int(max_seqs), int(max_pages)
        self._struct = veda_device_pages(self.pages, self.page_tokens, self.max_seqs, self.max_pages, _ptr(self.table), _ptr(self.length), _ptr(self.used))
        self._ref = C.byref(self._struct)


class StepTables:
    """What veda_pages_step writes for up to `rows` new rows of `seqs` requests, of which none grows by more than max_new; made here unless given.
    axes, frame (H, W): what `positions` are.  `batch` is the CacheBatch of the step's calls, on row buffers of `rows` rows."""

    def __init__(self, book: DevicePages, seqs: int, rows: int, max_new: int, axes: int = 1, frame: Tuple[int, int] = (1, 1),
                 page_table: Optional[torch.Tensor] = None, kv_len: Optional[torch.Tensor] = None, q_start: Optional[torch.Tensor] = None,
                 status: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None, row_seq: Optional[torch.Tensor] = None,
                 slots: Optional[torch.Tensor] = None):
        w, dev = "StepTables", book.device
        _ints(w, seqs, rows, max_new, axes, *frame)
        _need(seqs >= 0 and rows >= 0 and axes in (1, 3), w, "seqs and rows are not negative, axes are 1 or 3")

        def take(t, shape, dtype):
            if t is None:
                return torch.zeros(shape, dtype=dtype, device=dev)
            _need(tuple(t.shape) == shape and t.dtype == dtype and t.device == dev and t.is_contiguous(), w, f"a table must be contiguous {dtype} {list(shape)}")
            return t

        i32 = torch.int32
        self.page_table, self.kv_len = take(page_table, (seqs, book.max_pages), i32), take(kv_len, (seqs,), i32)
        self.q_start, self.status = take(q_start, (seqs + 1,), i32), take(status, (seqs,), i32)
        self.positions, self.row_seq = take(positions, (rows, axes), i32), take(row_seq, (rows,), i32)
        self.slots = take(slots, (rows,), torch.int64)
        self.seqs, self.rows, self.max_new, self.axes, self.frame, self.max_pages, self.device = seqs, rows, int(max_new), axes, tuple(frame), book.max_pages, dev
        self.batch = CacheBatch(self.page_table, self.kv_len, self.q_start, max_new)
        self._struct = veda_step_tables(book.max_pages, *(_ptr(t) for t in (self.page_table, self.kv_len, self.q_start, self.status, self.positions,
                                                                            self.row_seq, self.slots)))
        self._ref = C.byref(self._struct)


def veda_pages_step(book: DevicePages, out: StepTables, grow: torch.Tensor, seq: Optional[torch.Tensor] = None, keep: Optional[torch.Tensor] = None,
                    evict: Optional[torch.Tensor] = None) -> StepTables:
    """One step of the book: request i keeps the first keep[i] tokens of sequence seq[i] (all; sequence i), gives back the pages wholly within
    evict[i] = (first, last) of them (none) and grows by grow[i]; all i32 on the GPU, read when the kernels run.  Fills and returns `out`."""
    w = "veda_pages_step"
    _on(book.device, w)
    _need(out.max_pages == book.max_pages and out.device == book.device, w, "the tables were made for another book")
    n = out.seqs
    for t, shape in ((grow, (n,)), (seq, (n,)), (keep, (n,)), (evict, (n, 2))):
        if t is not None and (tuple(t.shape) != shape or t.dtype != torch.int32 or t.device != book.device or not t.is_contiguous()):
            _refuse(w, f"grow, seq and keep must be contiguous i32 [{n}], evict [{n}, 2], where the book is")
    step = veda_step(n, out.rows, out.max_new, out.axes, *out.frame, _ptr(seq), _ptr(keep), _ptr(evict), _ptr(grow))
    _check(load().veda_pages_step(book._ref, C.byref(step), out._ref, _stream_of(book.device)), w)
    return out


def veda_cache_attention(cache: Cache, batch: CacheBatch, q, k, v, softmax_scale: float, rope: Optional[Rope] = None,
                         positions: Optional[torch.Tensor] = None, block: int = 1, window: int = 0, sinks: int = 0,
                         buffers: Optional[dict] = None):
    """One attention call of a streaming step: q and k rotated, k and v appended, attention of the new rows over the cache (a Cache or a PackedCache).
    Returns (out [rows, q_heads, d], buffers); `buffers` (optional dict) is filled on the first call and reused afterwards, by calls
    of the same rows, heads and table (a captured call writes to them whenever it is replayed, so they are never exchanged for others).
    A call that is refused appends nothing and leaves the buffers as they were."""
    w, b = "veda_cache_attention", {} if buffers is None else buffers
    sq, _ = _attn_fits(cache, batch, q, softmax_scale, block, window, sinks, w)     # before K and V are written
    es = q.element_size()
    if rope is None and (q.data_ptr() % 16 or any(n > 1 and s * es % 16 for n, s in ((q.shape[0], sq.n), (q.shape[1], sq.h)))):
        raise VedaError(VEDA_ERR_UNSUPPORTED, w, "rows of q must begin at multiples of 16 bytes")
    append, attend, room = ((veda_packed_append, veda_packed_attn_fwd, veda_packed_attn_workspace_bytes) if isinstance(cache, PackedCache) else
                            (veda_cache_append, veda_cache_attn_fwd, veda_cache_attn_workspace_bytes))
    need = room(cache, batch, q.shape[1], q.shape[0])
    out, ws = b.get("out"), b.get("ws")
    if (out is not None and (out.shape != q.shape or out.dtype != q.dtype or out.device != q.device) or
            ws is not None and ws.numel() * ws.element_size() < need):
        _refuse(w, "these buffers were made for a call of other sizes")
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if ws is None:
        ws = torch.empty(need, dtype=torch.uint8, device=q.device)
    turned = None
    if rope is not None:
        turned = append(cache, batch, k, v, rope, positions, q, b.get("q"))
    else:
        append(cache, batch, k, v, None, positions)
    attend(cache, batch, q if rope is None else turned, softmax_scale, block, window, sinks, out, workspace=ws)
    b.update(out=out, ws=ws)
    if rope is not None:
        b["q"] = turned
    return out, b
