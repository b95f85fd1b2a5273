"""Thin ctypes binding of the C ABI in include/fi.h.

Only argument marshalling happens here: torch tensors provide device memory and the current CUDA stream;
every step of a look-up runs in the library's kernels.  Loading fails loudly when the library is missing:
there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import List, Optional, Sequence

import torch

from . import build as _build

FI_OK = 0
FI_ERR_INVALID_ARG, FI_ERR_CAPACITY, FI_ERR_OOM, FI_ERR_CUDA, FI_ERR_UNSUPPORTED, FI_ERR_TIMEOUT = 1, 2, 3, 4, 5, 6
FI_F32, FI_BF16 = 0, 1
FI_HIT_CONF_GT, FI_HIT_DIST_LE = 0, 1
FI_METRIC_SQL2, FI_METRIC_L2 = 0, 1
FI_PATH_AUTO, FI_PATH_STREAM, FI_PATH_GEMM = 0, 1, 2

EXPORTS = ["fi_cache_create", "fi_cache_destroy", "fi_cache_insert", "fi_cache_set_threshold", "fi_cache_set_path",
           "fi_cache_size", "fi_cache_lookup_batch", "fi_cascade_init", "fi_cascade_step", "fi_cache_lookup_batch_host",
           "fi_cascade_run_host", "fi_cache_poll_status", "fi_cache_set_profiling",
           "fi_cache_read_profile", "fi_lookup_noalloc", "fi_cache_compute_threshold", "fi_cache_clear", "fi_kmeans_step", "fi_cache_selftest_wait", "fi_cache_neighbor_tuples", "fi_merge_shard_lookups",
           "fi_projection_create", "fi_projection_destroy", "fi_projection_set_weights", "fi_projection_apply", "fi_projection_poll_status", "fi_projection_set_profiling",
           "fi_projection_read_profile",
           "fi_cascade_step_projected", "fi_cache_set_repair", "fi_cache_read_certificate",
           "fi_cache_read_slot_certificates", "fi_cache_lookup_view", "fi_cache_set_sm_limit", "fi_gemm_plan_describe",
           "fi_pages_create", "fi_pages_destroy", "fi_pages_extend", "fi_pages_release", "fi_head_norm_rope",
           "fi_head_norm_rope_backward", "fi_head_norm_rope_workspace", "fi_kv_create", "fi_kv_destroy", "fi_kv_append",
           "fi_kv_attend", "fi_kv_set_wait_limit", "fi_kv_poll_status", "fi_launch_count", "fi_last_error", "fi_status_string"]


class fi_cache_config_t(ctypes.Structure):
    _fields_ = [("dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("capacity", ctypes.c_int64),
                ("num_classes", ctypes.c_int32), ("k", ctypes.c_int32), ("rule", ctypes.c_int32),
                ("metric", ctypes.c_int32), ("threshold", ctypes.c_float), ("device", ctypes.c_int32),
                ("max_batch", ctypes.c_int32), ("path", ctypes.c_int32)]


class fi_lookup_out_t(ctypes.Structure):
    _fields_ = [("label", ctypes.c_void_p), ("conf", ctypes.c_void_p), ("hit", ctypes.c_void_p),
                ("topk_dist", ctypes.c_void_p), ("topk_idx", ctypes.c_void_p)]


class fi_cascade_state_t(ctypes.Structure):
    _fields_ = [("active_idx", ctypes.c_void_p), ("active_count", ctypes.c_void_p), ("miss_idx", ctypes.c_void_p),
                ("miss_count", ctypes.c_void_p), ("final_label", ctypes.c_void_p), ("exit_stage", ctypes.c_void_p),
                ("final_conf", ctypes.c_void_p), ("stage", ctypes.c_int32), ("batch0", ctypes.c_int32)]


def _fields(kind, names: str):
    return [(n, kind) for n in names.split()]


class fi_pages_config_t(ctypes.Structure):
    _fields_ = _fields(ctypes.c_int32, "page_size max_blocks max_batch device")


class fi_pages_extend_t(ctypes.Structure):
    _fields_ = _fields(ctypes.c_void_p, "lens free_pages free_count block_table row_idx batch_count new_lens slot_map "
                                        "positions cu_tokens granted lens_out free_count_out") \
        + [("table_ld", ctypes.c_int64)] + _fields(ctypes.c_int32, "rows num_pages batch_max max_tokens")


class fi_head_norm_rope_t(ctypes.Structure):
    _fields_ = _fields(ctypes.c_void_p, "q k q_out k_out dq_out dk_out q_weight k_weight rope positions tokens_dev "
                                        "dq_weight dk_weight workspace") \
        + _fields(ctypes.c_int64, "q_token_stride q_head_stride k_token_stride k_head_stride q_out_token_stride "
                                  "q_out_head_stride k_out_token_stride k_out_head_stride dq_out_token_stride "
                                  "dq_out_head_stride dk_out_token_stride dk_out_head_stride tokens") \
        + _fields(ctypes.c_int32, "q_heads k_heads head_dim rot_dim max_pos interleaved dtype") + [("eps", ctypes.c_float)]


class fi_kv_config_t(ctypes.Structure):
    _fields_ = _fields(ctypes.c_void_p, "k_codes v_codes k_meta v_meta") \
        + _fields(ctypes.c_int64, "page_stride head_stride token_stride meta_page_stride meta_head_stride meta_token_stride") \
        + _fields(ctypes.c_int32, "num_pages page_size q_heads kv_heads head_dim device")


class fi_kv_append_t(ctypes.Structure):
    _fields_ = _fields(ctypes.c_void_p, "k v slot_map tokens_dev k_stored v_stored") \
        + _fields(ctypes.c_int64, "k_token_stride k_head_stride v_token_stride v_head_stride tokens") + [("dtype", ctypes.c_int32)]


class fi_kv_attend_t(ctypes.Structure):
    _fields_ = _fields(ctypes.c_void_p, "q out lse lens block_table row_idx batch_count cu_tokens granted") \
        + _fields(ctypes.c_int64, "q_token_stride q_head_stride out_token_stride out_head_stride table_ld") \
        + _fields(ctypes.c_int32, "rows max_blocks batch_max max_tokens max_query window dtype") + [("scale", ctypes.c_float)]


class FiError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{status_string(status)}: {message}")
        self.status = status


_lib = None


def load_library(path: Optional[str] = None):
    """dlopen libficache.so (built in-tree by `build.build_library`) and declare the prototypes."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    path = path or _build.LIB
    if not os.path.exists(path):
        raise FileNotFoundError(f"{path} is missing: build it with paper_2002_02645_b200.build.build_library()")
    lib = ctypes.CDLL(path)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    lib.fi_cache_create.argtypes = [ctypes.POINTER(fi_cache_config_t), ctypes.POINTER(vp)]
    lib.fi_cache_destroy.argtypes = [vp]
    lib.fi_cache_insert.argtypes = [vp, vp, vp, vp, i64, vp]
    lib.fi_cache_set_threshold.argtypes = [vp, ctypes.c_float]
    lib.fi_cache_set_path.argtypes = [vp, i32]
    lib.fi_cache_size.argtypes = [vp]
    lib.fi_cache_size.restype = i64
    lib.fi_cache_lookup_batch.argtypes = [vp, vp, i64, vp, i32, vp, ctypes.POINTER(fi_lookup_out_t), vp]
    lib.fi_cascade_init.argtypes = [ctypes.POINTER(fi_cascade_state_t), i32, i32, vp]
    lib.fi_cascade_step.argtypes = [vp, vp, i64, ctypes.POINTER(fi_cascade_state_t), vp]
    lib.fi_cache_lookup_batch_host.argtypes = [vp, vp, i32, ctypes.POINTER(fi_lookup_out_t), vp]
    lib.fi_cascade_run_host.argtypes = [ctypes.POINTER(vp), i32, ctypes.POINTER(vp), i32, vp, vp, vp, vp, vp]
    lib.fi_cache_poll_status.argtypes = [vp]
    lib.fi_cache_clear.argtypes = [vp]
    lib.fi_cache_neighbor_tuples.argtypes = [vp, vp, i64, i32, vp, vp, vp, vp]
    lib.fi_merge_shard_lookups.argtypes = [i32, i32, i32, vp, vp, vp, vp, i32, i32, ctypes.c_float,
                                           ctypes.POINTER(fi_lookup_out_t), vp]
    lib.fi_projection_create.argtypes = [i32, i32, i32, i32, ctypes.POINTER(vp)]
    lib.fi_projection_destroy.argtypes = [vp]
    lib.fi_projection_set_weights.argtypes = [vp, vp, vp, vp]
    lib.fi_projection_poll_status.argtypes = [vp]
    lib.fi_projection_set_profiling.argtypes = [vp, i32]
    lib.fi_projection_read_profile.argtypes = [vp, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(i32)]
    lib.fi_projection_apply.argtypes = [vp, vp, i64, vp, i32, vp, vp, i64, vp]
    lib.fi_cascade_step_projected.argtypes = [vp, vp, vp, i64, ctypes.POINTER(fi_cascade_state_t), vp]
    lib.fi_cache_selftest_wait.argtypes = [vp, i64, vp]
    lib.fi_kmeans_step.argtypes = [vp, vp, i64, vp, i64, vp, vp, vp, vp, vp, vp]
    lib.fi_cache_compute_threshold.argtypes = [vp, vp, i64, vp, i64, ctypes.POINTER(ctypes.c_float),
                                               ctypes.POINTER(i64), vp]
    lib.fi_lookup_noalloc.argtypes = [vp, vp, vp, i64, i32, i32, i32, i32, i32, ctypes.c_float, vp, i64, i32,
                                      ctypes.POINTER(fi_lookup_out_t), vp]
    lib.fi_cache_lookup_view.argtypes = [vp]
    lib.fi_cache_lookup_view.restype = i64
    lib.fi_cache_set_sm_limit.argtypes = [vp, i32]
    lib.fi_cache_set_repair.argtypes = [vp, i32]
    lib.fi_cache_read_certificate.argtypes = [vp, ctypes.POINTER(i64), ctypes.POINTER(i64), ctypes.POINTER(ctypes.c_float)]
    lib.fi_cache_read_slot_certificates.argtypes = [vp, vp, i32]
    lib.fi_cache_set_profiling.argtypes = [vp, i32]
    lib.fi_cache_read_profile.argtypes = [vp, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(i32)]
    lib.fi_gemm_plan_describe.argtypes = [i32, i64, i32, i32, i32, i32, i32, ctypes.POINTER(i32), ctypes.POINTER(i32),
                                          ctypes.POINTER(i32)]
    lib.fi_gemm_plan_describe.restype = i32
    ptr = ctypes.POINTER
    lib.fi_pages_create.argtypes = [ptr(fi_pages_config_t), ptr(vp)]
    lib.fi_pages_destroy.argtypes = [vp]
    lib.fi_pages_extend.argtypes = [vp, ctypes.c_char_p, vp]           # a packed fi_pages_extend_t
    lib.fi_pages_release.argtypes = [vp, vp, i32, vp, vp, i32, vp, i64, vp, i32, vp, vp, vp, vp]
    lib.fi_head_norm_rope.argtypes = [ctypes.c_char_p, vp]             # a packed fi_head_norm_rope_t
    lib.fi_head_norm_rope_backward.argtypes = [ctypes.c_char_p, vp]
    lib.fi_head_norm_rope_workspace.argtypes = [i32]
    lib.fi_head_norm_rope_workspace.restype = i64
    lib.fi_kv_create.argtypes = [ptr(fi_kv_config_t), ptr(vp)]
    lib.fi_kv_destroy.argtypes = [vp]
    lib.fi_kv_append.argtypes = [vp, ctypes.c_char_p, vp]           # a packed fi_kv_append_t
    lib.fi_kv_attend.argtypes = [vp, ctypes.c_char_p, vp]           # a packed fi_kv_attend_t
    lib.fi_kv_set_wait_limit.argtypes = [vp, i64]
    lib.fi_kv_poll_status.argtypes = [vp]
    lib.fi_launch_count.argtypes = []
    lib.fi_launch_count.restype = i64
    lib.fi_last_error.argtypes = []
    lib.fi_last_error.restype = ctypes.c_char_p
    lib.fi_status_string.argtypes = [i32]
    lib.fi_status_string.restype = ctypes.c_char_p
    for name in EXPORTS:
        fn = getattr(lib, name)
        if fn.restype is ctypes.c_int:   # default: the fi_status_t functions
            fn.restype = i32
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load_library().fi_status_string(int(status)).decode()


def _check(status: int) -> None:
    if status != FI_OK:
        raise FiError(status, load_library().fi_last_error().decode())


PLAN_FIELDS = ("count", "m_tiles", "mg", "groups", "parts", "range16", "list_len", "tile_m", "lists", "mode", "n_tiles",
               "tail_tiles", "tail_slices", "pieces", "half", "span_full", "span_half")


def gemm_plan_describe(count: int, n_entries: int, num_ctas: int, k: int, dim: int, max_batch: int, cta: int = -1):
    """Host only: the work split of the distance GEMM as a dict, plus (spans mode, cta >= 0) that CTA's pieces as
    tuples (query tile, cache-row tile, first k-block, end k-block, 128-row MMAs, slot)."""
    plan = (ctypes.c_int32 * 17)()
    items = (ctypes.c_int32 * 18)()
    n = ctypes.c_int32(0)
    _check(load_library().fi_gemm_plan_describe(count, n_entries, num_ctas, k, dim, max_batch, cta, plan, items,
                                                ctypes.byref(n)))
    return dict(zip(PLAN_FIELDS, plan)), [tuple(items[6 * i:6 * i + 6]) for i in range(n.value)]


def launch_count() -> int:
    return int(load_library().fi_launch_count())


def _stream_ptr(device: torch.device) -> int:
    return torch.cuda.current_stream(device).cuda_stream


# the same for an ordinal, without making a Stream object, and the current ordinal: a decode step makes three of these calls per layer
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _dp(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


_TORCH_DTYPE = {FI_F32: torch.float32, FI_BF16: torch.bfloat16}


class LookupOut:
    """Device arrays a look-up writes (torch owns the memory)."""

    def __init__(self, batch: int, k: int, device, with_topk: bool = True):
        self.label = torch.empty(batch, dtype=torch.int32, device=device)
        self.conf = torch.empty(batch, dtype=torch.float32, device=device)
        self.hit = torch.empty(batch, dtype=torch.uint8, device=device)
        self.topk_dist = torch.empty(batch, k, dtype=torch.float32, device=device) if with_topk else None
        self.topk_idx = torch.empty(batch, k, dtype=torch.int32, device=device) if with_topk else None

    def as_struct(self) -> fi_lookup_out_t:
        return fi_lookup_out_t(_dp(self.label), _dp(self.conf), _dp(self.hit), _dp(self.topk_dist), _dp(self.topk_idx))


class FreezeCache:
    """CACHE[layer] and THRESHOLDS[layer] of one layer, resident on one GPU."""

    def __init__(self, *, dim: int, capacity: int, num_classes: int, k: int, dtype: int = FI_BF16,
                 rule: int = FI_HIT_CONF_GT, metric: int = FI_METRIC_SQL2, threshold: float = 0.0, device: int = 0,
                 max_batch: int = 1024, path: int = FI_PATH_AUTO):
        self._lib = load_library()
        self._h = ctypes.c_void_p()
        self.cfg = fi_cache_config_t(dim, dtype, capacity, num_classes, k, rule, metric, threshold, device, max_batch, path)
        self.device = torch.device("cuda", device)
        _check(self._lib.fi_cache_create(ctypes.byref(self.cfg), ctypes.byref(self._h)))

    # -- fi_cache_destroy
    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h.value:
            self._lib.fi_cache_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def handle(self) -> ctypes.c_void_p:
        return self._h

    @property
    def k(self) -> int:
        return self.cfg.k

    @property
    def dim(self) -> int:
        return self.cfg.dim

    def _check_vecs(self, t: torch.Tensor) -> None:
        if t.device != self.device or t.dtype != _TORCH_DTYPE[self.cfg.dtype] or t.dim() != 2 or t.shape[1] != self.cfg.dim \
                or t.stride(1) != 1:
            raise ValueError("vectors must be a 2-D tensor of the cache's dtype, dim and device with unit inner stride")

    # -- fi_cache_insert
    def insert(self, vecs: torch.Tensor, labels: torch.Tensor, weights: Optional[torch.Tensor] = None) -> None:
        self._check_vecs(vecs)
        if not vecs.is_contiguous():
            raise ValueError("inserted rows must be contiguous")
        if labels.dtype != torch.int32 or labels.device != self.device or labels.numel() != vecs.shape[0]:
            raise ValueError("labels must be int32 on the cache's device, one per row")
        if weights is not None and (weights.dtype != torch.float32 or weights.device != self.device
                                    or weights.numel() != vecs.shape[0]):
            raise ValueError("weights must be float32 on the cache's device, one per row")
        _check(self._lib.fi_cache_insert(self._h, _dp(vecs), _dp(labels), _dp(weights), vecs.shape[0],
                                         _stream_ptr(self.device)))

    # -- fi_cache_set_threshold / fi_cache_set_path / fi_cache_size / fi_cache_poll_status
    def set_threshold(self, tau: float) -> None:
        _check(self._lib.fi_cache_set_threshold(self._h, float(tau)))
        self.cfg.threshold = float(tau)

    def set_path(self, path: int) -> None:
        _check(self._lib.fi_cache_set_path(self._h, int(path)))

    def size(self) -> int:
        return int(self._lib.fi_cache_size(self._h))

    def poll_status(self) -> None:
        _check(self._lib.fi_cache_poll_status(self._h))

    # -- fi_cache_lookup_view / fi_cache_set_sm_limit
    def lookup_view(self) -> int:
        """Entries the most recent look-up covered (inserts still in flight on another stream are not among them)."""
        return int(self._lib.fi_cache_lookup_view(self._h))

    def set_sm_limit(self, sms: int) -> None:
        _check(self._lib.fi_cache_set_sm_limit(self._h, int(sms)))

    # -- fi_cache_set_repair / fi_cache_read_certificate / fi_cache_read_slot_certificates
    def set_repair(self, enable: bool) -> None:
        _check(self._lib.fi_cache_set_repair(self._h, 1 if enable else 0))

    def read_certificate(self):
        """(requests without a certificate since the last read, of those not repaired, largest observed score error)."""
        unc, unrep, err = ctypes.c_int64(0), ctypes.c_int64(0), ctypes.c_float(0.0)
        _check(self._lib.fi_cache_read_certificate(self._h, ctypes.byref(unc), ctypes.byref(unrep), ctypes.byref(err)))
        return int(unc.value), int(unrep.value), float(err.value)

    def slot_certificates(self, n: int) -> torch.Tensor:
        """Flags of the most recent look-up, slots 0..n-1 (host uint8 tensor, 1 = certified or repaired)."""
        flags = torch.zeros(max(n, 1), dtype=torch.uint8)
        _check(self._lib.fi_cache_read_slot_certificates(self._h, flags.data_ptr(), int(n)))
        return flags[:n]

    # -- fi_cache_neighbor_tuples
    def neighbor_tuples(self, topk_idx: torch.Tensor, index_offset: int):
        """(global index, label, weight) of the neighbours a look-up on this shard returned."""
        n = topk_idx.numel()
        gi = torch.empty_like(topk_idx)
        lab = torch.empty_like(topk_idx)
        wgt = torch.empty(topk_idx.shape, dtype=torch.float32, device=self.device)
        _check(self._lib.fi_cache_neighbor_tuples(self._h, _dp(topk_idx), n, int(index_offset), _dp(gi), _dp(lab), _dp(wgt),
                                                  _stream_ptr(self.device)))
        return gi, lab, wgt

    # -- fi_cache_selftest_wait
    def selftest_wait(self, limit_cycles: int = 2_000_000) -> None:
        """Enqueue the bounded-wait self-test; the next poll_status() raises FI_ERR_TIMEOUT."""
        _check(self._lib.fi_cache_selftest_wait(self._h, int(limit_cycles), _stream_ptr(self.device)))

    # -- fi_cache_clear
    def clear(self) -> None:
        _check(self._lib.fi_cache_clear(self._h))

    # -- fi_kmeans_step
    def kmeans_step(self, points: torch.Tensor, point_labels: torch.Tensor):
        """One Lloyd iteration with this cache's entries as the current centres (k must be 1).
        Returns (assignment [n], new centres [size, dim], counts [size], majority label [size], fraction [size])."""
        self._check_vecs(points)
        n, size = points.shape[0], self.size()
        assign = torch.empty(max(n, 1), dtype=torch.int32, device=self.device)
        centres = torch.empty(size, self.cfg.dim, dtype=_TORCH_DTYPE[self.cfg.dtype], device=self.device)
        counts = torch.empty(size, dtype=torch.int32, device=self.device)
        majority = torch.empty(size, dtype=torch.int32, device=self.device)
        fraction = torch.empty(size, dtype=torch.float32, device=self.device)
        _check(self._lib.fi_kmeans_step(self._h, _dp(points), points.stride(0), _dp(point_labels), n, _dp(assign),
                                        _dp(centres), _dp(counts), _dp(majority), _dp(fraction),
                                        _stream_ptr(self.device)))
        return assign[:n], centres, counts, majority, fraction

    # -- fi_cache_compute_threshold
    def compute_threshold(self, val_acts: torch.Tensor, model_labels: torch.Tensor):
        """ComputeThresholds for this layer: (threshold now set on the cache, number of wrong look-ups)."""
        self._check_vecs(val_acts)
        if model_labels.dtype != torch.int32 or model_labels.device != self.device \
                or model_labels.numel() != val_acts.shape[0]:
            raise ValueError("model_labels must be int32 on the cache's device, one per validation item")
        tau, wrong = ctypes.c_float(0.0), ctypes.c_int64(0)
        _check(self._lib.fi_cache_compute_threshold(self._h, _dp(val_acts), val_acts.stride(0), _dp(model_labels),
                                                    val_acts.shape[0], ctypes.byref(tau), ctypes.byref(wrong),
                                                    _stream_ptr(self.device)))
        return float(tau.value), int(wrong.value)

    # -- fi_cache_set_profiling / fi_cache_read_profile
    def set_profiling(self, enable: bool) -> None:
        _check(self._lib.fi_cache_set_profiling(self._h, 1 if enable else 0))

    def read_profile(self):
        """(summed distance-kernel milliseconds, launches covered) since the last read."""
        ms, n = ctypes.c_float(0.0), ctypes.c_int32(0)
        _check(self._lib.fi_cache_read_profile(self._h, ctypes.byref(ms), ctypes.byref(n)))
        return float(ms.value), int(n.value)

    # -- fi_cache_lookup_batch
    def lookup_batch(self, queries: torch.Tensor, *, row_idx: Optional[torch.Tensor] = None,
                     batch_max: Optional[int] = None, batch_count: Optional[torch.Tensor] = None,
                     out: Optional[LookupOut] = None, with_topk: bool = True) -> LookupOut:
        self._check_vecs(queries)
        if batch_max is None:
            batch_max = int(row_idx.numel()) if row_idx is not None else int(queries.shape[0])
        if out is None:
            out = LookupOut(batch_max, self.cfg.k, self.device, with_topk)
        st = out.as_struct()
        _check(self._lib.fi_cache_lookup_batch(self._h, _dp(queries), queries.stride(0), _dp(row_idx), batch_max,
                                               _dp(batch_count), ctypes.byref(st), _stream_ptr(self.device)))
        return out

    # -- fi_cache_lookup_batch_host
    def lookup_batch_host(self, queries_host: torch.Tensor, out_host: LookupOut) -> LookupOut:
        """queries_host and the arrays of out_host live in (pinned) host memory."""
        if queries_host.is_cuda or not queries_host.is_contiguous() or queries_host.shape[1] != self.cfg.dim:
            raise ValueError("queries_host must be a contiguous host tensor [batch, dim]")
        st = out_host.as_struct()
        _check(self._lib.fi_cache_lookup_batch_host(self._h, _dp(queries_host), queries_host.shape[0], ctypes.byref(st),
                                                    _stream_ptr(self.device)))
        return out_host


def lookup_noalloc(cache_vecs: torch.Tensor, labels: torch.Tensor, weights: torch.Tensor, queries: torch.Tensor, *,
                   k: int, rule: int = FI_HIT_CONF_GT, metric: int = FI_METRIC_SQL2, threshold: float = 0.0,
                   out: Optional[LookupOut] = None) -> LookupOut:
    """fi_lookup_noalloc: the streaming look-up on plain device arrays, scratch inside the library image.
    For callers that cannot allocate device memory; `weights` is required (ones for a plain k-NN cache).
    At most 256 requests per call; calls on one device must not overlap on the GPU."""
    dtype = FI_BF16 if cache_vecs.dtype == torch.bfloat16 else FI_F32
    if queries.dtype != cache_vecs.dtype or queries.dim() != 2 or cache_vecs.dim() != 2 or queries.stride(1) != 1 \
            or not cache_vecs.is_contiguous():
        raise ValueError("cache_vecs and queries must be 2-D tensors of one dtype; cache rows contiguous")
    dev = cache_vecs.device
    if out is None:
        out = LookupOut(queries.shape[0], k, dev)
    st = out.as_struct()
    with torch.cuda.device(dev):
        _check(load_library().fi_lookup_noalloc(_dp(cache_vecs), _dp(labels), _dp(weights), cache_vecs.shape[0],
                                                cache_vecs.shape[1], dtype, k, rule, metric, float(threshold),
                                                _dp(queries), queries.stride(0), queries.shape[0], ctypes.byref(st),
                                                _stream_ptr(dev)))
    return out


class Projection:
    """The dimensionality reduction in front of the look-up (Sec. 3): y = max(0, W x + b) in bf16."""

    def __init__(self, *, in_dim: int, out_dim: int = 1024, device: int = 0, max_batch: int = 1024):
        self._lib = load_library()
        self._h = ctypes.c_void_p()
        self.in_dim, self.out_dim, self.max_batch = in_dim, out_dim, max_batch
        self.device = torch.device("cuda", device)
        _check(self._lib.fi_projection_create(in_dim, out_dim, device, max_batch, ctypes.byref(self._h)))

    # -- fi_projection_destroy
    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h.value:
            self._lib.fi_projection_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def handle(self) -> ctypes.c_void_p:
        return self._h

    # -- fi_projection_set_weights
    def set_weights(self, weights: torch.Tensor, bias: Optional[torch.Tensor] = None) -> None:
        if weights.dtype != torch.bfloat16 or tuple(weights.shape) != (self.out_dim, self.in_dim) \
                or not weights.is_contiguous() or weights.device != self.device:
            raise ValueError("weights must be a contiguous bf16 [out_dim, in_dim] tensor on the projection's device")
        if bias is not None and (bias.dtype != torch.float32 or bias.numel() != self.out_dim or bias.device != self.device):
            raise ValueError("bias must be float32 [out_dim] on the projection's device")
        _check(self._lib.fi_projection_set_weights(self._h, _dp(weights), _dp(bias), _stream_ptr(self.device)))

    # -- fi_projection_poll_status
    def poll_status(self) -> None:
        _check(self._lib.fi_projection_poll_status(self._h))

    # -- fi_projection_set_profiling / fi_projection_read_profile
    def set_profiling(self, enable: bool) -> None:
        _check(self._lib.fi_projection_set_profiling(self._h, 1 if enable else 0))

    def read_profile(self):
        ms, n = ctypes.c_float(0.0), ctypes.c_int32(0)
        _check(self._lib.fi_projection_read_profile(self._h, ctypes.byref(ms), ctypes.byref(n)))
        return float(ms.value), int(n.value)

    # -- fi_projection_apply
    def apply(self, x: torch.Tensor, row_idx: Optional[torch.Tensor] = None, count: Optional[torch.Tensor] = None,
              out: Optional[torch.Tensor] = None) -> torch.Tensor:
        if x.dtype != torch.bfloat16 or x.dim() != 2 or x.shape[1] != self.in_dim or x.stride(1) != 1 or x.device != self.device:
            raise ValueError("x must be a bf16 [batch, in_dim] tensor on the projection's device with unit inner stride")
        batch = int(row_idx.numel()) if row_idx is not None else int(x.shape[0])
        if out is None:
            out = torch.zeros(batch, self.out_dim, dtype=torch.bfloat16, device=self.device)
        _check(self._lib.fi_projection_apply(self._h, _dp(x), x.stride(0), _dp(row_idx), batch, _dp(count), _dp(out),
                                             out.stride(0), _stream_ptr(self.device)))
        return out


def merge_shard_lookups(dist: torch.Tensor, global_idx: torch.Tensor, label: torch.Tensor, weight: torch.Tensor, *,
                        metric: int = FI_METRIC_SQL2, rule: int = FI_HIT_CONF_GT, threshold: float = 0.0) -> LookupOut:
    """fi_merge_shard_lookups on gathered tuples of shape [shards, batch, k]."""
    shards, batch, k = dist.shape
    out = LookupOut(batch, k, dist.device)
    st = out.as_struct()
    with torch.cuda.device(dist.device):
        _check(load_library().fi_merge_shard_lookups(shards, batch, k, _dp(dist.contiguous()), _dp(global_idx.contiguous()),
                                                     _dp(label.contiguous()), _dp(weight.contiguous()), metric, rule,
                                                     float(threshold), ctypes.byref(st), _stream_ptr(dist.device)))
    return out


class CascadeState:
    """Device arrays of a batch walking through the layers (torch owns the memory)."""

    def __init__(self, batch0: int, device):
        self.batch0 = batch0
        self.device = torch.device(device)
        self.idx = [torch.empty(max(batch0, 1), dtype=torch.int32, device=device) for _ in range(2)]
        self.count = [torch.zeros(1, dtype=torch.int32, device=device) for _ in range(2)]
        self.final_label = torch.empty(max(batch0, 1), dtype=torch.int32, device=device)
        self.exit_stage = torch.empty(max(batch0, 1), dtype=torch.int32, device=device)
        self.final_conf = torch.empty(max(batch0, 1), dtype=torch.float32, device=device)
        self.stage = 0

    def struct_for_stage(self, stage: int) -> fi_cascade_state_t:
        src, dst = (stage - 1) & 1, stage & 1
        active_idx = None if stage == 0 else _dp(self.idx[src])
        active_count = None if stage == 0 else _dp(self.count[src])
        return fi_cascade_state_t(active_idx, active_count, _dp(self.idx[dst]), _dp(self.count[dst]),
                                  _dp(self.final_label), _dp(self.exit_stage), _dp(self.final_conf), stage, self.batch0)

    def survivors(self, stage: int):
        """(ids, count) tensors alive after `stage` ran."""
        return self.idx[stage & 1], self.count[stage & 1]


def cascade_init(state: CascadeState, num_stages: int) -> None:
    st = state.struct_for_stage(0)
    _check(load_library().fi_cascade_init(ctypes.byref(st), num_stages, state.device.index or 0,
                                          _stream_ptr(state.device)))
    state.stage = 0


def cascade_step(cache: FreezeCache, stage_acts: torch.Tensor, state: CascadeState, stage: Optional[int] = None) -> None:
    cache._check_vecs(stage_acts)
    if stage is None:
        stage = state.stage
    st = state.struct_for_stage(stage)
    _check(load_library().fi_cascade_step(cache.handle, _dp(stage_acts), stage_acts.stride(0), ctypes.byref(st),
                                          _stream_ptr(cache.device)))
    state.stage = stage + 1


def cascade_step_projected(cache: FreezeCache, proj: Projection, stage_acts: torch.Tensor, state: CascadeState,
                           stage: Optional[int] = None) -> None:
    """fi_cascade_step_projected: project the survivors' activations, look them up, compact the misses."""
    if stage is None:
        stage = state.stage
    st = state.struct_for_stage(stage)
    _check(load_library().fi_cascade_step_projected(cache.handle, proj.handle, _dp(stage_acts), stage_acts.stride(0),
                                                    ctypes.byref(st), _stream_ptr(cache.device)))
    state.stage = stage + 1


def cascade_run_host(caches: Sequence[FreezeCache], acts_host: Sequence[torch.Tensor], final_label: torch.Tensor,
                     exit_stage: torch.Tensor, final_conf: torch.Tensor, arrivals: Optional[torch.Tensor] = None) -> None:
    """All stages with HOST activations and HOST outputs (copies inside, synchronises before returning)."""
    n = len(caches)
    batch0 = int(acts_host[0].shape[0])
    for t in list(acts_host) + [final_label, exit_stage, final_conf]:
        if t.is_cuda or not t.is_contiguous():
            raise ValueError("host variant: tensors must be contiguous host tensors")
    hs = (ctypes.c_void_p * n)(*[c.handle.value for c in caches])
    ap = (ctypes.c_void_p * n)(*[a.data_ptr() for a in acts_host])
    _check(load_library().fi_cascade_run_host(hs, n, ap, batch0, _dp(final_label), _dp(exit_stage), _dp(final_conf),
                                              _dp(arrivals), _stream_ptr(caches[0].device)))


# ---- attention layers behind the caches ----
#
# These calls are made several times per layer and decode step, where the host's time is the step's time: their argument
# blocks are packed in one go, and the checks ask the cheapest question that decides.

_FI_DTYPE = {torch.float32: FI_F32, torch.bfloat16: FI_BF16}


def _packer(kind) -> struct.Struct:
    """Packs the fields of a ctypes structure in order (native layout; null pointers are 0)."""
    code = {ctypes.c_void_p: "P", ctypes.c_int64: "q", ctypes.c_int32: "i", ctypes.c_float: "f"}
    p = struct.Struct("@" + "".join(code[t] for _, t in kind._fields_) + "0q")
    assert p.size == ctypes.sizeof(kind)
    return p


_pack_extend, _pack_norm, _pack_append, _pack_attend = (
    _packer(k).pack for k in (fi_pages_extend_t, fi_head_norm_rope_t, fi_kv_append_t, fi_kv_attend_t))


def _at(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.data_ptr()


def _check_flat(t: Optional[torch.Tensor], name: str, index: int, at_least: int = 0, dtype=torch.int32) -> None:
    if t is not None and (t.dtype is not dtype or t.get_device() != index or t.numel() < at_least or not t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous {dtype} tensor on cuda:{index} with at least {at_least} entries")


def _check_heads(t: torch.Tensor, name: str, index: int, dtype, tokens: int, heads: int, head_dim: int):
    """Strides between tokens and heads of a [tokens, heads, head_dim] tensor."""
    if t.dtype is not dtype or t.get_device() != index or t.shape != (tokens, heads, head_dim):
        raise ValueError(f"{name} must be {dtype} [{tokens}, {heads}, {head_dim}] on cuda:{index}")
    token, head, value = t.stride()
    if value != 1:
        raise ValueError(f"{name}: the values of a head must lie side by side")
    return token, head


def _check_table(block_table: torch.Tensor, rows: int, blocks: int, index: int) -> None:
    if block_table.dtype is not torch.int32 or block_table.get_device() != index or block_table.dim() != 2 \
            or block_table.size(0) < rows or block_table.size(1) < blocks or block_table.stride(1) != 1:
        raise ValueError(f"block_table must be int32 [rows, blocks] on cuda:{index}, a row for each entry of lens (at least "
                         f"{rows} x {blocks})")


class ExtendOut:
    """What KvTables.extend gives (torch owns the memory): slot_map [max_tokens] int64, positions [max_tokens], cu_tokens
    [batch + 1], granted [batch], lens [rows] and free_count [1] int32."""

    def __init__(self, batch: int, max_tokens: int, rows: int, device):
        self.slot_map = torch.empty(max_tokens, dtype=torch.int64, device=device)
        # one block of memory for the small ones; positions first, which the kernel writes 16 bytes at a time
        words = torch.empty(max_tokens + 2 * batch + rows + 2, dtype=torch.int32, device=device)
        self.positions, self.cu_tokens, self.granted, self.lens, self.free_count = words.split_with_sizes(
            [max_tokens, batch + 1, batch, rows, 1])


class KvTables:
    """Page tables of one layer's key/value store: fi_pages_*."""

    def __init__(self, *, page_size: int, max_blocks: int, max_batch: int = 1024, device: int = 0):
        self._lib = load_library()
        self._h = ctypes.c_void_p()
        self.page_size, self.max_blocks, self.max_batch = page_size, max_blocks, max_batch
        self.device, self._index = torch.device("cuda", device), device
        cfg = fi_pages_config_t(page_size, max_blocks, max_batch, device)
        _check(self._lib.fi_pages_create(ctypes.byref(cfg), ctypes.byref(self._h)))

    # -- fi_pages_destroy
    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h.value:
            self._lib.fi_pages_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check_state(self, lens, free_pages, free_count, block_table) -> int:
        index = self._index
        _check_flat(lens, "lens", index)
        _check_flat(free_pages, "free_pages", index)
        _check_flat(free_count, "free_count", index, 1)
        rows = lens.numel()
        _check_table(block_table, rows, self.max_blocks, index)
        return rows

    # -- fi_pages_extend
    def extend(self, lens: torch.Tensor, free_pages: torch.Tensor, free_count: torch.Tensor, block_table: torch.Tensor, *,
               new_lens: Optional[torch.Tensor] = None, row_idx: Optional[torch.Tensor] = None,
               batch_count: Optional[torch.Tensor] = None, max_tokens: Optional[int] = None,
               out: Optional[ExtendOut] = None) -> ExtendOut:
        """Places the step's new tokens (new_lens, or one per request) behind the stored ones.  block_table is written in
        place; lens and free_count stay as they are unless `out` holds them."""
        rows, index = self._check_state(lens, free_pages, free_count, block_table), self._index
        batch = row_idx.numel() if row_idx is not None else rows
        _check_flat(row_idx, "row_idx", index)
        _check_flat(batch_count, "batch_count", index, 1)
        _check_flat(new_lens, "new_lens", index, batch)
        if max_tokens is None:
            if new_lens is not None:
                raise ValueError("max_tokens is needed with new_lens")
            max_tokens = batch
        if out is None:
            out = ExtendOut(batch, max_tokens, rows, self.device)
        else:
            _check_flat(out.slot_map, "out.slot_map", index, max_tokens, torch.int64)
            _check_flat(out.positions, "out.positions", index, max_tokens)
            _check_flat(out.cu_tokens, "out.cu_tokens", index, batch + 1)
            _check_flat(out.granted, "out.granted", index, batch)
            _check_flat(out.lens, "out.lens", index, rows)
            _check_flat(out.free_count, "out.free_count", index, 1)
        args = _pack_extend(lens.data_ptr(), free_pages.data_ptr(), free_count.data_ptr(), block_table.data_ptr(), _at(row_idx),
                            _at(batch_count), _at(new_lens), out.slot_map.data_ptr(), out.positions.data_ptr(),
                            out.cu_tokens.data_ptr(), out.granted.data_ptr(), out.lens.data_ptr(), out.free_count.data_ptr(),
                            block_table.stride(0), rows, free_pages.numel(), batch, max_tokens)
        st = self._lib.fi_pages_extend(self._h, args, _raw_stream(index))
        if st:
            _check(st)
        return out

    # -- fi_pages_release
    def release(self, row_idx: torch.Tensor, lens: torch.Tensor, free_pages: torch.Tensor, free_count: torch.Tensor,
                block_table: torch.Tensor, *, batch_count: Optional[torch.Tensor] = None,
                out: Optional[Sequence[torch.Tensor]] = None):
        """Gives the pages of the listed rows back (free_pages is written in place); returns (lens, free_count) after it.  `out` may be
        (lens, free_count) themselves."""
        rows, index = self._check_state(lens, free_pages, free_count, block_table), self._index
        _check_flat(row_idx, "row_idx", index)
        _check_flat(batch_count, "batch_count", index, 1)
        if out is None:
            out = torch.empty(rows + 1, dtype=torch.int32, device=self.device).split_with_sizes([rows, 1])
        lens_out, count_out = out
        _check_flat(lens_out, "out[0]", index, rows)
        _check_flat(count_out, "out[1]", index, 1)
        st = self._lib.fi_pages_release(self._h, row_idx.data_ptr(), row_idx.numel(), _at(batch_count), lens.data_ptr(), rows,
                                        block_table.data_ptr(), block_table.stride(0), free_pages.data_ptr(), free_pages.numel(),
                                        free_count.data_ptr(), lens_out.data_ptr(), count_out.data_ptr(), _raw_stream(index))
        if st:
            _check(st)
        return lens_out, count_out


def _norm_rope_call(fn, q, k, q_weight, k_weight, rope, positions, eps, interleaved, count, q_res, k_res, dq_out=None,
                    dk_out=None, dq_weight=None, dk_weight=None, workspace=None):
    """Checks and packs the arguments of both directions; makes the results (q_res, k_res) that are not given."""
    dtype, index = q.dtype, q.get_device()
    if dtype not in _FI_DTYPE or q.dim() != 3 or index < 0:
        raise ValueError("q must be a float32 or bfloat16 [tokens, heads, head_dim] tensor on a GPU")
    tokens, q_heads, dim = q.shape
    strides = _check_heads(q, "q", index, dtype, tokens, q_heads, dim)
    if q_res is None:
        q_res = torch.empty_like(q)
        res_strides = q_res.stride()[:2]
    else:
        res_strides = _check_heads(q_res, "result for q", index, dtype, tokens, q_heads, dim)
    k_heads, k_strides, k_res_strides, dk_strides = 0, (0, 0), (0, 0), (0, 0)
    if k is not None:
        k_heads = k.size(1) if k.dim() == 3 else 0
        k_strides = _check_heads(k, "k", index, dtype, tokens, k_heads, dim)
        if k_res is None:
            k_res = torch.empty_like(k)
            k_res_strides = k_res.stride()[:2]
        else:
            k_res_strides = _check_heads(k_res, "result for k", index, dtype, tokens, k_heads, dim)
    else:
        k_res = None
    dq_strides = (0, 0)
    if dq_out is not None:
        dq_strides = _check_heads(dq_out, "dq_out", index, dtype, tokens, q_heads, dim)
        if k is not None:
            dk_strides = _check_heads(dk_out, "dk_out", index, dtype, tokens, k_heads, dim)
    _check_flat(q_weight, "q_weight", index, dim, torch.float32)
    _check_flat(k_weight, "k_weight", index, dim, torch.float32)
    max_pos = rot = 0
    if rope is not None:
        if positions is None or rope.dim() != 2:
            raise ValueError("rope must be [max_pos, rot_dim], and needs positions")
        _check_flat(rope, "rope", index, 0, torch.float32)
        _check_flat(positions, "positions", index, tokens)
        max_pos, rot = rope.shape
    _check_flat(count, "count", index, 1)
    args = _pack_norm(q.data_ptr(), _at(k), q_res.data_ptr(), _at(k_res), _at(dq_out), _at(dk_out), _at(q_weight), _at(k_weight),
                      _at(rope), _at(positions), _at(count), _at(dq_weight), _at(dk_weight), _at(workspace), *strides, *k_strides,
                      *res_strides, *k_res_strides, *dq_strides, *dk_strides, tokens, q_heads, k_heads, dim, rot, max_pos,
                      1 if interleaved else 0, _FI_DTYPE[dtype], eps)
    if _current_device() == index:
        st = fn(args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            st = fn(args, _raw_stream(index))
    if st:
        _check(st)
    return q_res, k_res


def head_norm_rope(q: torch.Tensor, k: Optional[torch.Tensor], q_weight: Optional[torch.Tensor],
                   k_weight: Optional[torch.Tensor], rope: Optional[torch.Tensor], positions: Optional[torch.Tensor], *,
                   eps: float = 1e-6, interleaved: bool = False, count: Optional[torch.Tensor] = None,
                   q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
    """fi_head_norm_rope: (q, k) normed head by head and turned to their positions.  q_out / k_out may be q / k.  Gradients flow to
    q, k and the weights; results that are given have none, so they are refused where one is asked for."""
    if (q.requires_grad or k is not None and k.requires_grad or q_weight is not None and q_weight.requires_grad
            or k_weight is not None and k_weight.requires_grad) and torch.is_grad_enabled():
        if q_out is not None or k_out is not None:
            raise ValueError("q_out and k_out are given, but a gradient is asked for")
        return _HeadNormRope.apply(q, k, q_weight, k_weight, rope, positions, eps, interleaved, count)
    return _norm_rope_call(load_library().fi_head_norm_rope, q, k, q_weight, k_weight, rope, positions, eps, interleaved, count,
                           q_out, k_out)


def head_norm_rope_backward(q: torch.Tensor, k: Optional[torch.Tensor], q_weight: Optional[torch.Tensor],
                            k_weight: Optional[torch.Tensor], rope: Optional[torch.Tensor], positions: Optional[torch.Tensor],
                            dq_out: torch.Tensor, dk_out: Optional[torch.Tensor], *, eps: float = 1e-6,
                            interleaved: bool = False, count: Optional[torch.Tensor] = None,
                            dq: Optional[torch.Tensor] = None, dk: Optional[torch.Tensor] = None):
    """fi_head_norm_rope_backward: (dq, dk, dq_weight, dk_weight) from the forward pass's inputs and the gradients of its
    results.  The gradient of a weight that is None is None."""
    lib = load_library()
    dim = q.shape[-1]
    dqw = q_weight.new_empty(dim) if q_weight is not None else None
    dkw = k_weight.new_empty(dim) if k_weight is not None and k is not None else None
    work = None
    if dqw is not None or dkw is not None:
        work = torch.empty(lib.fi_head_norm_rope_workspace(dim), dtype=torch.uint8, device=q.device)
    if dq_out is None or (k is not None and dk_out is None):
        raise ValueError("the gradients of the results are needed")
    dq, dk = _norm_rope_call(lib.fi_head_norm_rope_backward, q, k, q_weight, k_weight, rope, positions, eps, interleaved, count,
                             dq, dk, dq_out, dk_out, dqw, dkw, work)
    return dq, dk, dqw, dkw


def _as_heads(t: torch.Tensor) -> torch.Tensor:
    """t, or a copy that the kernels read: values of a head side by side, heads on 16-byte boundaries."""
    unit = 16 // t.element_size()
    ok = t.stride(2) == 1 and t.data_ptr() % 16 == 0 and t.stride(0) % unit == 0 and t.stride(1) % unit == 0
    return t if ok else t.clone(memory_format=torch.contiguous_format)


class _HeadNormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, rope, positions, eps, interleaved, count):
        ctx.save_for_backward(q, k, q_weight, k_weight, rope, positions, count)
        ctx.eps, ctx.interleaved = eps, interleaved
        return _norm_rope_call(load_library().fi_head_norm_rope, q, k, q_weight, k_weight, rope, positions, eps, interleaved, count,
                               None, None)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dq_out, dk_out):
        q, k, q_weight, k_weight, rope, positions, count = ctx.saved_tensors
        # tokens past the count have no gradient, and the kernel leaves them alone
        dq, dk = (None if t is None or count is None else torch.zeros_like(t) for t in (q, k))
        dq, dk, dqw, dkw = head_norm_rope_backward(q, k, q_weight, k_weight, rope, positions, _as_heads(dq_out),
                                                   None if k is None else _as_heads(dk_out), eps=ctx.eps,
                                                   interleaved=ctx.interleaved, count=count, dq=dq, dk=dk)
        dqw, dkw = (None if d is None else d.view_as(w) for d, w in ((dqw, q_weight), (dkw, k_weight)))
        return dq, dk, dqw, dkw, None, None, None, None, None


class KvCache:
    """Keys and values of one layer in 4 bits (fi_kv_*) over pools the caller owns: codes uint8 [pages, kv_heads, page_size,
    head_dim / 2], meta bfloat16 [pages, kv_heads, page_size, 2] (scale, offset).  For inference: the calls give no gradients.
    Attention calls of one object share its scratch: they belong on one stream."""

    def __init__(self, k_codes: torch.Tensor, k_meta: torch.Tensor, v_codes: torch.Tensor, v_meta: torch.Tensor, *, q_heads: int):
        self._lib = load_library()
        self._h = ctypes.c_void_p()
        dev = k_codes.device
        if k_codes.dim() != 4 or dev.type != "cuda":
            raise ValueError("k_codes must be uint8 [pages, kv_heads, page_size, head_dim / 2] on a GPU")
        pages, heads, page, half = k_codes.shape
        for codes, meta in ((k_codes, k_meta), (v_codes, v_meta)):
            if codes.dtype != torch.uint8 or codes.shape != k_codes.shape or codes.device != dev or codes.stride() != k_codes.stride() \
                    or codes.stride(3) != 1:
                raise ValueError("codes must be uint8 tensors of one shape and layout, bytes of a vector side by side")
            if meta.dtype != torch.bfloat16 or tuple(meta.shape) != (pages, heads, page, 2) or meta.device != dev \
                    or meta.stride() != k_meta.stride() or meta.stride(3) != 1 or any(s % 2 for s in meta.stride()[:3]):
                raise ValueError("meta must be bfloat16 [pages, kv_heads, page_size, 2] tensors of one layout, pairs side by side")
        self.k_codes, self.k_meta, self.v_codes, self.v_meta = k_codes, k_meta, v_codes, v_meta   # kept alive
        self.device, self._index = dev, k_codes.get_device()
        self.pages, self.kv_heads, self.page_size, self.head_dim = pages, heads, page, 2 * half
        self.q_heads = q_heads
        cs, ms = k_codes.stride(), k_meta.stride()
        cfg = fi_kv_config_t(_dp(k_codes), _dp(v_codes), _dp(k_meta), _dp(v_meta), cs[0], cs[1], cs[2], ms[0] // 2, ms[1] // 2,
                             ms[2] // 2, pages, page, q_heads, heads, 2 * half, self._index)
        _check(self._lib.fi_kv_create(ctypes.byref(cfg), ctypes.byref(self._h)))

    # -- fi_kv_destroy
    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h.value:
            self._lib.fi_kv_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- fi_kv_set_wait_limit
    def set_wait_limit(self, limit_cycles: int = 0) -> None:
        """Limit of the waits inside attend's kernels in SM cycles (0: the default); past it the next poll_status() raises
        FI_ERR_TIMEOUT."""
        _check(self._lib.fi_kv_set_wait_limit(self._h, int(limit_cycles)))

    # -- fi_kv_poll_status
    def poll_status(self) -> None:
        _check(self._lib.fi_kv_poll_status(self._h))

    # -- fi_kv_append
    def append(self, k: torch.Tensor, v: torch.Tensor, slot_map: torch.Tensor, *, count: Optional[torch.Tensor] = None,
               with_stored: bool = False):
        """Stores keys and values [tokens, kv_heads, head_dim] at their slots; with with_stored returns what the codes stand
        for, in k's dtype."""
        tokens, index, dtype = k.size(0), self._index, k.dtype
        kind = _FI_DTYPE.get(dtype)
        if kind is None:
            raise ValueError("k must be float32 or bfloat16")
        k_token, k_head = _check_heads(k, "k", index, dtype, tokens, self.kv_heads, self.head_dim)
        v_token, v_head = _check_heads(v, "v", index, dtype, tokens, self.kv_heads, self.head_dim)
        _check_flat(slot_map, "slot_map", index, tokens, torch.int64)
        _check_flat(count, "count", index, 1)
        ks = vs = None
        if with_stored:
            ks, vs = k.new_empty((2, tokens, self.kv_heads, self.head_dim)).unbind(0)
        st = self._lib.fi_kv_append(self._h, _pack_append(k.data_ptr(), v.data_ptr(), slot_map.data_ptr(), _at(count), _at(ks),
                                                          _at(vs), k_token, k_head, v_token, v_head, tokens, kind),
                                    _raw_stream(index))
        if st:
            _check(st)
        return (ks, vs) if with_stored else None

    # -- fi_kv_attend
    def attend(self, q: torch.Tensor, lens: torch.Tensor, block_table: torch.Tensor, *, cu_tokens: Optional[torch.Tensor] = None,
               row_idx: Optional[torch.Tensor] = None, batch_count: Optional[torch.Tensor] = None, max_query: int = 1,
               window: int = 0, scale: Optional[float] = None, out: Optional[torch.Tensor] = None, with_lse: bool = False,
               lse: Optional[torch.Tensor] = None, granted: Optional[torch.Tensor] = None):
        """Attention of q [tokens, q_heads, head_dim] (the last tokens of each request, which are stored already) over the
        stored keys and values; scale defaults to 1 / sqrt(head_dim).  Requests that KvTables.extend refused get zeros when its
        `granted` is given.  Returns out, or (out, lse)."""
        tokens, index, dtype, heads, dim = q.size(0), self._index, q.dtype, self.q_heads, self.head_dim
        kind = _FI_DTYPE.get(dtype)
        if kind is None:
            raise ValueError("q must be float32 or bfloat16")
        q_token, q_head = _check_heads(q, "q", index, dtype, tokens, heads, dim)
        _check_flat(lens, "lens", index)
        rows = lens.numel()
        _check_table(block_table, rows, 0, index)
        batch = rows
        if row_idx is not None:
            _check_flat(row_idx, "row_idx", index)
            batch = row_idx.numel()
        _check_flat(batch_count, "batch_count", index, 1)
        _check_flat(cu_tokens, "cu_tokens", index, batch + 1)
        _check_flat(granted, "granted", index, batch)
        if out is None:
            out = torch.empty_like(q)
            out_token, out_head, _ = out.stride()
        else:
            out_token, out_head = _check_heads(out, "out", index, dtype, tokens, heads, dim)
        if lse is not None:
            _check_flat(lse, "lse", index, tokens * heads, torch.float32)
        elif with_lse:
            lse = q.new_empty((tokens, heads), dtype=torch.float32)
        st = self._lib.fi_kv_attend(self._h, _pack_attend(
            q.data_ptr(), out.data_ptr(), _at(lse), lens.data_ptr(), block_table.data_ptr(), _at(row_idx), _at(batch_count),
            _at(cu_tokens), _at(granted), q_token, q_head, out_token, out_head, block_table.stride(0), rows, block_table.size(1), batch, tokens,
            max_query, window, kind, dim ** -0.5 if scale is None else scale), _raw_stream(index))
        if st:
            _check(st)
        return out if lse is None else (out, lse)
