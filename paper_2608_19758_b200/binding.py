"""ctypes binding of libfp2.so: argument marshalling only (every step of the path runs in the CUDA kernels).

The functions carry the names of the C ABI (include/fp2.h).  torch is used for device memory and streams.
There is no CPU fallback: if the library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import torch

from . import build as _build

FP2_OK = 0
STATUS_NAMES = {0: "FP2_OK", 1: "FP2_ERR_INVALID_ARG", 2: "FP2_ERR_UNSUPPORTED", 3: "FP2_ERR_CAPACITY",
                4: "FP2_ERR_CUDA", 5: "FP2_ERR_TIMEOUT"}

EXPORTS = ["fp2_plan_create", "fp2_plan_sizes", "fp2_plan_destroy", "fp2_plan_segment", "fp2_select_blocks",
           "fp2_pool_blocks",
           "fp2_sparse_prefill", "fp2_dense_prefill", "fp2_dense_prefill_static", "fp2_export_csr",
           "fp2_page_table_from_token_map", "fp2_plan_set_split", "fp2_pool_carry", "fp2_pool_carry_count",
           "fp2_read_status", "fp2_selftest_bounded_wait", "fp2_last_launch_count", "fp2_status_string",
           "fp2_window_prefill", "fp2_cache_create", "fp2_cache_destroy", "fp2_cache_sizes", "fp2_cache_append", "fp2_cache_expand", "fp2_decode",
           "fp2_cache_read_status"]


class Fp2Error(RuntimeError):
    def __init__(self, code: int, where: str):
        super().__init__(f"{where}: {STATUS_NAMES.get(code, code)}")
        self.code = code


class fp2_params(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("num_seqs", "total_q", "num_q_heads", "num_kv_heads", "head_dim",
                                         "block_size", "tile_rows", "page_size", "num_pages", "max_pages_per_seq",
                                         "sink_tokens", "window_tokens", "use_correction")] + \
               [("alpha", C.c_float), ("softmax_scale", C.c_float), ("dtype", C.c_int32)]


CACHE_BF16, CACHE_FP8_HEAD, CACHE_FP8_PAGE = 0, 1, 2     # fp2_cache_format


class fp2_cache_params(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("max_seqs", "num_q_heads", "num_kv_heads", "head_dim", "page_size", "num_pages",
                                         "max_pages_per_seq", "format")] + [("softmax_scale", C.c_float)]


_lib = None


def lib_path() -> str:
    return _build.LIB


def load(build_if_missing: bool = True) -> C.CDLL:
    """Loads (building first if the sources are newer) the shared library; raises if that is impossible."""
    global _lib
    if _lib is not None:
        return _lib
    if build_if_missing and _build.needs_build():
        _build.build()
    if not os.path.exists(_build.LIB):
        raise RuntimeError("libfp2.so is missing: run `python -m paper_2608_19758_b200.build`")
    lib = C.CDLL(_build.LIB)
    vp, i32p, i64p, f32p = C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p
    lib.fp2_plan_create.argtypes = [C.POINTER(fp2_params), C.POINTER(C.c_int32), C.POINTER(C.c_int32),
                                    C.POINTER(C.c_void_p)]
    lib.fp2_plan_create.restype = C.c_int
    lib.fp2_plan_sizes.argtypes = [C.c_void_p, C.POINTER(C.c_int64), C.POINTER(C.c_int64), C.POINTER(C.c_int64)]
    lib.fp2_plan_sizes.restype = C.c_int
    lib.fp2_plan_destroy.argtypes = [C.c_void_p]
    lib.fp2_plan_destroy.restype = None
    lib.fp2_plan_segment.argtypes = [C.c_void_p, C.c_int64, C.POINTER(C.c_int32), C.POINTER(C.c_int64)]
    lib.fp2_plan_segment.restype = C.c_int
    lib.fp2_select_blocks.argtypes = [C.c_void_p, vp, vp, vp, i32p, i32p, i32p, f32p, f32p, f32p, i64p, i32p, i32p,
                                      vp, C.c_void_p]
    lib.fp2_select_blocks.restype = C.c_int
    lib.fp2_pool_blocks.argtypes = [C.c_void_p, vp, vp, i32p, i32p, f32p, f32p, vp, C.c_void_p]
    lib.fp2_pool_blocks.restype = C.c_int
    lib.fp2_sparse_prefill.argtypes = [C.c_void_p, vp, vp, vp, i32p, i32p, i32p, i64p, i32p, i32p, f32p, f32p, f32p,
                                       vp, f32p, vp, C.c_int32, C.c_void_p]
    lib.fp2_sparse_prefill.restype = C.c_int
    lib.fp2_dense_prefill.argtypes = [C.c_void_p, vp, vp, vp, i32p, i32p, i32p, f32p, f32p, f32p, vp, f32p, vp,
                                      C.c_void_p]
    lib.fp2_dense_prefill.restype = C.c_int
    lib.fp2_dense_prefill_static.argtypes = [C.c_void_p, vp, vp, vp, i32p, i32p, i32p, f32p, f32p, f32p, vp, f32p,
                                             C.c_void_p]
    lib.fp2_dense_prefill_static.restype = C.c_int
    lib.fp2_window_prefill.argtypes = [C.c_void_p, vp, vp, vp, i32p, i32p, i32p, f32p, f32p, f32p, C.c_int32, C.c_int32, vp, f32p,
                                       vp, C.c_void_p]
    lib.fp2_window_prefill.restype = C.c_int
    lib.fp2_export_csr.argtypes = [C.c_void_p, i32p, i32p, C.c_int32, i32p, i32p, C.c_int64, vp, C.c_void_p]
    lib.fp2_export_csr.restype = C.c_int
    lib.fp2_page_table_from_token_map.argtypes = [C.c_void_p, i32p, C.c_int32, i32p, i32p, vp, C.c_void_p]
    lib.fp2_page_table_from_token_map.restype = C.c_int
    lib.fp2_pool_carry.argtypes = [C.c_void_p, vp, C.c_void_p, vp, C.POINTER(C.c_int32), C.c_void_p]
    lib.fp2_pool_carry.restype = C.c_int
    lib.fp2_pool_carry_count.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
    lib.fp2_pool_carry_count.restype = C.c_int
    lib.fp2_plan_set_split.argtypes = [C.c_void_p, C.c_int32]
    lib.fp2_plan_set_split.restype = C.c_int
    lib.fp2_selftest_bounded_wait.argtypes = [C.c_void_p, vp, C.c_void_p]
    lib.fp2_selftest_bounded_wait.restype = C.c_int
    lib.fp2_read_status.argtypes = [C.c_void_p, vp, C.POINTER(C.c_int32), C.c_void_p]
    lib.fp2_read_status.restype = C.c_int
    lib.fp2_last_launch_count.argtypes = [C.c_void_p]
    lib.fp2_last_launch_count.restype = C.c_int32
    lib.fp2_cache_create.argtypes = [C.POINTER(fp2_cache_params), C.POINTER(C.c_void_p)]
    lib.fp2_cache_create.restype = C.c_int
    lib.fp2_cache_destroy.argtypes = [C.c_void_p]
    lib.fp2_cache_destroy.restype = None
    lib.fp2_cache_sizes.argtypes = [C.c_void_p, C.POINTER(C.c_int64)]
    lib.fp2_cache_sizes.restype = C.c_int
    lib.fp2_cache_append.argtypes = [C.c_void_p, vp, vp, C.c_int64, i32p, i32p, i32p, C.c_int32, C.c_int32, vp, vp, f32p, f32p,
                                     vp, C.c_void_p]
    lib.fp2_cache_append.restype = C.c_int
    lib.fp2_cache_expand.argtypes = [C.c_void_p, vp, vp, i32p, i32p, C.c_int32, f32p, f32p, vp, vp, i32p, C.c_int32, vp,
                                     C.c_void_p]
    lib.fp2_cache_expand.restype = C.c_int
    lib.fp2_decode.argtypes = [C.c_void_p, vp, C.c_int64, vp, vp, i32p, i32p, i32p, C.c_int32, C.c_int32, f32p, f32p, C.c_int32,
                               C.c_int32, vp, f32p, vp, C.c_void_p]
    lib.fp2_decode.restype = C.c_int
    lib.fp2_cache_read_status.argtypes = [C.c_void_p, vp, C.POINTER(C.c_int32), C.c_void_p]
    lib.fp2_cache_read_status.restype = C.c_int
    lib.fp2_status_string.argtypes = [C.c_int]
    lib.fp2_status_string.restype = C.c_char_p
    _lib = lib
    return lib


def _check(code: int, where: str):
    if code != FP2_OK:
        raise Fp2Error(code, where)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()     # ctypes takes a plain integer for a void pointer


# The current stream's handle without a Stream object around it (4.3 us per stage call, of 11 to 15 us on the host).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None and torch.cuda.is_initialized():
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def fp2_status_string(code: int) -> str:
    return load().fp2_status_string(code).decode()


class Plan:
    """Owner of an fp2_plan handle (host-side metadata + one small device table)."""

    def __init__(self, params: dict, h_cu_seqlens_q, h_seqlens_k):
        lib = load()
        self.params = fp2_params(**params)
        ns = int(params["num_seqs"])
        cu = (C.c_int32 * (ns + 1))(*[int(x) for x in h_cu_seqlens_q])
        lk = (C.c_int32 * ns)(*[int(x) for x in h_seqlens_k])
        h = C.c_void_p()
        _check(lib.fp2_plan_create(C.byref(self.params), cu, lk, C.byref(h)), "fp2_plan_create")
        self.handle = h
        a, b, c = C.c_int64(), C.c_int64(), C.c_int64()
        _check(lib.fp2_plan_sizes(h, C.byref(a), C.byref(b), C.byref(c)), "fp2_plan_sizes")
        self.num_segments, self.idx_capacity, self.workspace_bytes = a.value, b.value, c.value
        p = self.params
        self._window_sizes = (p.total_q * p.num_q_heads * 128, p.num_pages * p.page_size * p.num_kv_heads * 128,
                              (p.num_seqs, p.max_pages_per_seq), (p.num_q_heads, p.total_q), p.num_q_heads if p.dtype else 0,
                              p.num_kv_heads, _E4M3 if p.dtype else _BF16)

    def segment(self, seg: int) -> dict:
        out = (C.c_int32 * 10)()
        off = C.c_int64()
        _check(load().fp2_plan_segment(self.handle, seg, out, C.byref(off)), "fp2_plan_segment")
        keys = ("b", "h", "t", "r0", "nrows", "pre", "Lk", "J_lo", "J_hi", "blk_off")
        d = dict(zip(keys, list(out)))
        d["off"] = off.value
        return d

    def set_split(self, target: int):
        """KV splitting (Eq. 18): < 0 off, 0 automatic, > 0 requested iterations per part."""
        _check(load().fp2_plan_set_split(self.handle, target), "fp2_plan_set_split")

    def last_launch_count(self) -> int:
        return int(load().fp2_last_launch_count(self.handle))

    def new_workspace(self, device="cuda") -> torch.Tensor:
        """Zeroed device workspace (torch's allocator returns 512-byte aligned blocks; 1024 is required,
        so over-allocate and slice)."""
        raw = torch.zeros(self.workspace_bytes + 1024, dtype=torch.uint8, device=device)
        shift = (-raw.data_ptr()) % 1024
        ws = raw[shift:shift + self.workspace_bytes]
        ws._fp2_keepalive = raw
        return ws

    def new_lists(self, device="cuda"):
        seg_offset = torch.zeros(self.num_segments + 1, dtype=torch.int64, device=device)
        seg_count = torch.zeros(max(self.num_segments, 1), dtype=torch.int32, device=device)
        blk_idx = torch.zeros(max(self.idx_capacity, 1), dtype=torch.int32, device=device)
        return seg_offset, seg_count, blk_idx

    def close(self):
        if getattr(self, "handle", None):
            load().fp2_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def fp2_select_blocks(plan: Plan, q, k_cache, v_cache, page_table, cu_seqlens_q, seqlens_k, q_scale, k_scale,
                      v_scale, seg_offset, seg_count, blk_idx, workspace, stream=None):
    _check(load().fp2_select_blocks(plan.handle, _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(page_table),
                                    _ptr(cu_seqlens_q), _ptr(seqlens_k), _ptr(q_scale), _ptr(k_scale),
                                    _ptr(v_scale), _ptr(seg_offset), _ptr(seg_count), _ptr(blk_idx),
                                    _ptr(workspace), _stream(stream)), "fp2_select_blocks")


def fp2_pool_blocks(plan: Plan, k_cache, v_cache, page_table, seqlens_k, k_scale, v_scale, workspace, stream=None):
    """Block-mean pooling alone: the pooled statistics of `workspace` are refreshed, no list is written."""
    _check(load().fp2_pool_blocks(plan.handle, _ptr(k_cache), _ptr(v_cache), _ptr(page_table), _ptr(seqlens_k),
                                  _ptr(k_scale), _ptr(v_scale), _ptr(workspace), _stream(stream)), "fp2_pool_blocks")


def fp2_sparse_prefill(plan: Plan, q, k_cache, v_cache, page_table, cu_seqlens_q, seqlens_k, seg_offset, seg_count,
                       blk_idx, q_scale, k_scale, v_scale, out, lse, workspace, pooled_valid: bool = True,
                       stream=None):
    _check(load().fp2_sparse_prefill(plan.handle, _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(page_table),
                                     _ptr(cu_seqlens_q), _ptr(seqlens_k), _ptr(seg_offset), _ptr(seg_count),
                                     _ptr(blk_idx), _ptr(q_scale), _ptr(k_scale), _ptr(v_scale), _ptr(out),
                                     _ptr(lse), _ptr(workspace), 1 if pooled_valid else 0, _stream(stream)),
           "fp2_sparse_prefill")


def fp2_dense_prefill(plan: Plan, q, k_cache, v_cache, page_table, cu_seqlens_q, seqlens_k, q_scale, k_scale,
                      v_scale, out, lse, workspace, stream=None):
    _check(load().fp2_dense_prefill(plan.handle, _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(page_table),
                                    _ptr(cu_seqlens_q), _ptr(seqlens_k), _ptr(q_scale), _ptr(k_scale),
                                    _ptr(v_scale), _ptr(out), _ptr(lse), _ptr(workspace), _stream(stream)),
           "fp2_dense_prefill")


def _check_window(plan, q, k_cache, v_cache, page_table, q_scale, k_scale, v_scale, out, lse, workspace):
    """What fp2_window_prefill reads and writes must be what the plan takes its address for; more elements may follow behind.  (Looked
    at in one expression, which is a microsecond, and again one by one only to say what is wrong.)"""
    q_size, pool, pt_shape, lse_shape, heads, kv_heads, kinds = plan._window_sizes
    dev = torch.cuda.current_device() if torch.cuda.is_initialized() or torch.cuda.is_available() else -1
    try:
        fits = (q.dtype in kinds and q.numel() >= q_size and q.get_device() == dev and q.is_contiguous() and
                k_cache.dtype in kinds and k_cache.numel() >= pool and k_cache.get_device() == dev and k_cache.is_contiguous() and
                v_cache.dtype in kinds and v_cache.numel() >= pool and v_cache.get_device() == dev and v_cache.is_contiguous() and
                out.dtype is torch.bfloat16 and out.numel() >= q_size and out.get_device() == dev and out.is_contiguous() and
                page_table.dtype is torch.int32 and page_table.shape == pt_shape and page_table.get_device() == dev and
                page_table.is_contiguous() and workspace.nbytes >= plan.workspace_bytes and workspace.get_device() == dev and
                (lse is None or lse.dtype is torch.float32 and lse.shape == lse_shape and lse.get_device() == dev and
                 lse.is_contiguous()))
        if heads:                       # FP8
            fits = (fits and q_scale.dtype is torch.float32 and q_scale.numel() >= heads and q_scale.get_device() == dev and
                    q_scale.is_contiguous() and k_scale.dtype is torch.float32 and k_scale.numel() >= kv_heads and
                    k_scale.get_device() == dev and k_scale.is_contiguous() and v_scale.dtype is torch.float32 and
                    v_scale.numel() >= kv_heads and v_scale.get_device() == dev and v_scale.is_contiguous())
    except AttributeError:              # None
        fits = False
    if fits:
        return
    where = "fp2_window_prefill"
    _room(where, dev, q, kinds, q_size)
    _room(where, dev, k_cache, kinds, pool)
    _room(where, dev, v_cache, kinds, pool)
    _room(where, dev, out, _BF16, q_size)
    _room(where, dev, page_table, _I32, pt_shape[0] * pt_shape[1])
    if page_table.dim() > 1 and page_table.shape[-1] != pt_shape[1]:           # (more sequences may follow, rows be no longer)
        _want(where, dev, page_table, _I32, pt_shape)
    if lse is not None:
        _want(where, dev, lse, _F32, lse_shape)
    for scale, n in ((q_scale, heads), (k_scale, kv_heads), (v_scale, kv_heads)) if heads else ():
        _room(where, dev, scale, _F32, n)
    if workspace is None or workspace.nbytes < plan.workspace_bytes or workspace.get_device() != dev:
        raise Fp2Error(1, f"{where}: workspace too small or not on device {dev}")


def fp2_window_prefill(plan: Plan, q, k_cache, v_cache, page_table, cu_seqlens_q, seqlens_k, q_scale, k_scale, v_scale,
                       window_tokens: int, sink_tokens: int, out, lse, workspace, stream=None):
    """Causal attention with a sliding window of `window_tokens` and the first `sink_tokens` tokens always visible."""
    _check_window(plan, q, k_cache, v_cache, page_table, q_scale, k_scale, v_scale, out, lse, workspace)
    _check(load().fp2_window_prefill(plan.handle, _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(page_table),
                                     _ptr(cu_seqlens_q), _ptr(seqlens_k), _ptr(q_scale), _ptr(k_scale), _ptr(v_scale),
                                     window_tokens, sink_tokens, _ptr(out), _ptr(lse), _ptr(workspace), _stream(stream)),
           "fp2_window_prefill")


def fp2_dense_prefill_static(plan: Plan, q, k_cache, v_cache, page_table, cu_seqlens_q, seqlens_k, q_scale, k_scale,
                             v_scale, out, lse, stream=None):
    """Dense prefill without a caller workspace: the library's built-in device scratch is used."""
    _check(load().fp2_dense_prefill_static(plan.handle, _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(page_table),
                                           _ptr(cu_seqlens_q), _ptr(seqlens_k), _ptr(q_scale), _ptr(k_scale),
                                           _ptr(v_scale), _ptr(out), _ptr(lse), _stream(stream)),
           "fp2_dense_prefill_static")


def fp2_export_csr(plan: Plan, seg_count, blk_idx, tile_tokens: int, cu, idx, workspace, stream=None):
    """Compact CSR of physical tiles (cu int32 [nseg + 1], idx int32) from the padded block lists."""
    _check(load().fp2_export_csr(plan.handle, _ptr(seg_count), _ptr(blk_idx), tile_tokens, _ptr(cu), _ptr(idx),
                                 idx.numel(), _ptr(workspace), _stream(stream)), "fp2_export_csr")


def fp2_page_table_from_token_map(plan: Plan, token_to_slot, seqlens_k, page_table, workspace, stream=None):
    """Page-level table [num_seqs, max_pages_per_seq] from a token-level slot map [num_seqs, max_tokens]."""
    _check(load().fp2_page_table_from_token_map(plan.handle, _ptr(token_to_slot), token_to_slot.shape[1],
                                                _ptr(seqlens_k), _ptr(page_table), _ptr(workspace),
                                                _stream(stream)), "fp2_page_table_from_token_map")


def fp2_pool_carry_count(dst: Plan, src: Plan, src_seq):
    """Blocks per sequence of `dst` whose pooled means would be carried over from `src` (host only)."""
    ns = len(src_seq)
    a = (C.c_int32 * max(ns, 1))(*src_seq)
    out = (C.c_int32 * max(ns, 1))()
    _check(load().fp2_pool_carry_count(dst.handle, src.handle, a, out), "fp2_pool_carry_count")
    return list(out)[:ns]


def fp2_pool_carry(dst: Plan, dst_workspace, src: Plan, src_workspace, src_seq, stream=None):
    """Copies the pooled means of the blocks complete in both chunks from src_workspace to dst_workspace; the next
    fp2_select_blocks on `dst` pools only the rest."""
    a = (C.c_int32 * max(len(src_seq), 1))(*src_seq)
    _check(load().fp2_pool_carry(dst.handle, _ptr(dst_workspace), src.handle, _ptr(src_workspace), a,
                                 _stream(stream)), "fp2_pool_carry")


def fp2_selftest_bounded_wait(plan: Plan, workspace, stream=None):
    """Launches the library's bounded-wait probe: a wait that runs out, recorded in the status block of `workspace`."""
    _check(load().fp2_selftest_bounded_wait(plan.handle, _ptr(workspace), _stream(stream)), "fp2_selftest_bounded_wait")


class Cache:
    """Owner of an fp2_cache handle: the shapes and the format of a paged KV cache (host memory only)."""

    def __init__(self, params: dict):
        lib = load()
        self.params = fp2_cache_params(**params)
        h = C.c_void_p()
        _check(lib.fp2_cache_create(C.byref(self.params), C.byref(h)), "fp2_cache_create")
        self.handle = h
        n = C.c_int64()
        _check(lib.fp2_cache_sizes(h, C.byref(n)), "fp2_cache_sizes")
        self.workspace_bytes = n.value
        self._device = torch.cuda.current_device() if torch.cuda.is_available() else -1
        p = self.params
        self._fp8 = p.format != CACHE_BF16
        self._kinds = _E4M3 if self._fp8 else _BF16
        self._max_pages, self._q_heads = p.max_pages_per_seq, p.num_q_heads
        self._pool = (p.num_pages, p.page_size, p.num_kv_heads, p.head_dim)
        self._scales = {CACHE_BF16: None, CACHE_FP8_HEAD: (p.num_kv_heads,), CACHE_FP8_PAGE: (p.num_pages, p.num_kv_heads)}[p.format]

    def new_workspace(self, device="cuda") -> torch.Tensor:
        """Zeroed device workspace, 1024-byte aligned (one per stream that runs calls at the same time)."""
        raw = torch.zeros(self.workspace_bytes + 1024, dtype=torch.uint8, device=device)
        shift = (-raw.data_ptr()) % 1024
        ws = raw[shift:shift + self.workspace_bytes]
        ws._fp2_keepalive = raw
        return ws

    def new_pages(self, device="cuda"):
        """Zeroed k_cache, v_cache, k_scale, v_scale of the cache's shapes (scales one; None for BF16)."""
        dt = torch.uint8 if self._fp8 else torch.bfloat16
        k, v = (torch.zeros(self._pool, dtype=dt, device=device) for _ in "kv")
        if self._scales is None:
            return k, v, None, None
        ks, vs = (torch.ones(self._scales, dtype=torch.float32, device=device) for _ in "kv")
        return k, v, ks, vs

    def _check_pages(self, where, k_cache, v_cache, k_scale, v_scale, page_table, seqlens_k, num_seqs, workspace):
        """The tensors that all calls share; returns the device's number.  (Written out: a call per tensor is a microsecond in all,
        of the ten that a call takes on the host.)"""
        dev, pool, kinds, pt_shape = self._device, self._pool, self._kinds, (num_seqs, self._max_pages)
        if not (k_cache.dtype in kinds and k_cache.shape == pool and k_cache.get_device() == dev and k_cache.is_contiguous() and
                v_cache.dtype in kinds and v_cache.shape == pool and v_cache.get_device() == dev and v_cache.is_contiguous() and
                page_table.dtype is torch.int32 and page_table.shape == pt_shape and page_table.get_device() == dev and
                page_table.is_contiguous() and seqlens_k.dtype is torch.int32 and seqlens_k.dim() == 1 and
                seqlens_k.get_device() == dev and seqlens_k.is_contiguous()):
            _want(where, dev, k_cache, kinds, pool)
            _want(where, dev, v_cache, kinds, pool)
            _want(where, dev, page_table, _I32, pt_shape)
            _want(where, dev, seqlens_k, _I32, (num_seqs,))
        shape = self._scales
        if shape is not None and not (
                k_scale is not None and k_scale.dtype is torch.float32 and k_scale.shape == shape and k_scale.get_device() == dev and
                k_scale.is_contiguous() and v_scale is not None and v_scale.dtype is torch.float32 and v_scale.shape == shape and
                v_scale.get_device() == dev and v_scale.is_contiguous()):
            _want(where, dev, k_scale, _F32, shape)
            _want(where, dev, v_scale, _F32, shape)
        if workspace.nbytes < self.workspace_bytes or workspace.get_device() != dev:
            raise Fp2Error(1, f"{where}: workspace too small or not on device {dev}")
        return dev

    def close(self):
        if getattr(self, "handle", None):
            load().fp2_cache_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


_E4M3, _BF16, _F32, _I32 = (torch.uint8, torch.float8_e4m3fn), (torch.bfloat16,), (torch.float32,), (torch.int32,)


def _want(where, dev, t, dtypes, shape):
    """The C ABI sees addresses only: what a tensor must be for the address to mean what the call takes it for.  `dev`: the device's
    number, -1 where there is none (host memory, which no call then gets to read)."""
    if t is None or t.dtype not in dtypes or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        got = "None" if t is None else f"{t.dtype} {tuple(t.shape)} on {t.device}, strides {t.stride()}"
        raise Fp2Error(1, f"{where}: wanted contiguous {dtypes[0]} {shape} on device {dev}, got {got}")


def _room(where, dev, t, dtypes, size):
    """As _want, for a tensor that may have more elements behind those that the call takes."""
    if t is None or t.dtype not in dtypes or t.numel() < size or t.get_device() != dev or not t.is_contiguous():
        got = "None" if t is None else f"{t.dtype} {tuple(t.shape)} on {t.device}, strides {t.stride()}"
        raise Fp2Error(1, f"{where}: wanted contiguous {dtypes[0]}, {size} elements on device {dev}, got {got}")


def _rows(where, dev, t, heads):
    """Tokens and token stride of a BF16 [tokens, heads, 128] tensor whose tokens may lie apart (a slice of a fused projection)."""
    if t.dim() == 3 and t.dtype is torch.bfloat16 and t.get_device() == dev:
        tokens, h, d = t.shape
        apart, head, dim = t.stride()
        if h == heads and d == 128 and dim == 1 and (head == 128 or heads == 1):
            return tokens, apart if tokens > 1 else heads * 128
    raise Fp2Error(1, f"{where}: wanted BF16 [tokens, {heads}, 128] on device {dev}, heads next to each other, got {t.dtype} "
                      f"{tuple(t.shape)} on {t.device}, strides {t.stride()}")


def fp2_cache_append(cache: Cache, k_new, v_new, page_table, cu_seqlens_new, seqlens_k, k_cache, v_cache, k_scale, v_scale,
                     workspace, stream=None):
    """Writes the keys and values of new tokens into their pages (quantised where the cache holds 8 bits; FP8_PAGE caches get
    the pages' scales too).  seqlens_k: tokens in the cache after the call."""
    ns, where = seqlens_k.numel(), "fp2_cache_append"
    dev = cache._check_pages(where, k_cache, v_cache, k_scale, v_scale, page_table, seqlens_k, ns, workspace)
    _want(where, dev, cu_seqlens_new, _I32, (ns + 1,))
    heads = cache._pool[2]
    total, stride = rows = _rows(where, dev, k_new, heads)
    if _rows(where, dev, v_new, heads) != rows:
        raise Fp2Error(1, f"{where}: k_new and v_new differ in tokens or strides")
    _check(load().fp2_cache_append(cache.handle, _ptr(k_new), _ptr(v_new), stride, _ptr(page_table), _ptr(cu_seqlens_new),
                                   _ptr(seqlens_k), ns, total, _ptr(k_cache), _ptr(v_cache), _ptr(k_scale),
                                   _ptr(v_scale), _ptr(workspace), _stream(stream)), where)


def fp2_cache_expand(cache: Cache, k_cache, v_cache, page_table, seqlens_k, k_scale, v_scale, k_out, v_out, out_page_table,
                     workspace, stream=None):
    """An 8-bit cache as BF16 pages [out_num_pages, page_size, num_kv_heads, 128] for stage calls of a BF16 plan."""
    ns, where = seqlens_k.numel(), "fp2_cache_expand"
    dev = cache._check_pages(where, k_cache, v_cache, k_scale, v_scale, page_table, seqlens_k, ns, workspace)
    _want(where, dev, out_page_table, _I32, tuple(page_table.shape))
    pool = (k_out.shape[0],) + cache._pool[1:]
    _want(where, dev, k_out, _BF16, pool)
    _want(where, dev, v_out, _BF16, pool)
    _check(load().fp2_cache_expand(cache.handle, _ptr(k_cache), _ptr(v_cache), _ptr(page_table), _ptr(seqlens_k), ns,
                                   _ptr(k_scale), _ptr(v_scale), _ptr(k_out), _ptr(v_out), _ptr(out_page_table),
                                   k_out.shape[0], _ptr(workspace), _stream(stream)), where)


def fp2_decode(cache: Cache, q, k_cache, v_cache, page_table, cu_seqlens_q, seqlens_k, k_scale, v_scale, out, lse, workspace,
               window_tokens: int = 0, sink_tokens: int = 0, stream=None):
    """Attention of the newest few tokens of every sequence over its pages, with an optional sliding window and sinks."""
    ns, where = seqlens_k.numel(), "fp2_decode"
    dev = cache._check_pages(where, k_cache, v_cache, k_scale, v_scale, page_table, seqlens_k, ns, workspace)
    _want(where, dev, cu_seqlens_q, _I32, (ns + 1,))
    heads = cache._q_heads
    total_q, stride = _rows(where, dev, q, heads)
    _want(where, dev, out, _BF16, (total_q, heads, 128))
    if lse is not None:
        _want(where, dev, lse, _F32, (heads, total_q))
    _check(load().fp2_decode(cache.handle, _ptr(q), stride, _ptr(k_cache), _ptr(v_cache), _ptr(page_table), _ptr(cu_seqlens_q),
                             _ptr(seqlens_k), ns, total_q, _ptr(k_scale), _ptr(v_scale), window_tokens, sink_tokens, _ptr(out),
                             _ptr(lse), _ptr(workspace), _stream(stream)), where)


def fp2_cache_read_status(cache: Cache, workspace, stream=None, raise_on_error: bool = True):
    words = (C.c_int32 * 8)()
    code = load().fp2_cache_read_status(cache.handle, _ptr(workspace), words, _stream(stream))
    if raise_on_error:
        _check(code, f"fp2_cache_read_status words={list(words)}")
    return code, list(words)


def fp2_read_status(plan: Plan, workspace, stream=None, raise_on_error: bool = True):
    words = (C.c_int32 * 8)()
    code = load().fp2_read_status(plan.handle, _ptr(workspace), words, _stream(stream))
    if raise_on_error:
        _check(code, f"fp2_read_status words={list(words)}")
    return code, list(words)


class DeviceCase:
    """A workload's tensors moved to the GPU, with a plan, workspace and list buffers (test / bench helper)."""

    def __init__(self, case, device="cuda", **param_overrides):
        self.case = case
        prm = case.params()
        prm.update(param_overrides)
        self.prm = prm
        self.plan = Plan(prm, case.cu_seqlens_q.tolist(), case.seqlens_k.tolist())
        dev = torch.device(device)
        self.q = case.q.to(dev)
        self.k_cache = case.k_cache.to(dev)
        self.v_cache = case.v_cache.to(dev)
        self.page_table = case.page_table.to(dev)
        self.cu_seqlens_q = case.cu_seqlens_q.to(dev)
        self.seqlens_k = case.seqlens_k.to(dev)
        self.q_scale = None if case.q_scale is None else case.q_scale.to(dev)
        self.k_scale = None if case.k_scale is None else case.k_scale.to(dev)
        self.v_scale = None if case.v_scale is None else case.v_scale.to(dev)
        self.workspace = self.plan.new_workspace(dev)
        self.seg_offset, self.seg_count, self.blk_idx = self.plan.new_lists(dev)
        self.out = torch.empty(case.total_q, prm["num_q_heads"], prm["head_dim"], dtype=torch.bfloat16, device=dev)
        self.lse = torch.empty(prm["num_q_heads"], case.total_q, dtype=torch.float32, device=dev)
        # Tests set this: every stage call then first overwrites the buffers it is about to fill (lists with -1,
        # outputs with NaN), so that a row or an entry the call fails to write cannot pass on an earlier call's values.
        self.poison = False

    def _poison_lists(self):
        if self.poison:
            self.seg_count.fill_(-1)
            self.blk_idx.fill_(-1)

    def _poison_outputs(self):
        if self.poison:
            self.out.fill_(float("nan"))
            self.lse.fill_(float("nan"))

    def select(self):
        self._poison_lists()
        fp2_select_blocks(self.plan, self.q, self.k_cache, self.v_cache, self.page_table, self.cu_seqlens_q,
                          self.seqlens_k, self.q_scale, self.k_scale, self.v_scale, self.seg_offset, self.seg_count,
                          self.blk_idx, self.workspace)

    def pool(self):
        fp2_pool_blocks(self.plan, self.k_cache, self.v_cache, self.page_table, self.seqlens_k, self.k_scale,
                        self.v_scale, self.workspace)

    def sparse(self, pooled_valid=True, seg_count=None, blk_idx=None):
        self._poison_outputs()
        fp2_sparse_prefill(self.plan, self.q, self.k_cache, self.v_cache, self.page_table, self.cu_seqlens_q,
                           self.seqlens_k, self.seg_offset, self.seg_count if seg_count is None else seg_count,
                           self.blk_idx if blk_idx is None else blk_idx, self.q_scale, self.k_scale, self.v_scale,
                           self.out, self.lse, self.workspace, pooled_valid)

    def dense(self):
        self._poison_outputs()
        fp2_dense_prefill(self.plan, self.q, self.k_cache, self.v_cache, self.page_table, self.cu_seqlens_q,
                          self.seqlens_k, self.q_scale, self.k_scale, self.v_scale, self.out, self.lse,
                          self.workspace)

    def window(self, window_tokens, sink_tokens=0):
        self._poison_outputs()
        fp2_window_prefill(self.plan, self.q, self.k_cache, self.v_cache, self.page_table, self.cu_seqlens_q, self.seqlens_k,
                           self.q_scale, self.k_scale, self.v_scale, window_tokens, sink_tokens, self.out, self.lse,
                           self.workspace)

    def export_csr(self, tile_tokens=64):
        """(cu, idx) device tensors of the lists currently in the buffers."""
        cu = torch.empty(self.plan.num_segments + 1, dtype=torch.int32, device=self.q.device)
        idx = torch.empty(max(self.plan.idx_capacity * (128 // tile_tokens), 1), dtype=torch.int32, device=self.q.device)
        fp2_export_csr(self.plan, self.seg_count, self.blk_idx, tile_tokens, cu, idx, self.workspace)
        return cu, idx

    def status(self, raise_on_error=True):
        return fp2_read_status(self.plan, self.workspace, raise_on_error=raise_on_error)

    def lists_host(self):
        """{seg: ascending int32 array} of the lists currently in the buffers."""
        off = self.seg_offset.cpu().numpy()
        cnt = self.seg_count.cpu().numpy()
        idx = self.blk_idx.cpu().numpy()
        return {s: idx[off[s]:off[s] + cnt[s]].copy() for s in range(self.plan.num_segments)}
