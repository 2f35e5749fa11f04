"""Thin ctypes binding of ``libadaspark_attn.so``: the same entry points as
``include/adaspark_attn.h``, argument marshalling only.  Every step of AdaS-Attn runs inside the
library's CUDA kernels; torch is used here for device memory and streams only.

There is no CPU fallback: if the shared library is missing, ``load()`` raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libadaspark_attn.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_NOT_PARTITIONED, ERR_WORKSPACE_TOO_SMALL, ERR_CUDA, \
    ERR_TIMEOUT = range(7)
STATUS_NAMES = ["OK", "ERR_INVALID_ARG", "ERR_UNSUPPORTED", "ERR_NOT_PARTITIONED",
                "ERR_WORKSPACE_TOO_SMALL", "ERR_CUDA", "ERR_TIMEOUT"]


class Config(ctypes.Structure):
    _fields_ = [("cube_t", ctypes.c_int32), ("cube_h", ctypes.c_int32), ("cube_w", ctypes.c_int32),
                ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("top_p", ctypes.c_float),
                ("softmax_scale", ctypes.c_float), ("device", ctypes.c_int32), ("top_k", ctypes.c_int32)]


class Layout(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in (
        "n_cubes", "cube_tokens", "s_video", "s_cap", "bitmap_words", "k_cube_bytes",
        "v_cube_bytes", "cube_keys_bytes", "forward_workspace_bytes", "decode_workspace_bytes")]


class Pages(ctypes.Structure):
    _fields_ = [("k_pages", ctypes.c_void_p), ("v_pages", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("page_stride", ctypes.c_int64), ("scale_stride", ctypes.c_int64),
                ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("format", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


PAGES_BF16, PAGES_E4M3 = 0, 1


class AdasparkError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES[status] if 0 <= status < 7 else status}: {message}")
        self.status = status


_lib: Optional[ctypes.CDLL] = None

EXPORTS = ["adaspark_attn_create", "adaspark_attn_partition", "adaspark_attn_get_layout",
           "adaspark_attn_forward", "adaspark_attn_forward_host", "adaspark_attn_forward_prefix", "adaspark_attn_forward_chunk", "adaspark_attn_decode", "adaspark_attn_destroy",
           "adaspark_attn_last_error", "adaspark_attn_last_launch_count",
           "adaspark_attn_set_prefill_kernel", "adaspark_attn_set_gather", "adaspark_attn_enable_stage_timing",
           "adaspark_attn_get_stage_times", "adaspark_attn_get_attention_kernel_ms", "adaspark_attn_decode_static",
           "adaspark_attn_text_workspace_bytes", "adaspark_attn_prompt", "adaspark_attn_paged_write",
           "adaspark_attn_paged_read", "adaspark_attn_paged_decode",
           "adaspark_attn_debug_umma_selftest", "adaspark_attn_debug_imma_selftest",
           "adaspark_attn_debug_fastdiv", "adaspark_attn_debug_wait_timeout"]


def load() -> ctypes.CDLL:
    """dlopen the in-tree library; raises if it has not been built (no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2604_08077_b200.build` "
                           "(there is no CPU or PyTorch fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    lib.adaspark_attn_create.argtypes = [ctypes.POINTER(Config), ctypes.POINTER(vp)]
    lib.adaspark_attn_partition.argtypes = [vp, i32, i32, i32, i32, i32, ctypes.POINTER(sz)]
    lib.adaspark_attn_get_layout.argtypes = [vp, ctypes.POINTER(Layout)]
    lib.adaspark_attn_forward.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.adaspark_attn_forward_host.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.adaspark_attn_forward_prefix.argtypes = [vp, vp, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.adaspark_attn_forward_chunk.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.adaspark_attn_decode.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.adaspark_attn_decode_static.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.adaspark_attn_debug_umma_selftest.argtypes = [vp, vp, vp, vp, vp, vp, vp]
    lib.adaspark_attn_debug_imma_selftest.argtypes = [vp, vp, vp, vp, vp]
    lib.adaspark_attn_debug_wait_timeout.argtypes = [ctypes.c_uint64, vp, vp, vp]
    lib.adaspark_attn_debug_fastdiv.argtypes = [ctypes.c_int32, ctypes.c_int32]
    lib.adaspark_attn_debug_fastdiv.restype = ctypes.c_int32
    lib.adaspark_attn_destroy.argtypes = [vp]
    lib.adaspark_attn_last_error.argtypes = [vp]
    lib.adaspark_attn_last_error.restype = ctypes.c_char_p
    lib.adaspark_attn_last_launch_count.argtypes = [vp]
    lib.adaspark_attn_last_launch_count.restype = ctypes.c_int64
    lib.adaspark_attn_set_prefill_kernel.argtypes = [vp, i32]
    lib.adaspark_attn_set_gather.argtypes = [vp, ctypes.c_float, ctypes.c_uint64]
    lib.adaspark_attn_enable_stage_timing.argtypes = [vp, i32]
    lib.adaspark_attn_get_stage_times.argtypes = [vp, ctypes.POINTER(ctypes.c_float)]
    lib.adaspark_attn_get_attention_kernel_ms.argtypes = [vp, ctypes.POINTER(ctypes.c_float)]
    i64, pages = ctypes.c_int64, ctypes.POINTER(Pages)
    rows = [vp, i64, i64]                                       # pointer, token stride, head stride
    lib.adaspark_attn_text_workspace_bytes.argtypes = [vp]
    lib.adaspark_attn_text_workspace_bytes.restype = i64
    lib.adaspark_attn_prompt.argtypes = [vp, *rows, *rows, *rows, vp, vp, i32, i32, i32, vp, vp, vp, sz, vp, vp]
    lib.adaspark_attn_paged_write.argtypes = [vp, pages, *rows, *rows, vp, i32, i32, vp, i32, vp, vp, vp]
    lib.adaspark_attn_paged_read.argtypes = [vp, pages, vp, i32, i32, vp, i32, vp, vp, vp, vp, vp]
    lib.adaspark_attn_paged_decode.argtypes = [vp, *rows, *rows, *rows, pages, vp, i32, vp, i32, vp, vp, vp, sz, vp, vp]
    for name in EXPORTS:
        if name not in ("adaspark_attn_last_error", "adaspark_attn_last_launch_count", "adaspark_attn_text_workspace_bytes"):
            getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    assert t.is_contiguous(), "tensors crossing the C ABI must be contiguous"
    return t.data_ptr()


def _stream_ptr(stream) -> Optional[int]:
    if stream is None:
        if not torch.cuda.is_available():   # host-side argument checks still run without a GPU
            return None
        return torch.cuda.current_stream().cuda_stream or None
    return stream.cuda_stream or None


# ---- the C entry points, one Python function each (raw: pointers are ints or tensors) ----------

def adaspark_attn_create(config: Config) -> int:
    h = ctypes.c_void_p()
    st = load().adaspark_attn_create(ctypes.byref(config), ctypes.byref(h))
    if st != OK:
        raise AdasparkError(st, "adaspark_attn_create rejected the configuration")
    return h.value


def _check(handle: int, st: int):
    if st != OK:
        raise AdasparkError(st, load().adaspark_attn_last_error(handle).decode())


def adaspark_attn_partition(handle: int, batch: int, frames: int, grid_h: int, grid_w: int,
                            n_text_max: int) -> int:
    ws = ctypes.c_size_t(0)
    _check(handle, load().adaspark_attn_partition(handle, batch, frames, grid_h, grid_w, n_text_max,
                                                  ctypes.byref(ws)))
    return ws.value


def adaspark_attn_get_layout(handle: int) -> Layout:
    lay = Layout()
    _check(handle, load().adaspark_attn_get_layout(handle, ctypes.byref(lay)))
    return lay


def adaspark_attn_forward(handle: int, q, k, v, n_text: int, out, k_cube, v_cube, cube_keys,
                          sel_bitmap, sel_count, workspace, workspace_bytes: int, stream=None):
    _check(handle, load().adaspark_attn_forward(
        handle, _ptr(q), _ptr(k), _ptr(v), n_text, _ptr(out), _ptr(k_cube), _ptr(v_cube),
        _ptr(cube_keys), _ptr(sel_bitmap), _ptr(sel_count), _ptr(workspace), workspace_bytes,
        _stream_ptr(stream)))


def adaspark_attn_forward_host(handle: int, q_host, k_host, v_host, n_text: int, out_host, q_dev, k_dev, v_dev,
                               out_dev, k_cube, v_cube, cube_keys, workspace, workspace_bytes: int, stream=None):
    """Prefill from and to host (pinned) tensors: the library issues the copies on the stream."""
    _check(handle, load().adaspark_attn_forward_host(
        handle, _ptr(q_host), _ptr(k_host), _ptr(v_host), n_text, _ptr(out_host), _ptr(q_dev), _ptr(k_dev),
        _ptr(v_dev), _ptr(out_dev), _ptr(k_cube), _ptr(v_cube), _ptr(cube_keys), _ptr(workspace),
        workspace_bytes, _stream_ptr(stream)))


def adaspark_attn_forward_prefix(handle: int, q, k, v, n_prefix: int, n_text: int, out, k_cube, v_cube, cube_keys,
                                 sel_bitmap, sel_count, workspace, workspace_bytes: int, stream=None):
    _check(handle, load().adaspark_attn_forward_prefix(
        handle, _ptr(q), _ptr(k), _ptr(v), n_prefix, n_text, _ptr(out), _ptr(k_cube), _ptr(v_cube),
        _ptr(cube_keys), _ptr(sel_bitmap), _ptr(sel_count), _ptr(workspace), workspace_bytes,
        _stream_ptr(stream)))


def adaspark_attn_forward_chunk(handle: int, q, k, v, frame_begin: int, frame_count: int, n_text: int, out,
                                k_cube, v_cube, cube_keys, sel_bitmap, sel_count, workspace,
                                workspace_bytes: int, stream=None):
    _check(handle, load().adaspark_attn_forward_chunk(
        handle, _ptr(q), _ptr(k), _ptr(v), frame_begin, frame_count, n_text, _ptr(out), _ptr(k_cube),
        _ptr(v_cube), _ptr(cube_keys), _ptr(sel_bitmap), _ptr(sel_count), _ptr(workspace), workspace_bytes,
        _stream_ptr(stream)))


def adaspark_attn_decode(handle: int, q_new, k_new, v_new, k_cube, v_cube, cube_keys, text_len, out,
                         sel_bitmap, workspace, workspace_bytes: int, stream=None):
    _check(handle, load().adaspark_attn_decode(
        handle, _ptr(q_new), _ptr(k_new), _ptr(v_new), _ptr(k_cube), _ptr(v_cube), _ptr(cube_keys),
        _ptr(text_len), _ptr(out), _ptr(sel_bitmap), _ptr(workspace), workspace_bytes,
        _stream_ptr(stream)))


STATIC_SCRATCH_BYTES = 8 << 20


def adaspark_attn_decode_static(handle: int, q_new, k_new, v_new, k_cube, v_cube, cube_keys, text_len,
                                out, sel_bitmap, stream=None):
    """Decode step that takes no workspace: for callers that cannot allocate device memory when
    they decode (all memory already owned by their own pool, or no cudaMalloc allowed inside the
    serving loop).  Scratch is the library's built-in 8 MiB array, shared by all calls on a device."""
    _check(handle, load().adaspark_attn_decode_static(
        handle, _ptr(q_new), _ptr(k_new), _ptr(v_new), _ptr(k_cube), _ptr(v_cube), _ptr(cube_keys),
        _ptr(text_len), _ptr(out), _ptr(sel_bitmap), _stream_ptr(stream)))


def adaspark_attn_debug_umma_selftest(a, b, c, d_out, e_out, status, stream=None) -> int:
    """128x128x128 tcgen05 self-test (see include/adaspark_attn_debug.h); returns the status code."""
    return int(load().adaspark_attn_debug_umma_selftest(_ptr(a), _ptr(b), _ptr(c), _ptr(d_out),
                                                       _ptr(e_out), _ptr(status), _stream_ptr(stream)))


def adaspark_attn_debug_imma_selftest(a, b, d_out, status, stream=None) -> int:
    """128x128x128 int8 tcgen05 self-test (see include/adaspark_attn_debug.h); returns the status code."""
    return int(load().adaspark_attn_debug_imma_selftest(_ptr(a), _ptr(b), _ptr(d_out), _ptr(status),
                                                       _stream_ptr(stream)))


def adaspark_attn_debug_wait_timeout(limit_ns: int, status, waited_ns, stream=None) -> int:
    """A bounded device wait that is made to expire (see include/adaspark_attn_debug.h)."""
    return int(load().adaspark_attn_debug_wait_timeout(int(limit_ns), _ptr(status), _ptr(waited_ns),
                                                       _stream_ptr(stream)))


def adaspark_attn_debug_fastdiv(n: int, d: int) -> int:
    """n // d by the kernels' multiply-shift index arithmetic (host only)."""
    return int(load().adaspark_attn_debug_fastdiv(n, d))


def adaspark_attn_destroy(handle: int):
    load().adaspark_attn_destroy(handle)


def adaspark_attn_last_launch_count(handle: int) -> int:
    return int(load().adaspark_attn_last_launch_count(handle))


def adaspark_attn_set_prefill_kernel(handle: int, which: int):
    _check(handle, load().adaspark_attn_set_prefill_kernel(handle, which))


def adaspark_attn_set_gather(handle: int, pairs_per_block: float, budget_bytes: int):
    _check(handle, load().adaspark_attn_set_gather(handle, float(pairs_per_block), int(budget_bytes)))


def adaspark_attn_enable_stage_timing(handle: int, enable: bool):
    _check(handle, load().adaspark_attn_enable_stage_timing(handle, int(enable)))


def adaspark_attn_get_stage_times(handle: int):
    """Milliseconds of the four stages of the last timed call (waits for its last event)."""
    ms = (ctypes.c_float * 4)()
    _check(handle, load().adaspark_attn_get_stage_times(handle, ms))
    return [float(x) for x in ms]


def adaspark_attn_get_attention_kernel_ms(handle: int) -> float:
    """Milliseconds of the union attention kernel of the last timed prefill."""
    ms = (ctypes.c_float * 1)()
    _check(handle, load().adaspark_attn_get_attention_kernel_ms(handle, ms))
    return float(ms[0])


# ---- text beside the video (tensors: a row argument is (tensor or pointer, token stride, head stride)) ----

def adaspark_attn_text_workspace_bytes(handle: int) -> int:
    return int(load().adaspark_attn_text_workspace_bytes(handle))


def adaspark_attn_prompt(handle: int, q, k, v, cu_q, cu_k, batch: int, n_q: int, n_k: int, out, lse, workspace,
                         workspace_bytes: int, status, stream: Optional[int]):
    """q, k, v: (pointer, token stride, head stride); the others pointers or None."""
    st = load().adaspark_attn_prompt(handle, *q, *k, *v, cu_q, cu_k, batch, n_q, n_k, out, lse, workspace, workspace_bytes, status, stream)
    if st != OK:
        _check(handle, st)


def adaspark_attn_paged_write(handle: int, pages: Pages, k, v, cu, batch: int, n: int, block_table, table_width: int, kv_len,
                              status, stream: Optional[int]):
    st = load().adaspark_attn_paged_write(handle, pages, *k, *v, cu, batch, n, block_table, table_width, kv_len, status, stream)
    if st != OK:
        _check(handle, st)


def adaspark_attn_paged_read(handle: int, pages: Pages, cu, batch: int, n: int, block_table, table_width: int, kv_len, k_out, v_out,
                             status, stream: Optional[int]):
    st = load().adaspark_attn_paged_read(handle, pages, cu, batch, n, block_table, table_width, kv_len, k_out, v_out, status, stream)
    if st != OK:
        _check(handle, st)


def adaspark_attn_paged_decode(handle: int, q, k_new, v_new, pages: Pages, block_table, table_width: int, kv_len, batch: int, out, lse,
                               workspace, workspace_bytes: int, status, stream: Optional[int]):
    st = load().adaspark_attn_paged_decode(handle, *q, *k_new, *v_new, pages, block_table, table_width, kv_len, batch, out, lse, workspace,
                                           workspace_bytes, status, stream)
    if st != OK:
        _check(handle, st)


class WorkspaceHeader(ctypes.Structure):
    _fields_ = [("status", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("executed_kv_blocks", ctypes.c_uint64), ("decode_kv_blocks", ctypes.c_uint64),
                ("fallback_rows", ctypes.c_uint32), ("max_tile_kv_blocks", ctypes.c_uint32),
                ("gather_entries", ctypes.c_uint32), ("gather_items", ctypes.c_uint32),
                ("gather_pair_tiles", ctypes.c_uint32), ("reserved2", ctypes.c_uint32)]


# ---- a small convenience owner of the handle and of the caller-side buffers --------------------

def _refuse(message: str):
    raise AdasparkError(ERR_INVALID_ARG, message)


class PagedCache:
    """Pages of keys and values [n_pages, n_kv_heads, page_size, head_dim], bf16, or float8_e4m3fn with uint8 scales
    [n_pages, n_kv_heads, page_size] (see adaspark_attn_pages_t).  Inside a page everything is dense; pages may lie apart (a slice
    of a larger pool), keys and values alike."""

    def __init__(self, k_pages, v_pages, k_scale=None, v_scale=None):
        if k_pages.dim() != 4 or k_pages.shape != v_pages.shape or k_pages.dtype != v_pages.dtype or k_pages.device != v_pages.device:
            _refuse("PagedCache: k_pages and v_pages are not two alike tensors [pages, kv heads, page size, head_dim]")
        if k_pages.dtype == torch.bfloat16:
            fmt = PAGES_BF16
            if k_scale is not None or v_scale is not None:
                _refuse("PagedCache: bf16 pages have no scales")
        elif k_pages.dtype == torch.float8_e4m3fn:
            fmt = PAGES_E4M3
            for s in (k_scale, v_scale):
                if s is None or s.dtype != torch.uint8 or s.shape != k_pages.shape[:3] or s.device != k_pages.device:
                    _refuse("PagedCache: e4m3 pages need uint8 scales [pages, kv heads, page size] beside them")
        else:
            _refuse(f"PagedCache: pages of {k_pages.dtype}: bfloat16 or float8_e4m3fn are held")

        def stride_of(a, b):
            inner = a[0].numel() if a.shape[0] else 0
            for t in (a, b):
                if t.shape[0] and not t[0].is_contiguous():
                    _refuse("PagedCache: a page has to be dense")
            if a.shape[0] <= 1:
                return inner
            if a.stride(0) != b.stride(0) or a.stride(0) < inner:
                _refuse("PagedCache: keys and values need the same distance from page to page, of at least a page")
            return a.stride(0)

        if k_pages.shape[0] == 0:
            _refuse("PagedCache: no pages")
        self.k_pages, self.v_pages, self.k_scale, self.v_scale = k_pages, v_pages, k_scale, v_scale
        self.device = k_pages.device
        self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = k_pages.shape
        self.pages = Pages(k_pages.data_ptr(), v_pages.data_ptr(), k_scale.data_ptr() if fmt else None,
                           v_scale.data_ptr() if fmt else None, stride_of(k_pages, v_pages),
                           stride_of(k_scale, v_scale) if fmt else 0, self.n_pages, self.page_size, fmt, 0)

class AdaSAttn:
    """Owns a handle plus the torch-allocated caches and workspace for one partition."""

    def __init__(self, *, cube, n_q_heads, n_kv_heads, head_dim, top_p, softmax_scale=0.0,
                 device: int = 0, top_k: int = 0):
        self.cfg = Config(cube[0], cube[1], cube[2], n_q_heads, n_kv_heads, head_dim, float(top_p),
                          float(softmax_scale), device, int(top_k))
        self.handle = adaspark_attn_create(self.cfg)
        self.device = torch.device("cuda", device)
        self.layout: Optional[Layout] = None
        self._text = None

    def set_gather(self, pairs_per_block: float, budget_bytes: int = 24 << 30):
        """Threshold and workspace budget of the query-gather path (budget: before partition())."""
        adaspark_attn_set_gather(self.handle, pairs_per_block, budget_bytes)

    def partition(self, batch, frames, grid_h, grid_w, n_text_max):
        self.ws_bytes = adaspark_attn_partition(self.handle, batch, frames, grid_h, grid_w, n_text_max)
        self.layout = lay = adaspark_attn_get_layout(self.handle)
        self.batch = batch
        dev, c = self.device, self.cfg
        self.k_cube = torch.empty(lay.k_cube_bytes // 2, dtype=torch.bfloat16, device=dev).view(
            batch, c.n_kv_heads, lay.s_cap, c.head_dim)
        self.v_cube = torch.empty(lay.v_cube_bytes // 2, dtype=torch.bfloat16, device=dev).view(
            batch, c.n_kv_heads, lay.s_cap // 64, c.head_dim, 64)
        self.cube_keys = torch.empty(batch, c.n_kv_heads, lay.n_cubes, c.head_dim,
                                     dtype=torch.float32, device=dev)
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=dev)
        return self

    def forward(self, q, k, v, n_text, *, out=None, want_selection=False, stream=None, n_prefix=0):
        """q may be None: builds only the caches.  Returns (out, sel_bitmap, sel_count).
        n_prefix > 0: the first n_prefix tokens of the tensors are text that precedes the video."""
        lay = self.layout
        bitmap = count = None
        if q is not None:
            if out is None:
                out = torch.empty_like(q)
            if want_selection:
                B, S, Hq, _ = q.shape
                bitmap = torch.empty(B, Hq, S, lay.bitmap_words, dtype=torch.int32, device=q.device)
                count = torch.empty(B, Hq, S, dtype=torch.int32, device=q.device)
        if n_prefix:
            adaspark_attn_forward_prefix(self.handle, q, k, v, n_prefix, n_text, out, self.k_cube, self.v_cube,
                                         self.cube_keys, bitmap, count, self.workspace, self.ws_bytes, stream)
        else:
            adaspark_attn_forward(self.handle, q, k, v, n_text, out, self.k_cube, self.v_cube,
                                  self.cube_keys, bitmap, count, self.workspace, self.ws_bytes, stream)
        return out, bitmap, count

    def forward_host(self, q_host, k_host, v_host, n_text, out_host, staging, stream=None):
        """Prefill with host tensors; `staging` = (q, k, v, out) device tensors of the same shapes."""
        qd, kd, vd, od = staging
        adaspark_attn_forward_host(self.handle, q_host, k_host, v_host, n_text, out_host, qd, kd, vd, od,
                                   self.k_cube, self.v_cube, self.cube_keys, self.workspace, self.ws_bytes, stream)
        return out_host

    def forward_chunk(self, q, k, v, frame_begin, frame_count, n_text, *, out=None, want_selection=False,
                      stream=None):
        """One chunk of a chunked prefill (n_text < 0: more video follows).  q may be None."""
        lay = self.layout
        bitmap = count = None
        if q is not None:
            if out is None:
                out = torch.empty_like(q)
            if want_selection:
                B, S, Hq, _ = q.shape
                bitmap = torch.empty(B, Hq, S, lay.bitmap_words, dtype=torch.int32, device=q.device)
                count = torch.empty(B, Hq, S, dtype=torch.int32, device=q.device)
        adaspark_attn_forward_chunk(self.handle, q, k, v, frame_begin, frame_count, n_text, out, self.k_cube,
                                    self.v_cube, self.cube_keys, bitmap, count, self.workspace, self.ws_bytes,
                                    stream)
        return out, bitmap, count

    def decode(self, q_new, k_new, v_new, text_len, *, out=None, want_selection=False, stream=None):
        lay = self.layout
        if out is None:
            out = torch.empty_like(q_new)
        bitmap = None
        if want_selection:
            B, _, Hq, _ = q_new.shape
            bitmap = torch.empty(B, Hq, lay.bitmap_words, dtype=torch.int32, device=q_new.device)
        adaspark_attn_decode(self.handle, q_new, k_new, v_new, self.k_cube, self.v_cube,
                             self.cube_keys, text_len, out, bitmap, self.workspace, self.ws_bytes,
                             stream)
        return out, bitmap

    # ---- text beside the video: packed prompts and a paged cache (no partition() needed) ----

    def paged_cache(self, n_pages: int, page_size: int, *, e4m3: bool = False) -> PagedCache:
        """A zeroed pool of pages for this handle's heads: bf16, or 8 bits a value."""
        c, dev = self.cfg, self.device
        shape = (n_pages, c.n_kv_heads, page_size, c.head_dim)
        dtype = torch.float8_e4m3fn if e4m3 else torch.bfloat16
        pages = [torch.zeros(shape, dtype=dtype, device=dev) for _ in range(2)]
        scales = [torch.zeros(shape[:3], dtype=torch.uint8, device=dev) for _ in range(2)] if e4m3 else [None, None]
        return PagedCache(*pages, *scales)

    def _text_buffers(self):
        """Workspace and status word of the text calls, made once."""
        if self._text is None:
            n = adaspark_attn_text_workspace_bytes(self.handle)
            ws = torch.empty(n, dtype=torch.uint8, device=self.device)
            self._text = (ws, n, ws.data_ptr(), torch.zeros(1, dtype=torch.int32, device=self.device))
            self._text = (*self._text, self._text[3].data_ptr())
        return self._text

    def text_status(self) -> int:
        """What the text calls of this object found wrong on the device since the last look: 0 = nothing (waits for the device)."""
        if self._text is None:
            return 0
        got = int(self._text[3].item())
        if got:
            self._text[3].zero_()
        return got

    def _stream(self, stream):
        return (torch.cuda.current_stream(self.device) if stream is None else stream).cuda_stream or None

    def _rows(self, t, heads: int, what: str):
        """(pointer, token stride, head stride) of a bf16 tensor [rows, heads, head_dim] on this device."""
        shape, strides = t.shape, t.stride()
        if len(shape) != 3 or shape[1] != heads or shape[2] != self.cfg.head_dim or t.dtype != torch.bfloat16:
            _refuse(f"{what}: {t.dtype} {tuple(shape)} is not bfloat16 [rows, {heads}, {self.cfg.head_dim}]")
        if strides[2] != 1:
            _refuse(f"{what}: the values of a row have to lie side by side")
        if t.device != self.device:
            _refuse(f"{what} is on {t.device}, not on {self.device}")
        # (the stride of an axis of one entry says nothing)
        return t.data_ptr(), strides[0] if shape[0] > 1 else 0, strides[1] if heads > 1 else 0

    def _dense(self, t, shape, dtype, what: str) -> int:
        if t.shape != shape or t.dtype != dtype or not t.is_contiguous():
            _refuse(f"{what}: {t.dtype} {tuple(t.shape)} is not dense {dtype} {tuple(shape)}")
        if t.device != self.device:
            _refuse(f"{what} is on {t.device}, not on {self.device}")
        return t.data_ptr()

    def _ints(self, t, what: str, dims: int = 1) -> int:
        if t.dtype != torch.int32 or t.dim() != dims or not t.is_contiguous() or t.device != self.device:
            _refuse(f"{what}: dense int32 with {dims} axes on {self.device} is needed")
        return t.data_ptr()

    def _cache(self, cache: PagedCache) -> Pages:
        if cache.n_kv_heads != self.cfg.n_kv_heads or cache.head_dim != self.cfg.head_dim or cache.device != self.device:
            _refuse(f"cache of {cache.n_kv_heads} heads of {cache.head_dim} on {cache.device}: not this handle's")
        return cache.pages

    def prompt(self, q, k, v, cu_q, cu_k=None, *, out=None, lse=None, want_lse=False, stream=None):
        """Causal attention of packed prompts: q [n_q, Hq, D], k and v [n_k, Hkv, D] bf16, cu_q (and cu_k, if the keys of a sequence
        are more than its queries) int32 [batch + 1].  Returns (out, lse); lse is None unless given or wanted."""
        c = self.cfg
        ws, ws_bytes, ws_ptr, status, status_ptr = self._text_buffers()
        qr, kr, vr = self._rows(q, c.n_q_heads, "q"), self._rows(k, c.n_kv_heads, "k"), self._rows(v, c.n_kv_heads, "v")
        n_q, n_k = q.shape[0], k.shape[0]
        if v.shape[0] != n_k:
            _refuse(f"v has {v.shape[0]} rows, k {n_k}")
        cq = self._ints(cu_q, "cu_q")
        ck = cq if cu_k is None else self._ints(cu_k, "cu_k")
        batch = cu_q.shape[0] - 1
        if batch < 0 or (cu_k is not None and cu_k.shape[0] != batch + 1):
            _refuse("cu_q and cu_k hold batch + 1 entries each")
        if out is None:
            out = torch.empty(n_q, c.n_q_heads, c.head_dim, dtype=torch.bfloat16, device=self.device)
        if lse is None and want_lse:
            lse = torch.empty(n_q, c.n_q_heads, dtype=torch.float32, device=self.device)
        adaspark_attn_prompt(self.handle, qr, kr, vr, cq, ck, batch, n_q, n_k,
                             self._dense(out, (n_q, c.n_q_heads, c.head_dim), torch.bfloat16, "out"),
                             None if lse is None else self._dense(lse, (n_q, c.n_q_heads), torch.float32, "lse"),
                             ws_ptr, ws_bytes, status_ptr, self._stream(stream))
        return out, lse

    def paged_write(self, cache: PagedCache, k, v, cu, block_table, kv_len, *, stream=None):
        """Packed keys and values into the pages: the rows cu[b] .. cu[b + 1] - 1 become the last tokens of sequence b, which
        then holds kv_len[b].  block_table int32 [batch, width]."""
        status_ptr = self._text_buffers()[4]
        kr, vr = self._rows(k, self.cfg.n_kv_heads, "k"), self._rows(v, self.cfg.n_kv_heads, "v")
        if k.shape[0] != v.shape[0]:
            _refuse(f"v has {v.shape[0]} rows, k {k.shape[0]}")
        batch = self._batch(cu, block_table, kv_len)
        adaspark_attn_paged_write(self.handle, self._cache(cache), kr, vr, self._ints(cu, "cu"), batch, k.shape[0],
                                  self._ints(block_table, "block_table", 2), block_table.shape[1], self._ints(kv_len, "kv_len"),
                                  status_ptr, self._stream(stream))

    def paged_read(self, cache: PagedCache, cu, block_table, kv_len, k_out, v_out, *, stream=None):
        """The last cu[b + 1] - cu[b] tokens of every sequence from the pages into k_out, v_out: bf16 [n, Hkv, D].  Returns them."""
        c = self.cfg
        status_ptr = self._text_buffers()[4]
        n = k_out.shape[0]
        batch = self._batch(cu, block_table, kv_len)
        adaspark_attn_paged_read(self.handle, self._cache(cache), self._ints(cu, "cu"), batch, n,
                                 self._ints(block_table, "block_table", 2), block_table.shape[1], self._ints(kv_len, "kv_len"),
                                 self._dense(k_out, (n, c.n_kv_heads, c.head_dim), torch.bfloat16, "k_out"),
                                 self._dense(v_out, (n, c.n_kv_heads, c.head_dim), torch.bfloat16, "v_out"), status_ptr, self._stream(stream))
        return k_out, v_out

    @staticmethod
    def _batch(cu, block_table, kv_len) -> int:
        batch = kv_len.shape[0]
        if block_table.dim() != 2 or block_table.shape[0] != batch or (cu is not None and cu.shape[0] != batch + 1):
            _refuse(f"kv_len of {batch} sequences, block table {tuple(block_table.shape)}, cu {None if cu is None else tuple(cu.shape)}")
        return batch

    def paged_decode(self, q, k_new, v_new, cache: PagedCache, block_table, kv_len, *, out=None, lse=None, want_lse=False,
                     stream=None):
        """One new token per sequence against its pages.  q [batch, Hq, D]; k_new, v_new [batch, Hkv, D] are stored as token
        kv_len[b] - 1 first (None: they are there).  kv_len 0: a slot without a sequence.  Returns (out, lse)."""
        c = self.cfg
        ws, ws_bytes, ws_ptr, status, status_ptr = self._text_buffers()
        batch = self._batch(None, block_table, kv_len)
        if q.shape[0] != batch or (k_new is None) != (v_new is None) or (k_new is not None and (k_new.shape[0] != batch or v_new.shape[0] != batch)):
            _refuse("q, k_new and v_new hold a row for each entry of kv_len (k_new and v_new both or neither)")
        none = (None, 0, 0)
        if out is None:
            out = torch.empty(batch, c.n_q_heads, c.head_dim, dtype=torch.bfloat16, device=self.device)
        if lse is None and want_lse:
            lse = torch.empty(batch, c.n_q_heads, dtype=torch.float32, device=self.device)
        adaspark_attn_paged_decode(self.handle, self._rows(q, c.n_q_heads, "q"), none if k_new is None else self._rows(k_new, c.n_kv_heads, "k_new"),
                                   none if v_new is None else self._rows(v_new, c.n_kv_heads, "v_new"), self._cache(cache),
                                   self._ints(block_table, "block_table", 2), block_table.shape[1], self._ints(kv_len, "kv_len"), batch,
                                   self._dense(out, (batch, c.n_q_heads, c.head_dim), torch.bfloat16, "out"),
                                   None if lse is None else self._dense(lse, (batch, c.n_q_heads), torch.float32, "lse"),
                                   ws_ptr, ws_bytes, status_ptr, self._stream(stream))
        return out, lse

    def header(self) -> WorkspaceHeader:
        """Copy of the workspace header of the last call (synchronises the device)."""
        raw = self.workspace[:ctypes.sizeof(WorkspaceHeader)].cpu().numpy().tobytes()
        return WorkspaceHeader.from_buffer_copy(raw)

    def launches(self) -> int:
        return adaspark_attn_last_launch_count(self.handle)

    def close(self):
        if self.handle:
            adaspark_attn_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
