"""Thin ctypes binding of ``libadaspark_attn.so``: the same entry points as
``include/adaspark_attn.h``, argument marshalling only.  Every step of AdaS-Attn runs inside the
library's CUDA kernels; torch is used here for device memory and streams only.

There is no CPU fallback: if the shared library is missing, ``load()`` raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
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


PAGES_BF16, PAGES_E4M3 = 0, 1
_BF16, _INT32 = torch.bfloat16, torch.int32

# The arguments of the text calls, packed as the header's structs lay them out (one bytes object per call: a quarter of the time that
# ctypes takes for two dozen arguments).  A row argument is (pointer, token stride, head stride).
_PAGES = struct.Struct("4Q2q4i")          # adaspark_attn_pages_t
_PROMPT = struct.Struct("QqqQqqQqq5QqQ4i")  # adaspark_attn_prompt_t
_PAGED_ROWS = struct.Struct("QqqQqq4Q4i")   # adaspark_attn_paged_rows_t behind its pages
_PAGED_DECODE = struct.Struct("QqqQqqQqq5QqQ2i")   # adaspark_attn_paged_decode_t behind its pages
_WINDOW = struct.Struct("2i")               # adaspark_attn_paged_decode_window_t behind its step
_PAGED_PROMPT = struct.Struct("Qqq6QqQ6i")  # adaspark_attn_paged_prompt_t behind its pages
_ROTATE = struct.Struct("QqqQqqQqqQqq4Qfi")  # adaspark_attn_rotate_t
_PAGED_APPEND = struct.Struct("QqqQqqQqqQqq8Qf3i")   # adaspark_attn_paged_append_t behind its pages


class RotaryStruct(ctypes.Structure):
    """adaspark_attn_rotary_t."""
    _fields_ = [("turns", ctypes.c_uint64 * 64), ("axis", ctypes.c_uint8 * 64), ("pairs", ctypes.c_int32), ("axes", ctypes.c_int32),
                ("adjacent", ctypes.c_int32), ("reserved", ctypes.c_int32)]


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
           "adaspark_attn_paged_read", "adaspark_attn_paged_decode", "adaspark_attn_paged_decode_window",
           "adaspark_attn_paged_prompt", "adaspark_attn_rotary_init", "adaspark_attn_rotate", "adaspark_attn_paged_append",
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
    lib.adaspark_attn_text_workspace_bytes.argtypes = [vp]
    lib.adaspark_attn_text_workspace_bytes.restype = ctypes.c_int64
    lib.adaspark_attn_rotary_init.argtypes = [ctypes.POINTER(RotaryStruct), ctypes.POINTER(ctypes.c_double), ctypes.POINTER(i32), i32, i32, i32]
    for name in ("prompt", "paged_write", "paged_read", "paged_decode", "paged_decode_window", "paged_prompt", "rotate", "paged_append"):
        getattr(lib, "adaspark_attn_" + name).argtypes = [vp, ctypes.c_char_p, vp]
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


# ---- text beside the video: pointers (None: NULL), rows as (pointer, token stride, head stride), pages from pages_struct() ----

_NO_ROWS = (0, 0, 0)


def adaspark_attn_text_workspace_bytes(handle: int) -> int:
    return int(load().adaspark_attn_text_workspace_bytes(handle))


def pages_struct(k_pages, v_pages, k_scale, v_scale, page_stride: int, scale_stride: int, n_pages: int, page_size: int,
                 page_format: int) -> bytes:
    """adaspark_attn_pages_t."""
    return _PAGES.pack(k_pages or 0, v_pages or 0, k_scale or 0, v_scale or 0, page_stride, scale_stride, n_pages, page_size, page_format, 0)


def adaspark_attn_prompt(handle: int, q, k, v, cu_q, cu_k, batch: int, n_q: int, n_k: int, out, lse, workspace,
                         workspace_bytes: int, status, stream: Optional[int]):
    st = (_lib or load()).adaspark_attn_prompt(handle, _PROMPT.pack(*q, *k, *v, cu_q or 0, cu_k or 0, out or 0, lse or 0, workspace or 0, workspace_bytes,
                                                                    status or 0, batch, n_q, n_k, 0), stream)
    if st != OK:
        _check(handle, st)


def adaspark_attn_paged_write(handle: int, pages: bytes, k, v, cu, batch: int, n: int, block_table, table_width: int, kv_len,
                              status, stream: Optional[int]):
    st = (_lib or load()).adaspark_attn_paged_write(handle, pages + _PAGED_ROWS.pack(*k, *v, cu or 0, kv_len or 0, block_table or 0, status or 0, batch, n,
                                                                                     table_width, 0), stream)
    if st != OK:
        _check(handle, st)


def adaspark_attn_paged_read(handle: int, pages: bytes, k, v, cu, batch: int, n: int, block_table, table_width: int, kv_len,
                             status, stream: Optional[int]):
    st = (_lib or load()).adaspark_attn_paged_read(handle, pages + _PAGED_ROWS.pack(*k, *v, cu or 0, kv_len or 0, block_table or 0, status or 0, batch, n,
                                                                                    table_width, 0), stream)
    if st != OK:
        _check(handle, st)


def adaspark_attn_paged_decode(handle: int, q, k_new, v_new, pages: bytes, block_table, table_width: int, kv_len, batch: int, out, lse,
                               workspace, workspace_bytes: int, status, stream: Optional[int]):
    st = (_lib or load()).adaspark_attn_paged_decode(handle, pages + _PAGED_DECODE.pack(*q, *k_new, *v_new, kv_len or 0, block_table or 0, out or 0, lse or 0,
                                                                                        workspace or 0, workspace_bytes, status or 0, batch, table_width), stream)
    if st != OK:
        _check(handle, st)


def adaspark_attn_paged_decode_window(handle: int, q, k_new, v_new, pages: bytes, block_table, table_width: int, kv_len, batch: int, out, lse,
                                      workspace, workspace_bytes: int, status, window: int, sinks: int, stream: Optional[int]):
    try:
        call = pages + _PAGED_DECODE.pack(*q, *k_new, *v_new, kv_len or 0, block_table or 0, out or 0, lse or 0, workspace or 0, workspace_bytes, status or 0, batch,
                                          table_width) + _WINDOW.pack(window, sinks)
    except struct.error as e:
        _refuse(f"paged_decode_window: window {window}, sinks {sinks}: {e}")
    st = (_lib or load()).adaspark_attn_paged_decode_window(handle, call, stream)
    if st != OK:
        _check(handle, st)


def adaspark_attn_paged_prompt(handle: int, q, pages: bytes, cu, batch: int, n: int, block_table, table_width: int, kv_len, window: int, sinks: int,
                               out, lse, workspace, workspace_bytes: int, status, stream: Optional[int]):
    try:
        call = pages + _PAGED_PROMPT.pack(*q, cu or 0, kv_len or 0, block_table or 0, out or 0, lse or 0, workspace or 0, workspace_bytes, status or 0, batch, n, table_width,
                                          window, sinks, 0)
    except struct.error as e:
        _refuse(f"paged_prompt: window {window}, sinks {sinks}: {e}")
    st = (_lib or load()).adaspark_attn_paged_prompt(handle, call, stream)
    if st != OK:
        _check(handle, st)


def adaspark_attn_rotary_init(radians, axis, axes: int, adjacent: bool) -> RotaryStruct:
    """The rotation of pairs that turn by radians[i] per position on axis[i] (None: axis 0)."""
    got, n = RotaryStruct(), len(radians)
    st = load().adaspark_attn_rotary_init(ctypes.byref(got), (ctypes.c_double * max(n, 1))(*radians),
                                          (ctypes.c_int32 * max(n, 1))(*axis) if axis is not None else None, n, axes, int(adjacent))
    if st != OK:
        raise AdasparkError(st, f"adaspark_attn_rotary_init: {n} pairs on {axes} axes: not a multiple of 8 up to 64, a frequency that is no number, or an axis that is none")
    return got


def adaspark_attn_rotate(handle: int, q, k, q_out, k_out, positions, rotary: Optional[int], q_norm, k_norm, eps: float, n: int, stream: Optional[int]):
    """rotary: address of a RotaryStruct, or None."""
    try:
        call = _ROTATE.pack(*q, *k, *q_out, *k_out, positions or 0, rotary or 0, q_norm or 0, k_norm or 0, eps, n)
    except (struct.error, OverflowError) as e:
        _refuse(f"rotate: eps {eps}: {e}")
    st = (_lib or load()).adaspark_attn_rotate(handle, call, stream)
    if st != OK:
        _check(handle, st)


def adaspark_attn_paged_append(handle: int, q, k, v, q_out, pages: bytes, cu, batch: int, n: int, block_table, table_width: int, kv_len, positions,
                               rotary: Optional[int], q_norm, k_norm, eps: float, status, stream: Optional[int]):
    try:
        call = pages + _PAGED_APPEND.pack(*q, *k, *v, *q_out, cu or 0, kv_len or 0, block_table or 0, positions or 0, rotary or 0, q_norm or 0, k_norm or 0, status or 0, eps, batch,
                                          n, table_width)
    except (struct.error, OverflowError) as e:
        _refuse(f"paged_append: eps {eps}: {e}")
    st = (_lib or load()).adaspark_attn_paged_append(handle, call, stream)
    if st != OK:
        _check(handle, st)


class WorkspaceHeader(ctypes.Structure):
    _fields_ = [("status", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("executed_kv_blocks", ctypes.c_uint64), ("decode_kv_blocks", ctypes.c_uint64),
                ("fallback_rows", ctypes.c_uint32), ("max_tile_kv_blocks", ctypes.c_uint32),
                ("gather_entries", ctypes.c_uint32), ("gather_items", ctypes.c_uint32),
                ("gather_pair_tiles", ctypes.c_uint32), ("reserved2", ctypes.c_uint32)]


# ---- a small convenience owner of the handle and of the caller-side buffers --------------------

def _raw_stream(index: int) -> int:
    """The current stream of a device, as torch hands it to its own generated code: 0.1 us instead of 2 for the stream object."""
    return torch._C._cuda_getCurrentRawStream(index)


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
        self.device, self.index = k_pages.device, k_pages.get_device()
        self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = k_pages.shape
        self.page_stride = stride_of(k_pages, v_pages)
        self.pages = pages_struct(k_pages.data_ptr(), v_pages.data_ptr(), k_scale.data_ptr() if fmt else None,
                                  v_scale.data_ptr() if fmt else None, self.page_stride, stride_of(k_scale, v_scale) if fmt else 0,
                                  self.n_pages, self.page_size, fmt)

    def __reduce__(self):                                      # (a copy has the addresses of its own tensors)
        return type(self), (self.k_pages, self.v_pages, self.k_scale, self.v_scale)


class Rotary:
    """A rotation of a head's pairs by the positions of its token (see adaspark_attn_rotary_t).  sections: how many pairs follow each axis of
    the positions, one axis behind the other (default: all head_dim / 2 on one), pair i turning by theta^(-i / pairs) per position; frequencies and
    axis give every pair's own radians per position, and axis, instead (scaled or interleaved rotations).  adjacent: pairs are neighbours (2 i, 2 i + 1),
    else (i, i + pairs)."""

    def __init__(self, head_dim: int, *, sections=None, theta: float = 1e4, frequencies=None, axis=None, adjacent: bool = False):
        if frequencies is None:
            if axis is not None:
                _refuse("Rotary: axis comes with frequencies")
            sections = [head_dim // 2] if sections is None else [int(n) for n in sections]
            if not sections or min(sections) < 0 or not float(theta) > 0:
                _refuse(f"Rotary: sections {sections}, theta {theta}")
            n = sum(sections)
            frequencies, axis = [float(theta) ** (-i / n) for i in range(n)], [a for a, m in enumerate(sections) for _ in range(m)]
            axes = len(sections)
        else:
            if sections is not None:
                _refuse("Rotary: sections or frequencies, not both")
            frequencies = [float(f) for f in frequencies]
            axis = None if axis is None else [int(a) for a in axis]
            if axis is not None and len(axis) != len(frequencies):
                _refuse(f"Rotary: {len(axis)} axes for {len(frequencies)} frequencies")
            axes = 1 + max(axis, default=0) if axis else 1
        if 2 * len(frequencies) > head_dim:
            _refuse(f"Rotary: {len(frequencies)} pairs in a head of {head_dim}")
        self.struct = adaspark_attn_rotary_init(frequencies, axis, axes, adjacent)
        self.axes, self.pairs, self.head_dim = axes, len(frequencies), head_dim

    @property
    def address(self) -> int:                                  # (worked out anew: a copy has a struct of its own)
        return ctypes.addressof(self.struct)


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
        self._index, self._n_q_heads, self._n_kv_heads, self._head_dim = device, n_q_heads, n_kv_heads, head_dim

    def _capturing(self, stream=None) -> bool:
        """Is a stream (None: the current one of this object's device) in capture?"""
        with torch.cuda.device(self.device), torch.cuda.stream(stream):
            return torch.cuda.is_current_stream_capturing()

    def _empty(self, shape, dtype, stream):
        """An output of a call on `stream`: memory of that stream, whose earlier uses it comes behind, and not handed on before the current stream
        has come to the end of what it does with it, either."""
        if stream is None or stream.cuda_stream == _raw_stream(self._index):
            return torch.empty(shape, dtype=dtype, device=self.device)
        with torch.cuda.stream(stream):
            t = torch.empty(shape, dtype=dtype, device=self.device)
        t.record_stream(torch.cuda.current_stream(self.device))
        return t

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
        if not self._capturing():
            torch.cuda.current_stream(dev).synchronize()             # what used this memory before; calls may be on any stream
        self._streams = {_raw_stream(self._index)}
        return self

    def _use(self, stream):
        """A video call on `stream` (None: torch's current one).  The first time that one is seen, torch's allocator is told that it uses the
        caches and the workspace, which are not handed on before it has come to the end of its calls then."""
        raw = _raw_stream(torch.cuda.current_device()) if stream is None else stream.cuda_stream
        if raw not in self._streams:
            for t in (self.k_cube, self.v_cube, self.cube_keys, self.workspace):
                t.record_stream(torch.cuda.current_stream() if stream is None else stream)
            self._streams.add(raw)

    def forward(self, q, k, v, n_text, *, out=None, want_selection=False, stream=None, n_prefix=0):
        """q may be None: builds only the caches.  Returns (out, sel_bitmap, sel_count).
        n_prefix > 0: the first n_prefix tokens of the tensors are text that precedes the video."""
        lay = self.layout
        self._use(stream)
        bitmap = count = None
        if q is not None:
            if out is None:
                out = self._empty(q.shape, q.dtype, stream)
            if want_selection:
                B, S, Hq, _ = q.shape
                bitmap = self._empty((B, Hq, S, lay.bitmap_words), torch.int32, stream)
                count = self._empty((B, Hq, S), torch.int32, stream)
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
        self._use(stream)
        adaspark_attn_forward_host(self.handle, q_host, k_host, v_host, n_text, out_host, qd, kd, vd, od,
                                   self.k_cube, self.v_cube, self.cube_keys, self.workspace, self.ws_bytes, stream)
        return out_host

    def forward_chunk(self, q, k, v, frame_begin, frame_count, n_text, *, out=None, want_selection=False,
                      stream=None):
        """One chunk of a chunked prefill (n_text < 0: more video follows).  q may be None."""
        lay = self.layout
        self._use(stream)
        bitmap = count = None
        if q is not None:
            if out is None:
                out = self._empty(q.shape, q.dtype, stream)
            if want_selection:
                B, S, Hq, _ = q.shape
                bitmap = self._empty((B, Hq, S, lay.bitmap_words), torch.int32, stream)
                count = self._empty((B, Hq, S), torch.int32, stream)
        adaspark_attn_forward_chunk(self.handle, q, k, v, frame_begin, frame_count, n_text, out, self.k_cube,
                                    self.v_cube, self.cube_keys, bitmap, count, self.workspace, self.ws_bytes,
                                    stream)
        return out, bitmap, count

    def decode(self, q_new, k_new, v_new, text_len, *, out=None, want_selection=False, stream=None):
        lay = self.layout
        self._use(stream)
        if out is None:
            out = self._empty(q_new.shape, q_new.dtype, stream)
        bitmap = None
        if want_selection:
            B, _, Hq, _ = q_new.shape
            bitmap = self._empty((B, Hq, lay.bitmap_words), torch.int32, stream)
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

    def _text_buffers(self, stream):
        """(status pointer, workspace pointer, workspace bytes) of the text calls, made once.  Waits for the stream that they are made on, so
        that a call on any stream comes behind the clearing of the status and whatever used this memory before."""
        if self._capturing() or (stream is not None and self._capturing(stream)):
            _refuse("the first text call of an object allocates its workspace: make one before a capture begins")
        n = adaspark_attn_text_workspace_bytes(self.handle)
        self._text_ws = torch.empty(n, dtype=torch.uint8, device=self.device)
        self._text_flag = torch.zeros(1, dtype=torch.int32, device=self.device)
        torch.cuda.current_stream(self.device).synchronize()
        self._text_streams = {_raw_stream(self._index)}
        self._text = (self._text_flag.data_ptr(), self._text_ws.data_ptr(), n)
        return self._text

    def text_status(self) -> int:
        """What the text calls of this object found wrong on the device since the last look: 0 = nothing.  Waits for the device, whatever
        streams the calls are on (so not inside a capture), and for the clearing of what it returns."""
        if self._text is None:
            return 0
        if self._capturing():
            _refuse("text_status waits for the device: not inside a capture")
        torch.cuda.synchronize(self.device)
        got = int(self._text_flag.item())
        if got:
            self._text_flag.zero_()
            torch.cuda.current_stream(self.device).synchronize()
        return got

    def _stream(self, stream):
        """The stream of a text call for the C entry.  The first time that one is seen, torch's allocator is told that it uses the workspace and
        the status, which are not handed on before it has come to the end of its calls then."""
        raw = _raw_stream(self._index) if stream is None else stream.cuda_stream
        if raw not in self._text_streams:
            for t in (self._text_ws, self._text_flag):
                t.record_stream(torch.cuda.current_stream(self.device) if stream is None else stream)
            self._text_streams.add(raw)
        return raw or None

    def _rows(self, t, heads: int, what: str):
        """(pointer, token stride, head stride) of a bf16 tensor [rows, heads, head_dim] on this device, and its rows."""
        shape, strides = t.shape, t.stride()
        if len(shape) == 3:                                    # (in one go: what is wrong is worked out below)
            n, h, d = shape
            s0, s1, s2 = strides
            if h == heads and d == self._head_dim and s2 == 1 and t.dtype is _BF16 and t.get_device() == self._index and \
                    (s0 >= d or n <= 1) and (s1 >= d or heads == 1):
                # (the stride of an axis of one entry says nothing)
                return (t.data_ptr(), s0 if n > 1 else 0, s1 if heads > 1 else 0), n
        if t.dtype is not _BF16 or len(shape) != 3 or shape[1] != heads or shape[2] != self._head_dim:
            _refuse(f"{what}: {t.dtype} {tuple(shape)} is not bfloat16 [rows, {heads}, {self._head_dim}]")
        if t.get_device() != self._index:
            _refuse(f"{what} is on {t.device}, not on {self.device}")
        _refuse(f"{what}: the values of a row have to lie side by side, and rows apart (strides {tuple(strides)})")   # (0 would say dense)

    def _dense(self, t, shape, dtype, what: str) -> int:
        if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != self._index:
            _refuse(f"{what}: {t.dtype} {tuple(t.shape)} on {t.device} is not dense {dtype} {tuple(shape)} on {self.device}")
        return t.data_ptr()

    def _ints(self, t, n: int, what: str) -> int:
        if t.dtype is not torch.int32 or t.shape != (n,) or not t.is_contiguous() or t.get_device() != self._index:
            _refuse(f"{what}: {t.dtype} {tuple(t.shape)} on {t.device} is not dense int32 [{n}] on {self.device}")
        return t.data_ptr()

    def _tables(self, block_table, kv_len):
        """(batch, pointer of the block table, its width, pointer of kv_len)."""
        shape = block_table.shape
        if block_table.dtype is not torch.int32 or len(shape) != 2 or not block_table.is_contiguous() or block_table.get_device() != self._index:
            _refuse(f"block_table: {block_table.dtype} {tuple(shape)} on {block_table.device} is not dense int32 [batch, pages] on {self.device}")
        return shape[0], block_table.data_ptr(), shape[1], self._ints(kv_len, shape[0], "kv_len")

    def _cache(self, cache: PagedCache) -> bytes:
        if cache.n_kv_heads != self._n_kv_heads or cache.head_dim != self._head_dim or cache.index != self._index:
            _refuse(f"cache of {cache.n_kv_heads} heads of {cache.head_dim} on {cache.device}: not this handle's")
        return cache.pages

    def _turn(self, rotary, positions, n: int, q_norm, k_norm):
        """(positions, rotary, weights of the norms) of n tokens as pointers."""
        where = turned = None
        axes = 1
        if rotary is not None:
            if rotary.head_dim != self._head_dim:
                _refuse(f"rotary is one of heads of {rotary.head_dim}")
            turned, axes = rotary.address, rotary.axes
        if positions is not None:
            shape = positions.shape
            if positions.dtype is not _INT32 or (shape != (axes, n) and (axes != 1 or shape != (n,))) or not positions.is_contiguous() or \
                    positions.get_device() != self._index:
                _refuse(f"positions: {positions.dtype} {tuple(shape)} on {positions.device} is not dense int32 [{axes}, {n}] on {self.device}")
            where = positions.data_ptr()
        if q_norm is not None:
            q_norm = self._dense(q_norm, (self._head_dim,), _BF16, "q_norm")
        if k_norm is not None:
            k_norm = self._dense(k_norm, (self._head_dim,), _BF16, "k_norm")
        return where, turned, q_norm, k_norm

    def rotate(self, q, k, positions=None, rotary: Optional[Rotary] = None, *, q_norm=None, k_norm=None, eps: float = 1e-6, q_out=None, k_out=None, stream=None):
        """Queries [n, Hq, D] and keys [n, Hkv, D] (either may be None), each head with its norm (q_norm, k_norm: bf16 [D]) and turned by its
        positions, int32 [n] or [axes, n].  Outputs may be the inputs themselves.  Returns (q_out, k_out)."""
        Hq, Hkv = self._n_q_heads, self._n_kv_heads
        qr = qo = kr = ko = _NO_ROWS
        if q is not None:
            qr, n = self._rows(q, Hq, "q")
            if q_out is None:
                q_out = self._empty((n, Hq, self._head_dim), _BF16, stream)
            qo, n_q = self._rows(q_out, Hq, "q_out")
        elif q_out is not None:
            _refuse("q_out without q")
        if k is not None:
            kr, n_k = self._rows(k, Hkv, "k")
            if k_out is None:
                k_out = self._empty((n_k, Hkv, self._head_dim), _BF16, stream)
            ko, n_o = self._rows(k_out, Hkv, "k_out")
            if n_o != n_k:
                _refuse(f"k_out has {n_o} rows, k {n_k}")
            if q is None:
                n = n_q = n_k
            elif n_k != n:
                _refuse(f"q has {n} rows, k {n_k}")
        elif k_out is not None:
            _refuse("k_out without k")
        elif q is None:
            _refuse("rotate: neither q nor k")
        if n_q != n:
            _refuse(f"q_out has {n_q} rows, q {n}")
        if rotary is not None and positions is None and rotary.pairs:
            _refuse("rotate: a rotation needs positions")
        where, turned, q_norm, k_norm = self._turn(rotary, positions, n, q_norm, k_norm)
        adaspark_attn_rotate(self.handle, qr, kr, qo, ko, where, turned, q_norm, k_norm, eps, n, _raw_stream(self._index) if stream is None else stream.cuda_stream)
        return q_out, k_out

    def paged_append(self, cache: PagedCache, q, k, v, cu, block_table, kv_len, rotary: Optional[Rotary] = None, *, positions=None, q_norm=None, k_norm=None,
                     eps: float = 1e-6, q_out=None, stream=None):
        """rotate() on the way into the pages: packed rows as paged_write() takes them, keys with their norm and turned, values as they are; q (may
        be None) comes back.  positions None: places in the sequence.  Returns q_out."""
        status = (self._text or self._text_buffers(stream))[0]
        (kr, n), (vr, n_v) = self._rows(k, self._n_kv_heads, "k"), self._rows(v, self._n_kv_heads, "v")
        qr = qo = _NO_ROWS
        n_q = n_o = n
        if q is not None:
            qr, n_q = self._rows(q, self._n_q_heads, "q")
            if q_out is None:
                q_out = self._empty((n_q, self._n_q_heads, self._head_dim), torch.bfloat16, stream)
            qo, n_o = self._rows(q_out, self._n_q_heads, "q_out")
        elif q_out is not None:
            _refuse("q_out without q")
        if n_v != n or n_q != n or n_o != n:
            _refuse(f"q, k, v and q_out have {n_q}, {n}, {n_v} and {n_o} rows")
        batch, table, width, lens = self._tables(block_table, kv_len)
        adaspark_attn_paged_append(self.handle, qr, kr, vr, qo, self._cache(cache), self._ints(cu, batch + 1, "cu"), batch, n, table, width, lens,
                                   *self._turn(rotary, positions, n, q_norm, k_norm), eps, status, self._stream(stream))
        return q_out

    def paged_prompt(self, q, cache: PagedCache, cu, block_table, kv_len, *, window: int = 0, sinks: int = 0, out=None, lse=None, want_lse=False, stream=None):
        """Several new tokens per sequence, in the pages already (paged_append, paged_write): the rows cu[b] .. cu[b + 1] - 1 of q [n, Hq, D] are
        the last tokens of sequence b, which holds kv_len[b].  A token sees those up to itself; with a window, the last `window` of them and the
        first `sinks` ones of the sequence.  Returns (out, lse)."""
        status, ws, ws_bytes = self._text or self._text_buffers(stream)
        Hq, D = self._n_q_heads, self._head_dim
        batch, table, width, lens = self._tables(block_table, kv_len)
        qr, n = self._rows(q, Hq, "q")
        if out is None:
            out = self._empty((n, Hq, D), torch.bfloat16, stream)
        if lse is None and want_lse:
            lse = self._empty((n, Hq), torch.float32, stream)
        adaspark_attn_paged_prompt(self.handle, qr, self._cache(cache), self._ints(cu, batch + 1, "cu"), batch, n, table, width, lens, window, sinks,
                                   self._dense(out, (n, Hq, D), torch.bfloat16, "out"),
                                   None if lse is None else self._dense(lse, (n, Hq), torch.float32, "lse"), ws, ws_bytes, status,
                                   self._stream(stream))
        return out, lse

    def prompt(self, q, k, v, cu_q, cu_k=None, *, out=None, lse=None, want_lse=False, stream=None):
        """Causal attention of packed prompts: q [n_q, Hq, D], k and v [n_k, Hkv, D] bf16, cu_q (and cu_k, if the keys of a sequence
        are more than its queries) int32 [batch + 1].  Returns (out, lse); lse is None unless given or wanted.  The text calls of one
        object share a workspace: calls that may overlap on the GPU (other streams, graphs replayed side by side) need an object each."""
        status, ws, ws_bytes = self._text or self._text_buffers(stream)
        Hq, D = self._n_q_heads, self._head_dim
        (qr, n_q), (kr, n_k), (vr, n_v) = self._rows(q, Hq, "q"), self._rows(k, self._n_kv_heads, "k"), self._rows(v, self._n_kv_heads, "v")
        if n_v != n_k:
            _refuse(f"v has {n_v} rows, k {n_k}")
        n_cu = cu_q.numel()
        cq = self._ints(cu_q, n_cu, "cu_q")
        if n_cu == 0:
            _refuse("cu_q: batch + 1 entries are needed")
        if out is None:
            out = self._empty((n_q, Hq, D), torch.bfloat16, stream)
        if lse is None and want_lse:
            lse = self._empty((n_q, Hq), torch.float32, stream)
        adaspark_attn_prompt(self.handle, qr, kr, vr, cq, cq if cu_k is None else self._ints(cu_k, n_cu, "cu_k"), n_cu - 1, n_q, n_k,
                             self._dense(out, (n_q, Hq, D), torch.bfloat16, "out"),
                             None if lse is None else self._dense(lse, (n_q, Hq), torch.float32, "lse"), ws, ws_bytes, status,
                             self._stream(stream))
        return out, lse

    def paged_write(self, cache: PagedCache, k, v, cu, block_table, kv_len, *, stream=None):
        """Packed keys and values into the pages: the rows cu[b] .. cu[b + 1] - 1 become the last tokens of sequence b, which
        then holds kv_len[b].  block_table int32 [batch, width].  No two rows of a call may have the same place: it would hold a mixture."""
        self._paged_rows(adaspark_attn_paged_write, cache, k, v, cu, block_table, kv_len, stream)

    def paged_read(self, cache: PagedCache, cu, block_table, kv_len, k_out, v_out, *, stream=None):
        """The last cu[b + 1] - cu[b] tokens of every sequence from the pages into k_out, v_out: bf16 [n, Hkv, D].  Returns them."""
        self._paged_rows(adaspark_attn_paged_read, cache, k_out, v_out, cu, block_table, kv_len, stream)
        return k_out, v_out

    def _paged_rows(self, call, cache, k, v, cu, block_table, kv_len, stream):
        status = (self._text or self._text_buffers(stream))[0]
        (kr, n), (vr, n_v) = self._rows(k, self._n_kv_heads, "k"), self._rows(v, self._n_kv_heads, "v")
        if n_v != n:
            _refuse(f"v has {n_v} rows, k {n}")
        batch, table, width, lens = self._tables(block_table, kv_len)
        call(self.handle, self._cache(cache), kr, vr, self._ints(cu, batch + 1, "cu"), batch, n, table, width, lens, status, self._stream(stream))

    def paged_decode(self, q, k_new, v_new, cache: PagedCache, block_table, kv_len, *, window: int = 0, sinks: int = 0, out=None, lse=None,
                     want_lse=False, stream=None):
        """One new token per sequence against its pages.  q [batch, Hq, D]; k_new, v_new [batch, Hkv, D] are stored as token
        kv_len[b] - 1 first (None: they are there).  kv_len 0: a slot without a sequence.  window > 0: against the last `window` tokens
        (itself among them) and the first `sinks` ones.  Returns (out, lse)."""
        status, ws, ws_bytes = self._text or self._text_buffers(stream)
        Hq, D = self._n_q_heads, self._head_dim
        batch, table, width, lens = self._tables(block_table, kv_len)
        qr, n = self._rows(q, Hq, "q")
        kr = vr = _NO_ROWS
        n_k = n_v = batch
        if k_new is not None and v_new is not None:
            (kr, n_k), (vr, n_v) = self._rows(k_new, self._n_kv_heads, "k_new"), self._rows(v_new, self._n_kv_heads, "v_new")
        elif k_new is not None or v_new is not None:
            _refuse("k_new and v_new come together")
        if n != batch or n_k != batch or n_v != batch:
            _refuse(f"q, k_new and v_new hold a row for each of the {batch} entries of kv_len")
        if out is None:
            out = self._empty((batch, Hq, D), torch.bfloat16, stream)
        if lse is None and want_lse:
            lse = self._empty((batch, Hq), torch.float32, stream)
        call = (self.handle, qr, kr, vr, self._cache(cache), table, width, lens, batch, self._dense(out, (batch, Hq, D), torch.bfloat16, "out"),
                None if lse is None else self._dense(lse, (batch, Hq), torch.float32, "lse"), ws, ws_bytes, status)
        if window == 0:
            if sinks < 0:
                _refuse(f"sinks {sinks}")
            adaspark_attn_paged_decode(*call, self._stream(stream))
        else:
            adaspark_attn_paged_decode_window(*call, window, sinks, self._stream(stream))
        return out, lse

    def header(self) -> WorkspaceHeader:
        """Copy of the workspace header of the last call (waits for the device, whatever stream that call is on)."""
        torch.cuda.synchronize(self.device)
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
