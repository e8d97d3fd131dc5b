"""Thin ctypes binding over libvlcache.so: argument marshalling only.

Every function has the name and argument order of its C-ABI entry point (include/vlcache.h).
Tensors are torch CUDA tensors (PyTorch is used for device memory and streams only); their
data_ptr() is handed to the library together with torch's current stream.  Nothing here
computes: if the shared library is missing, importing this module raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libvlcache.so")

VLC_OK, VLC_ERR_INVALID_ARG, VLC_ERR_SHAPE, VLC_ERR_DTYPE, VLC_ERR_CAPACITY, VLC_ERR_HIP, VLC_ERR_UNIMPLEMENTED = range(7)
VLC_F32, VLC_BF16 = 0, 1
STATUS_NAMES = ["VLC_OK", "VLC_ERR_INVALID_ARG", "VLC_ERR_SHAPE", "VLC_ERR_DTYPE", "VLC_ERR_CAPACITY",
                "VLC_ERR_HIP", "VLC_ERR_UNIMPLEMENTED"]


class VlcError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES[status] if 0 <= status < len(STATUS_NAMES) else status}: {message}")
        self.status = status


class vlc_shape(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("B", "L", "Hq", "Hkv", "d", "m", "tau", "dtype")] + [("lens", C.c_void_p)] +
                [("flags", C.c_int32), ("reserved", C.c_int32)])


class vlc_cache_layout(C.Structure):
    _fields_ = [("status_off", C.c_size_t), ("slot_off_off", C.c_size_t), ("kept_off", C.c_size_t),
                ("kv_off", C.c_size_t), ("idx_off", C.c_size_t), ("scratch_off", C.c_size_t),
                ("total_bytes", C.c_size_t), ("slots_per_request", C.c_int64), ("scale_off", C.c_size_t),
                ("kv_fp8", C.c_int32), ("unit_slots", C.c_int32), ("tail_unit_slots", C.c_int32),
                ("layer_unit_slots", C.c_int32), ("appended_off", C.c_size_t),
                ("list_items_off", C.c_size_t * 3), ("list_index_off", C.c_size_t * 3),
                ("list_by_size", C.c_int32 * 3), ("list_reserved", C.c_int32)]


class vlc_cache_options(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("kv_fp8", "unit_slots", "tail_unit_slots", "layer_unit_slots", "decode_order",
                                         "decode_merge", "decode_zigzag", "gather_rows", "select_fold")] + \
               [("reserved", C.c_int32 * 7)]


VLC_PAGES_PLAIN, VLC_PAGES_FP8, VLC_PAGES_INT8 = 0, 1, 2


class vlc_pages_shape(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("L", "Hq", "Hkv", "d", "page_slots", "n_pages", "dtype", "format")] + \
               [("reserved", C.c_int32 * 4)]


class vlc_pages_layout(C.Structure):
    _fields_ = [(n, C.c_size_t) for n in ("status_off", "counters_off", "k_off", "v_off", "k_scale_off", "v_scale_off",
                                          "total_bytes")]


class vlc_chunk(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("B", "max_pages", "max_new", "max_len")] + \
               [("table", C.c_void_p), ("lens", C.c_void_p), ("reserved", C.c_int32 * 2)]


class vlc_rows(C.Structure):
    _fields_ = [("data", C.c_void_p)] + [(n, C.c_int64) for n in ("layer", "request", "head", "row")]


class vlc_row_stats(C.Structure):
    _fields_ = [("row_max", C.c_void_p), ("row_sum", C.c_void_p)] + [(n, C.c_int64) for n in ("layer", "request", "head")]


def _load() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built: run `python -c 'import __graft_entry__ as g; g.build()'` "
                          "(there is no fallback path)")
    lib = C.CDLL(LIB_PATH)
    vp, sz, i32, i64, f32 = C.c_void_p, C.c_size_t, C.c_int32, C.c_int64, C.c_float
    shp = C.POINTER(vlc_shape)
    lib.vlc_last_error_string.restype = C.c_char_p
    lib.vlc_version.restype = C.c_char_p
    lib.vlc_workspace_bytes.restype = sz
    lib.vlc_workspace_bytes.argtypes = [shp]
    lib.vlc_score.restype = C.c_int
    lib.vlc_score.argtypes = [shp, vp, vp, vp, f32, vp, vp, vp, vp, vp, sz, vp]
    lib.vlc_score_static_max_workspace.restype = sz
    lib.vlc_score_static_max_workspace.argtypes = []
    lib.vlc_score_static.restype = C.c_int
    lib.vlc_score_static.argtypes = [shp, vp, vp, vp, f32, vp, vp, vp, vp, vp]
    lib.vlc_sparsity.restype = C.c_int
    lib.vlc_sparsity.argtypes = [shp, vp, vp, vp, vp, f32, vp, vp, vp, sz, vp]
    lib.vlc_window_attn_workspace_bytes.restype = C.c_int
    lib.vlc_window_attn_workspace_bytes.argtypes = [shp, C.POINTER(sz)]
    lib.vlc_window_attn.restype = C.c_int
    lib.vlc_window_attn.argtypes = [shp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.vlc_score_from_stats.restype = C.c_int
    lib.vlc_score_from_stats.argtypes = [shp, vp, vp, vp, f32, vp, vp, vp, vp, vp]
    lib.vlc_allocate.restype = C.c_int
    lib.vlc_allocate.argtypes = [shp, vp, i64, i64, vp, vp, vp]
    lib.vlc_sparsity_allocate.restype = C.c_int
    lib.vlc_sparsity_allocate.argtypes = [shp, vp, vp, i64, i64, vp, vp, vp]
    lib.vlc_cache_bytes.restype = sz
    lib.vlc_cache_bytes.argtypes = [shp, i32, i64]
    lib.vlc_cache_create.restype = C.c_int
    lib.vlc_cache_create.argtypes = [shp, i32, i64, vp, sz, C.POINTER(vp)]
    lib.vlc_cache_bytes_fp8.restype = sz
    lib.vlc_cache_bytes_fp8.argtypes = [shp, i32, i64]
    lib.vlc_cache_create_fp8.restype = C.c_int
    lib.vlc_cache_create_fp8.argtypes = [shp, i32, i64, vp, sz, C.POINTER(vp)]
    lib.vlc_cache_bytes_opt.restype = sz
    lib.vlc_cache_bytes_opt.argtypes = [shp, i32, i64, C.POINTER(vlc_cache_options)]
    lib.vlc_cache_create_opt.restype = C.c_int
    lib.vlc_cache_create_opt.argtypes = [shp, i32, i64, C.POINTER(vlc_cache_options), vp, sz, C.POINTER(vp)]
    lib.vlc_cache_destroy.restype = None
    lib.vlc_cache_destroy.argtypes = [vp]
    lib.vlc_cache_get_layout.restype = C.c_int
    lib.vlc_cache_get_layout.argtypes = [vp, C.POINTER(vlc_cache_layout)]
    lib.vlc_cache_status.restype = C.c_int
    lib.vlc_cache_status.argtypes = [vp, vp]
    lib.vlc_topk_compact.restype = C.c_int
    lib.vlc_topk_compact.argtypes = [vp, vp, vp, i32, vp, vp, vp, vp]
    lib.vlc_topk_compact_recent_frac.restype = C.c_int
    lib.vlc_topk_compact_recent_frac.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, vp]
    lib.vlc_cache_hit_rate.restype = C.c_int
    lib.vlc_cache_hit_rate.argtypes = [vp, vp, vp, vp, vp]
    lib.vlc_decode_attn.restype = C.c_int
    lib.vlc_decode_attn.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.vlc_decode_attn_steps.restype = C.c_int
    lib.vlc_decode_attn_steps.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp, vp, vp]
    pgs, chk, rows = C.POINTER(vlc_pages_shape), C.POINTER(vlc_chunk), C.POINTER(vlc_rows)
    lib.vlc_pages_bytes.restype = sz
    lib.vlc_pages_bytes.argtypes = [pgs]
    lib.vlc_pages_create.restype = C.c_int
    lib.vlc_pages_create.argtypes = [pgs, vp, sz, C.POINTER(vp)]
    lib.vlc_pages_destroy.restype = None
    lib.vlc_pages_destroy.argtypes = [vp]
    lib.vlc_pages_get_layout.restype = C.c_int
    lib.vlc_pages_get_layout.argtypes = [vp, C.POINTER(vlc_pages_layout)]
    for name in ("vlc_pages_clear", "vlc_pages_status"):
        getattr(lib, name).restype = C.c_int
        getattr(lib, name).argtypes = [vp, vp]
    lib.vlc_pages_write.restype = C.c_int
    lib.vlc_pages_write.argtypes = [vp, chk, i32, i32, rows, rows, vp]
    lib.vlc_pages_read.restype = C.c_int
    lib.vlc_pages_read.argtypes = [vp, chk, i32, i32, i32, i32, rows, rows, vp]
    lib.vlc_pages_attn_workspace_bytes.restype = C.c_int
    lib.vlc_pages_attn_workspace_bytes.argtypes = [vp, chk, i32, C.POINTER(sz)]
    lib.vlc_pages_attn.restype = C.c_int
    lib.vlc_pages_attn.argtypes = [vp, chk, i32, i32, rows, rows, rows, vp, rows, C.POINTER(vlc_row_stats), vp, sz, vp]
    lib.vlc_probe_read_stream.restype = C.c_int
    lib.vlc_probe_read_stream.argtypes = [vp, sz, vp, i32, vp]
    return lib


lib = _load()


def _check(status: int) -> None:
    if status != VLC_OK:
        raise VlcError(status, lib.vlc_last_error_string().decode())


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("tensors handed to libvlcache must be contiguous CUDA tensors")
    return t.data_ptr()


def _stream() -> int:
    # the handle itself: torch.cuda.current_stream() builds a Stream object around it on every call
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


VLC_SHAPE_SCORE_PLAIN_ALU = 1


def make_shape(B, L, Hq, Hkv, d, m, tau, dtype, lens=None, flags=0) -> vlc_shape:
    """lens: optional int32 device tensor [B, 2] of per-request (m_b, tau_b); the caller keeps it alive."""
    code = {torch.float32: VLC_F32, torch.bfloat16: VLC_BF16, "f32": VLC_F32, "bf16": VLC_BF16}.get(dtype, dtype)
    if lens is not None:
        assert lens.dtype == torch.int32 and lens.is_cuda and lens.is_contiguous() and tuple(lens.shape) == (B, 2)
    return vlc_shape(B, L, Hq, Hkv, d, m, tau, code, None if lens is None else lens.data_ptr(), int(flags), 0)


def vlc_version() -> str:
    return lib.vlc_version().decode()


def vlc_last_error_string() -> str:
    return lib.vlc_last_error_string().decode()


def vlc_workspace_bytes(shape: vlc_shape) -> int:
    n = lib.vlc_workspace_bytes(C.byref(shape))
    if n == 0:
        raise VlcError(VLC_ERR_SHAPE, vlc_last_error_string())
    return n


def vlc_score(shape, q_win, k, sm_scale, p, scores, row_max, row_sum, nnz, workspace) -> None:
    _check(lib.vlc_score(C.byref(shape), _ptr(q_win), _ptr(k), _ptr(sm_scale), float(p), _ptr(scores),
                         _ptr(row_max), _ptr(row_sum), _ptr(nnz), _ptr(workspace),
                         0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()))


def vlc_score_static_max_workspace() -> int:
    return lib.vlc_score_static_max_workspace()


def vlc_score_static(shape, q_win, k, sm_scale, p, scores, row_max, row_sum, nnz) -> None:
    _check(lib.vlc_score_static(C.byref(shape), _ptr(q_win), _ptr(k), _ptr(sm_scale), float(p), _ptr(scores),
                                _ptr(row_max), _ptr(row_sum), _ptr(nnz), _stream()))


def vlc_sparsity(shape, q_win, k, sm_scale, row_max, p, nnz, gamma, workspace) -> None:
    _check(lib.vlc_sparsity(C.byref(shape), _ptr(q_win), _ptr(k), _ptr(sm_scale), _ptr(row_max), float(p),
                            _ptr(nnz), _ptr(gamma), _ptr(workspace),
                            0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()))


def vlc_window_attn_workspace_bytes(shape: vlc_shape) -> int:
    n = C.c_size_t(0)
    _check(lib.vlc_window_attn_workspace_bytes(C.byref(shape), C.byref(n)))
    return n.value


def vlc_window_attn(shape, q_win, k, v, sm_scale, out, row_max, row_sum, workspace) -> None:
    _check(lib.vlc_window_attn(C.byref(shape), _ptr(q_win), _ptr(k), _ptr(v), _ptr(sm_scale), _ptr(out),
                               _ptr(row_max), _ptr(row_sum), _ptr(workspace),
                               0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()))


def vlc_score_from_stats(shape, q_win, k, sm_scale, p, row_max, row_sum, scores, nnz) -> None:
    _check(lib.vlc_score_from_stats(C.byref(shape), _ptr(q_win), _ptr(k), _ptr(sm_scale), float(p), _ptr(row_max),
                                    _ptr(row_sum), _ptr(scores), _ptr(nnz), _stream()))


def vlc_allocate(shape, nnz, alpha_num, alpha_den, k_out, beta_out) -> None:
    _check(lib.vlc_allocate(C.byref(shape), _ptr(nnz), int(alpha_num), int(alpha_den), _ptr(k_out),
                            _ptr(beta_out), _stream()))


def vlc_sparsity_allocate(shape, nnz, gamma, alpha_num, alpha_den, k_out, beta_out) -> None:
    _check(lib.vlc_sparsity_allocate(C.byref(shape), _ptr(nnz), _ptr(gamma), int(alpha_num), int(alpha_den), _ptr(k_out),
                                     _ptr(beta_out), _stream()))


def vlc_cache_bytes(shape, T_max, sum_k_max) -> int:
    n = lib.vlc_cache_bytes(C.byref(shape), int(T_max), int(sum_k_max))
    if n == 0:
        raise VlcError(VLC_ERR_INVALID_ARG, vlc_last_error_string())
    return n


def vlc_cache_bytes_fp8(shape, T_max, sum_k_max) -> int:
    n = lib.vlc_cache_bytes_fp8(C.byref(shape), int(T_max), int(sum_k_max))
    if n == 0:
        raise VlcError(VLC_ERR_INVALID_ARG, vlc_last_error_string())
    return n


def make_options(**kw) -> vlc_cache_options:
    """vlc_cache_options with the named fields set and everything else 0 (the library's choice)."""
    o = vlc_cache_options()
    for name, value in kw.items():
        if name == "reserved" or name not in {f[0] for f in vlc_cache_options._fields_}:
            raise ValueError(f"vlc_cache_options has no field {name}")
        setattr(o, name, int(value))
    return o


def vlc_cache_bytes_opt(shape, T_max, sum_k_max, options) -> int:
    n = lib.vlc_cache_bytes_opt(C.byref(shape), int(T_max), int(sum_k_max), None if options is None else C.byref(options))
    if n == 0:
        raise VlcError(VLC_ERR_INVALID_ARG, vlc_last_error_string())
    return n


class Cache:
    """Owns the arena tensor and the library's host-side handle."""

    def __init__(self, shape: vlc_shape, T_max: int, sum_k_max: int, device="cuda", fp8: bool = False,
                 options: Optional[vlc_cache_options] = None):
        if options is None:
            options = make_options(kv_fp8=int(bool(fp8)))
        elif fp8:
            options.kv_fp8 = 1
        self.shape, self.T_max, self.sum_k_max, self.fp8 = shape, int(T_max), int(sum_k_max), bool(options.kv_fp8)
        self.options = options
        nbytes = vlc_cache_bytes_opt(shape, T_max, sum_k_max, options)
        self.arena = torch.empty(nbytes, dtype=torch.uint8, device=device)
        handle = C.c_void_p()
        _check(lib.vlc_cache_create_opt(C.byref(shape), self.T_max, self.sum_k_max, C.byref(options), self.arena.data_ptr(),
                                        nbytes, C.byref(handle)))
        self.handle = handle
        lay = vlc_cache_layout()
        _check(lib.vlc_cache_get_layout(self.handle, C.byref(lay)))
        self.layout = lay

    def close(self) -> None:
        if self.handle:
            lib.vlc_cache_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def vlc_cache_create(shape, T_max, sum_k_max, device="cuda") -> Cache:
    return Cache(shape, T_max, sum_k_max, device)


def vlc_cache_create_fp8(shape, T_max, sum_k_max, device="cuda") -> Cache:
    return Cache(shape, T_max, sum_k_max, device, fp8=True)


def vlc_cache_create_opt(shape, T_max, sum_k_max, options, device="cuda") -> Cache:
    return Cache(shape, T_max, sum_k_max, device, options=options)


def vlc_cache_status(cache: Cache) -> None:
    """Synchronises the stream; raises VlcError if the device flagged a budget or capacity error."""
    _check(lib.vlc_cache_status(cache.handle, _stream()))


def vlc_topk_compact(cache: Cache, scores, k, n_recent, k_full, v_full, idx_out) -> None:
    _check(lib.vlc_topk_compact(cache.handle, _ptr(scores), _ptr(k), int(n_recent), _ptr(k_full), _ptr(v_full),
                                _ptr(idx_out), _stream()))


def vlc_topk_compact_recent_frac(cache: Cache, scores, k, recent_num, recent_den, k_full, v_full, idx_out) -> None:
    _check(lib.vlc_topk_compact_recent_frac(cache.handle, _ptr(scores), _ptr(k), int(recent_num), int(recent_den),
                                            _ptr(k_full), _ptr(v_full), _ptr(idx_out), _stream()))


def vlc_cache_hit_rate(cache: Cache, scores_star, hits_out, rate_out) -> None:
    _check(lib.vlc_cache_hit_rate(cache.handle, _ptr(scores_star), _ptr(hits_out), _ptr(rate_out), _stream()))


def vlc_decode_attn(cache: Cache, layer_begin, layer_end, q, k_new, v_new, sm_scale, out) -> None:
    _check(lib.vlc_decode_attn(cache.handle, int(layer_begin), int(layer_end), _ptr(q), _ptr(k_new), _ptr(v_new),
                               _ptr(sm_scale), _ptr(out), _stream()))


def vlc_probe_read_stream(buf, sink, blocks) -> None:
    _check(lib.vlc_probe_read_stream(_ptr(buf), buf.numel() * buf.element_size(), _ptr(sink), int(blocks), _stream()))


def vlc_decode_attn_steps(cache: Cache, layer_begin, layer_end, n_steps, q, k_new, v_new, sm_scale, out) -> None:
    _check(lib.vlc_decode_attn_steps(cache.handle, int(layer_begin), int(layer_end), int(n_steps), _ptr(q),
                                     _ptr(k_new), _ptr(v_new), _ptr(sm_scale), _ptr(out), _stream()))


# ---- the paged prompt cache ---------------------------------------------------------------------------------------
_PAGE_FORMATS = {"plain": VLC_PAGES_PLAIN, "fp8": VLC_PAGES_FP8, "int8": VLC_PAGES_INT8}


def make_pages_shape(L, Hq, Hkv, d, page_slots, n_pages, dtype, format="plain") -> vlc_pages_shape:
    code = {torch.float32: VLC_F32, torch.bfloat16: VLC_BF16, "f32": VLC_F32, "bf16": VLC_BF16}.get(dtype, dtype)
    return vlc_pages_shape(L, Hq, Hkv, d, page_slots, n_pages, code, _PAGE_FORMATS.get(format, format))


def vlc_pages_bytes(shape: vlc_pages_shape) -> int:
    n = lib.vlc_pages_bytes(C.byref(shape))
    if n == 0:
        raise VlcError(VLC_ERR_INVALID_ARG, vlc_last_error_string())
    return n


class Pages:
    """Owns the arena tensor of a paged prompt cache and the library's host-side handle; cleared on the current stream."""

    def __init__(self, shape: vlc_pages_shape, device="cuda"):
        self.handle = None
        self.shape = shape
        self.dtype = torch.float32 if shape.dtype == VLC_F32 else torch.bfloat16
        nbytes = vlc_pages_bytes(shape)
        self.arena = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.device_index = self.arena.get_device()
        handle = C.c_void_p()
        _check(lib.vlc_pages_create(C.byref(shape), self.arena.data_ptr(), nbytes, C.byref(handle)))
        self.handle = handle
        self.layout = vlc_pages_layout()
        _check(lib.vlc_pages_get_layout(self.handle, C.byref(self.layout)))
        vlc_pages_clear(self)

    def close(self) -> None:
        if self.handle:
            lib.vlc_pages_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def vlc_pages_create(shape: vlc_pages_shape, device="cuda") -> Pages:
    return Pages(shape, device)


def vlc_pages_clear(pages: Pages) -> None:
    _check(lib.vlc_pages_clear(pages.handle, _pages_stream(pages)))


def vlc_pages_status(pages: Pages) -> None:
    """Synchronises the stream; raises VlcError if the device flagged lengths or a page out of range."""
    _check(lib.vlc_pages_status(pages.handle, _pages_stream(pages)))


def make_chunk(table: torch.Tensor, max_new: int, max_len: int, lens: Optional[torch.Tensor] = None) -> vlc_chunk:
    """table: int32 device tensor [B, max_pages]; lens: optional int32 device tensor [B, 2] of (n_b, c_b).  Both stay alive
    with the returned structure."""
    if table.dtype != torch.int32 or table.dim() != 2:
        raise ValueError("table must be an int32 tensor [B, max_pages]")
    if lens is not None and (lens.dtype != torch.int32 or tuple(lens.shape) != (table.shape[0], 2)):
        raise ValueError("lens must be an int32 tensor [B, 2]")
    c = vlc_chunk(table.shape[0], table.shape[1], int(max_new), int(max_len), _ptr(table), _ptr(lens))
    c.tensors = (table, lens)
    c.device_index = table.get_device()
    if lens is not None and lens.get_device() != c.device_index:
        raise ValueError("table and lens must lie on one device")
    return c


def _rows(t: Optional[torch.Tensor], name: str, pages: Pages, dims) -> Optional[vlc_rows]:
    """vlc_rows of a tensor [layers, B, heads, rows, d] of any strides, d contiguous."""
    if t is None:
        return None
    if t.dtype is not pages.dtype or t.shape != dims:
        raise ValueError(f"{name} must be {pages.dtype} of shape {dims}, not {t.dtype} {tuple(t.shape)}")
    layer, request, head, row, last = t.stride()
    if t.get_device() != pages.device_index or last != 1:
        raise ValueError(f"{name} must lie on {pages.arena.device} with its last dimension contiguous")
    return vlc_rows(t.data_ptr(), layer, request, head, row)


def _pages_stream(pages: Pages, chunk: Optional[vlc_chunk] = None) -> int:
    if pages.device_index != torch.cuda.current_device():
        raise ValueError(f"the pages lie on {pages.arena.device}, which is not the current device")
    if chunk is not None and chunk.device_index != pages.device_index:
        raise ValueError(f"the chunk's table and lens must lie on {pages.arena.device}")
    return torch._C._cuda_getCurrentRawStream(pages.device_index)


def _ref(r):
    return None if r is None else C.byref(r)


def vlc_pages_write(pages: Pages, chunk: vlc_chunk, layer_begin, layer_end, k_new, v_new) -> None:
    s = pages.shape
    dims = (layer_end - layer_begin, chunk.B, s.Hkv, chunk.max_new, s.d)
    k, v = _rows(k_new, "k_new", pages, dims), _rows(v_new, "v_new", pages, dims)
    st = lib.vlc_pages_write(pages.handle, chunk, layer_begin, layer_end, _ref(k), _ref(v), _pages_stream(pages, chunk))
    if st:
        _check(st)


def vlc_pages_read(pages: Pages, chunk: vlc_chunk, layer_begin, layer_end, first, k_out, v_out) -> None:
    """Reads as many positions from `first` on as k_out and v_out [layers, B, Hkv, count, d] have rows."""
    s = pages.shape
    count = k_out.shape[3]
    dims = (layer_end - layer_begin, chunk.B, s.Hkv, count, s.d)
    k, v = _rows(k_out, "k_out", pages, dims), _rows(v_out, "v_out", pages, dims)
    _check(lib.vlc_pages_read(pages.handle, C.byref(chunk), int(layer_begin), int(layer_end), int(first), int(count), _ref(k), _ref(v),
                              _pages_stream(pages, chunk)))


def vlc_pages_attn_workspace_bytes(pages: Pages, chunk: vlc_chunk, n_layers) -> int:
    n = C.c_size_t(0)
    _check(lib.vlc_pages_attn_workspace_bytes(pages.handle, C.byref(chunk), int(n_layers), C.byref(n)))
    return n.value


def vlc_pages_attn(pages: Pages, chunk: vlc_chunk, layer_begin, layer_end, q, k_new, v_new, sm_scale, out, row_max, row_sum,
                   workspace) -> None:
    """q, out [layers, B, Hq, max_new, d]; k_new, v_new [layers, B, Hkv, max_new, d] or None; row_max, row_sum fp32
    [layers, B, Hq, max_new] of equal strides, or None."""
    s = pages.shape
    n = layer_end - layer_begin
    qd, kd = (n, chunk.B, s.Hq, chunk.max_new, s.d), (n, chunk.B, s.Hkv, chunk.max_new, s.d)
    stats = None
    if (row_max is None) != (row_sum is None):
        raise ValueError("row_max and row_sum come together")
    if row_max is not None:
        for t in (row_max, row_sum):
            if t.dtype != torch.float32 or t.shape != qd[:4] or t.get_device() != pages.device_index:
                raise ValueError(f"row_max and row_sum must be fp32 of shape {qd[:4]} on {pages.arena.device}")
        if row_max.stride() != row_sum.stride() or (chunk.max_new > 1 and row_max.stride(3) != 1):
            raise ValueError("row_max and row_sum must have equal strides and contiguous rows")
        stats = vlc_row_stats(row_max.data_ptr(), row_sum.data_ptr(), *row_max.stride()[:3])
    if sm_scale is not None and (sm_scale.dtype is not torch.float32 or sm_scale.numel() < s.L or sm_scale.get_device() != pages.device_index):
        raise ValueError(f"sm_scale must be fp32 of {s.L} numbers on {pages.arena.device}")
    if workspace is not None and workspace.get_device() != pages.device_index:
        raise ValueError(f"workspace must lie on {pages.arena.device}")
    qr, o = _rows(q, "q", pages, qd), _rows(out, "out", pages, qd)
    k, v = _rows(k_new, "k_new", pages, kd), _rows(v_new, "v_new", pages, kd)
    st = lib.vlc_pages_attn(pages.handle, chunk, layer_begin, layer_end, _ref(qr), _ref(k), _ref(v), _ptr(sm_scale), _ref(o), _ref(stats),
                            _ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(), _pages_stream(pages, chunk))
    if st:
        _check(st)
