"""ctypes binding of the ckv C ABI (include/ckv.h): argument marshalling only.

Every function takes torch tensors that live on the GPU, passes their pointers to the
library and returns; all arithmetic runs in the CUDA kernels.  There is no CPU fallback:
if libckv.so is missing or cannot be loaded the import of this module fails.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from dataclasses import dataclass

import torch

from . import build as _build

F32, BF16 = 0, 1
SELECT_GLOBAL, SELECT_CHUNK = 0, 1
OK = 0

EXPORTS = ["ckv_compress_plan", "ckv_workspace_bytes", "ckv_compress_prefill", "ckv_compress_append", "ckv_compress_append_batch",
           "ckv_decode_workspace_bytes", "ckv_decode_attn", "ckv_status_string", "ckv_workspace_status",
           "ckv_decode_attn_static", "ckv_compress_append_recluster", "ckv_decode_attn_paged", "ckv_pages_gather",
           "ckv_pages_scatter", "ckv_pages_plan", "ckv_paged_workspace_bytes", "ckv_compress_paged",
           "ckv_decode_append_attn_paged", "ckv_pages_resize", "ckv_pages_write", "ckv_pages_summarize", "ckv_pages_select",
           "ckv_decode_attn_selected", "ckv_pages_quantize", "ckv_pages_dequantize", "ckv_decode_quantized_workspace_bytes",
           "ckv_decode_attn_quantized"]

RESIZE_OK, RESIZE_NO_PAGES, RESIZE_TABLE_FULL, RESIZE_SLOTS_FULL, RESIZE_INCONSISTENT = range(5)   # device status of pages_resize


class CkvPagePool(C.Structure):
    _fields_ = [("k_pages", C.c_void_p), ("v_pages", C.c_void_p), ("deg_pages", C.c_void_p), ("logdeg_pages", C.c_void_p)]


class CkvCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("deg", C.c_void_p), ("logdeg", C.c_void_p),
                ("L", C.c_int32), ("H", C.c_int32), ("D", C.c_int32), ("dtype", C.c_int32),
                ("cap", C.c_int64), ("len", C.c_int64), ("pending", C.c_int64)]


class CkvParams(C.Structure):
    _fields_ = [("chunk", C.c_int32), ("n_sink", C.c_int32), ("n_recent", C.c_int32), ("n_rounds_max", C.c_int32),
                ("r_init", C.c_float), ("r_decay", C.c_float), ("r_min", C.c_float), ("select", C.c_int32),
                ("budget", C.c_int64)]


class CkvTokenRows(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("deg", C.c_void_p),
                ("k_token_stride", C.c_int64), ("k_head_stride", C.c_int64), ("v_token_stride", C.c_int64), ("v_head_stride", C.c_int64),
                ("deg_token_stride", C.c_int64), ("deg_head_stride", C.c_int64),
                ("H", C.c_int32), ("D", C.c_int32), ("dtype", C.c_int32)]


class CkvQuantPool(C.Structure):
    _fields_ = [("k_codes", C.c_void_p), ("v_codes", C.c_void_p), ("k_scales", C.c_void_p), ("v_scales", C.c_void_p),
                ("deg_pages", C.c_void_p), ("logdeg_pages", C.c_void_p)]


class CkvLayerView(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("logdeg", C.c_void_p), ("len", C.c_int64), ("cap", C.c_int64)]


def _load():
    path = _build.LIB
    if not os.path.exists(path):
        path = _build.build()
    lib = C.CDLL(path)
    lib.ckv_status_string.restype = C.c_char_p
    lib.ckv_status_string.argtypes = [C.c_int]
    lib.ckv_compress_plan.restype = C.c_int
    lib.ckv_compress_plan.argtypes = [C.c_int64, C.POINTER(CkvParams), C.POINTER(C.c_int64), C.POINTER(C.c_int64),
                                      C.POINTER(C.c_int64)]
    lib.ckv_workspace_bytes.restype = C.c_size_t
    lib.ckv_workspace_bytes.argtypes = [C.POINTER(CkvCache), C.POINTER(CkvParams)]
    lib.ckv_compress_prefill.restype = C.c_int
    lib.ckv_compress_prefill.argtypes = [C.POINTER(CkvCache), C.POINTER(CkvCache), C.POINTER(CkvParams), C.c_void_p,
                                         C.c_void_p, C.c_size_t, C.c_void_p, C.POINTER(C.c_int64)]
    lib.ckv_compress_append.restype = C.c_int
    lib.ckv_compress_append.argtypes = [C.POINTER(CkvCache), C.c_void_p, C.c_void_p, C.c_int32, C.POINTER(CkvParams),
                                        C.c_void_p, C.c_size_t, C.c_void_p]
    lib.ckv_compress_append_batch.restype = C.c_int
    lib.ckv_compress_append_batch.argtypes = [C.POINTER(CkvCache), C.c_int32, C.c_void_p, C.c_void_p, C.POINTER(CkvParams),
                                              C.c_void_p, C.c_size_t, C.c_void_p]
    lib.ckv_compress_append_recluster.restype = C.c_int
    lib.ckv_compress_append_recluster.argtypes = [C.POINTER(CkvCache), C.POINTER(CkvCache), C.c_void_p, C.c_void_p, C.c_int32,
                                                  C.POINTER(CkvParams), C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p,
                                                  C.POINTER(C.c_int64)]
    lib.ckv_decode_attn_paged.restype = C.c_int
    lib.ckv_decode_attn_paged.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                          C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_float, C.c_int64, C.c_void_p, C.c_size_t,
                                          C.c_void_p]
    lib.ckv_pages_gather.restype = C.c_int
    lib.ckv_pages_gather.argtypes = [C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32,
                                     C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]
    lib.ckv_pages_scatter.restype = C.c_int
    lib.ckv_pages_scatter.argtypes = [C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_int32,
                                      C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.ckv_decode_append_attn_paged.restype = C.c_int
    lib.ckv_decode_append_attn_paged.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32,
                                                 C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_float,
                                                 C.c_int64, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.ckv_pages_plan.restype = C.c_int
    lib.ckv_pages_plan.argtypes = [C.c_int64, C.POINTER(CkvParams), C.c_int32, C.POINTER(C.c_int64), C.POINTER(C.c_int64),
                                   C.POINTER(C.c_int64), C.POINTER(C.c_int32), C.POINTER(C.c_int64)]
    lib.ckv_paged_workspace_bytes.restype = C.c_size_t
    lib.ckv_paged_workspace_bytes.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int64, C.POINTER(CkvParams)]
    lib.ckv_compress_paged.restype = C.c_int
    lib.ckv_compress_paged.argtypes = [C.POINTER(CkvPagePool), C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p,
                                       C.c_int64, C.c_int32, C.c_void_p, C.c_int64, C.POINTER(CkvParams), C.c_void_p, C.c_size_t,
                                       C.c_void_p, C.POINTER(C.c_int64), C.POINTER(C.c_int32)]
    lib.ckv_workspace_status.restype = C.c_int
    lib.ckv_workspace_status.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(C.c_int32)]
    lib.ckv_decode_workspace_bytes.restype = C.c_size_t
    lib.ckv_decode_workspace_bytes.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int64]
    lib.ckv_decode_attn.restype = C.c_int
    lib.ckv_decode_attn.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p,
                                    C.c_void_p, C.c_float, C.c_int64, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.ckv_decode_attn_static.restype = C.c_int
    lib.ckv_decode_attn_static.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p,
                                           C.c_void_p, C.c_float, C.c_int64, C.c_void_p]
    p, i32, i64, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float
    for name, args in {
            "ckv_pages_resize": [p, p, i32, i32, p, i64, p, i64, p, p, i64, p, p, p, p, p, p],
            "ckv_pages_write": [p, p, i64, p, p, p, p, i64, i32, p],
            "ckv_pages_summarize": [p, p, i32, p, p, i32, i32, i32, i32, i64, p, p, p],
            "ckv_pages_select": [p, p, p, i32, i32, i32, i32, i32, i32, p, f32, i64, i32, i32, i32, p, p],
            "ckv_decode_attn_selected": [p, p, p, p, i32, p, i32, i32, i32, i32, i32, i32, p, p, f32, p],
            "ckv_pages_quantize": [p, p, i64, p, i64, i32, p],
            "ckv_pages_dequantize": [p, i64, p, i32, i32, i32, i32, p, p, p, p, i64, p],
            "ckv_decode_attn_quantized": [p, p, i32, i32, i32, i32, i32, i32, p, p, f32, i64, p, C.c_size_t, p]}.items():
        getattr(lib, name).restype = C.c_int
        getattr(lib, name).argtypes = args
    lib.ckv_decode_quantized_workspace_bytes.restype = C.c_size_t
    lib.ckv_decode_quantized_workspace_bytes.argtypes = [i32, i32, i32, i32, i64]
    return lib


lib = _load()


class CkvError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        super().__init__(f"ckv status {status}: {lib.ckv_status_string(status).decode()}")


def _check(status: int):
    if status != OK:
        raise CkvError(status)


_DTYPE_CODES = {torch.float32: F32, torch.bfloat16: BF16}


def dtype_code(t: torch.dtype) -> int:
    return _DTYPE_CODES[t]


@dataclass
class Params:
    """Mirror of ckv_params.  Ratios are stored as float32, like the C struct."""
    chunk: int = 256
    n_sink: int = 16
    n_recent: int = 64
    n_rounds_max: int = 8
    r_init: float = 0.8
    r_decay: float = 0.2
    r_min: float = 0.2
    select: int = SELECT_GLOBAL
    budget: int = 0

    def c(self) -> CkvParams:
        return CkvParams(self.chunk, self.n_sink, self.n_recent, self.n_rounds_max, self.r_init, self.r_decay,
                         self.r_min, self.select, self.budget)

    def as_float32(self):
        """(r_init, r_decay, r_min) as the float32 values the library sees."""
        p = self.c()
        return float(p.r_init), float(p.r_decay), float(p.r_min)


def compress_plan(length: int, params: Params):
    """ckv_compress_plan: (final length, rounds, destination capacity needed).  Host only."""
    out_len, rounds, cap = C.c_int64(), C.c_int64(), C.c_int64()
    _check(lib.ckv_compress_plan(length, C.byref(params.c()), C.byref(out_len), C.byref(rounds), C.byref(cap)))
    return out_len.value, rounds.value, cap.value


class Cache:
    """One sequence's cache on the GPU: k, v [L, H, cap, D]; deg int32 and logdeg fp32 [L, H, cap]."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, deg: torch.Tensor | None, logdeg: torch.Tensor | None,
                 length: int, pending: int = 0):
        assert k.is_contiguous() and v.is_contiguous() and k.shape == v.shape and k.dim() == 4
        self.k, self.v, self.deg, self.logdeg = k, v, deg, logdeg
        self.len, self.pending = length, pending

    @classmethod
    def empty(cls, L, H, cap, D, dtype, device="cuda", with_logdeg=True):
        k = torch.empty((L, H, cap, D), dtype=dtype, device=device)
        v = torch.empty_like(k)
        deg = torch.zeros((L, H, cap), dtype=torch.int32, device=device)
        logdeg = torch.zeros((L, H, cap), dtype=torch.float32, device=device) if with_logdeg else None
        return cls(k, v, deg, logdeg, 0)

    @property
    def cap(self):
        return self.k.shape[2]

    def c(self) -> CkvCache:
        L, H, cap, D = self.k.shape
        return CkvCache(self.k.data_ptr(), self.v.data_ptr(),
                        self.deg.data_ptr() if self.deg is not None else None,
                        self.logdeg.data_ptr() if self.logdeg is not None else None,
                        L, H, D, dtype_code(self.k.dtype), cap, self.len, self.pending)


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_ptr():
    """The current CUDA stream as a pointer (the raw-handle query is several times cheaper than building a Stream object,
    which matters for calls that take ten microseconds on the GPU)."""
    if _raw_stream is not None:
        return C.c_void_p(_raw_stream(torch.cuda.current_device()))
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def workspace_bytes(cache: Cache, params: Params) -> int:
    return lib.ckv_workspace_bytes(C.byref(cache.c()), C.byref(params.c()))


def compress_prefill(src: Cache, dst: Cache, params: Params, workspace: torch.Tensor, assign: torch.Tensor | None = None):
    """ckv_compress_prefill on the current stream.  Returns the number of rounds; dst.len is updated."""
    cs, cd, rounds = src.c(), dst.c(), C.c_int64()
    _check(lib.ckv_compress_prefill(C.byref(cs), C.byref(cd), C.byref(params.c()),
                                    assign.data_ptr() if assign is not None else None,
                                    workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream_ptr(),
                                    C.byref(rounds)))
    dst.len, dst.pending = cd.len, cd.pending
    return rounds.value


def compress_append(cache: Cache, k_new: torch.Tensor, v_new: torch.Tensor, params: Params, workspace: torch.Tensor):
    """ckv_compress_append on the current stream; cache.len / cache.pending are updated."""
    assert k_new.is_contiguous() and v_new.is_contiguous() and k_new.shape == v_new.shape
    cc = cache.c()
    _check(lib.ckv_compress_append(C.byref(cc), k_new.data_ptr(), v_new.data_ptr(), k_new.shape[2], C.byref(params.c()),
                                   workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream_ptr()))
    cache.len, cache.pending = cc.len, cc.pending


def compress_append_batch(caches, k_new: torch.Tensor, v_new: torch.Tensor, params: Params, workspace: torch.Tensor):
    """ckv_compress_append_batch on the current stream: one new token for each cache of the list (k_new, v_new:
    [L, H, len(caches), D]); every cache's len / pending are updated."""
    assert k_new.is_contiguous() and v_new.is_contiguous() and k_new.shape == v_new.shape and k_new.shape[2] == len(caches)
    arr = (CkvCache * len(caches))(*[c.c() for c in caches])
    _check(lib.ckv_compress_append_batch(arr, len(caches), k_new.data_ptr(), v_new.data_ptr(), C.byref(params.c()),
                                         workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream_ptr()))
    for c, cc in zip(caches, arr):
        c.len, c.pending = cc.len, cc.pending


def compress_append_recluster(cache: Cache, spare: Cache, k_new: torch.Tensor, v_new: torch.Tensor, params: Params,
                              interval: int, workspace: torch.Tensor) -> int:
    """ckv_compress_append_recluster on the current stream: append, and one clustering round over the whole cache
    whenever it reaches budget + interval tokens.  The two Cache objects trade tensors like the C structs trade
    buffers, so `cache` always holds the live cache.  Returns the number of re-clusterings."""
    assert k_new.is_contiguous() and v_new.is_contiguous() and k_new.shape == v_new.shape
    cc, cs, calls = cache.c(), spare.c(), C.c_int64()
    live_before = cc.k
    _check(lib.ckv_compress_append_recluster(C.byref(cc), C.byref(cs), k_new.data_ptr(), v_new.data_ptr(), k_new.shape[2],
                                             C.byref(params.c()), interval, workspace.data_ptr(),
                                             workspace.numel() * workspace.element_size(), _stream_ptr(), C.byref(calls)))
    if cc.k != live_before:   # an odd number of rounds ran: the tensors trade places
        cache.k, spare.k = spare.k, cache.k
        cache.v, spare.v = spare.v, cache.v
        cache.deg, spare.deg = spare.deg, cache.deg
        cache.logdeg, spare.logdeg = spare.logdeg, cache.logdeg
    cache.len, cache.pending = cc.len, cc.pending
    return calls.value


def workspace_status(workspace: torch.Tensor) -> int:
    """ckv_workspace_status: synchronises the current stream and returns the device status word (0 = fine)."""
    st = C.c_int32(-1)
    _check(lib.ckv_workspace_status(workspace.data_ptr(), _stream_ptr(), C.byref(st)))
    return st.value


def layer_views(caches, layer: int, device="cuda") -> torch.Tensor:
    """Device array of ckv_layer_view for one layer of a batch of caches (as an int64 tensor of 5 words each)."""
    rows = []
    for c in caches:
        L, H, cap, D = c.k.shape
        es = c.k.element_size()
        off = layer * H * cap
        rows.append([c.k.data_ptr() + off * D * es, c.v.data_ptr() + off * D * es,
                     (c.logdeg.data_ptr() + off * 4) if c.logdeg is not None else 0, c.len, cap])
    return torch.tensor(rows, dtype=torch.int64).to(device)


def pages_plan(length: int, params: Params, page_tokens: int):
    """ckv_pages_plan: (final length, rounds, scratch pages needed, result in scratch?, pages kept).  Host only."""
    out_len, rounds, scratch, kept, in_scratch = C.c_int64(), C.c_int64(), C.c_int64(), C.c_int64(), C.c_int32()
    _check(lib.ckv_pages_plan(length, C.byref(params.c()), page_tokens, C.byref(out_len), C.byref(rounds), C.byref(scratch),
                              C.byref(in_scratch), C.byref(kept)))
    return out_len.value, rounds.value, scratch.value, bool(in_scratch.value), kept.value


def paged_workspace_bytes(L: int, H: int, D: int, dtype: torch.dtype, length: int, params: Params) -> int:
    return lib.ckv_paged_workspace_bytes(L, H, D, dtype_code(dtype), length, C.byref(params.c()))


def compress_paged(pools, block_table: torch.Tensor, length: int, has_deg: bool, scratch_table: torch.Tensor, params: Params,
                   workspace: torch.Tensor):
    """ckv_compress_paged on the current stream.  pools: one (k_pages, v_pages, deg_pages, logdeg_pages or None) per layer,
    k_pages [n_pages, H, page_tokens, D].  Returns (final length, result in the scratch table's pages?)."""
    kp = pools[0][0]
    n_pages, H, P, D = kp.shape
    arr = (CkvPagePool * len(pools))(*[CkvPagePool(k.data_ptr(), v.data_ptr(), d.data_ptr(), lg.data_ptr() if lg is not None else None)
                                       for k, v, d, lg in pools])
    out_len, in_scratch = C.c_int64(), C.c_int32()
    _check(lib.ckv_compress_paged(arr, len(pools), H, D, dtype_code(kp.dtype), P, block_table.data_ptr(), length, int(has_deg),
                                  scratch_table.data_ptr() if scratch_table is not None else None,
                                  scratch_table.numel() if scratch_table is not None else 0, C.byref(params.c()),
                                  workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream_ptr(),
                                  C.byref(out_len), C.byref(in_scratch)))
    return out_len.value, bool(in_scratch.value)


def layer_views_all(caches, device="cuda") -> torch.Tensor:
    """[L, Bz, 5] int64: the ckv_layer_view arrays of every layer of a batch of caches, built and copied to the device
    in one go (views[l] is the argument of ckv_decode_attn for layer l)."""
    L = caches[0].k.shape[0]
    base = []
    for c in caches:
        _, H, cap, D = c.k.shape
        base.append([c.k.data_ptr(), c.v.data_ptr(), c.logdeg.data_ptr() if c.logdeg is not None else 0, c.len, cap,
                     H * cap * D * c.k.element_size(), H * cap * 4])
    t = torch.tensor(base, dtype=torch.int64)                       # [Bz, 7]
    lay = torch.arange(L, dtype=torch.int64).view(L, 1)
    out = torch.empty((L, len(caches), 5), dtype=torch.int64)
    out[:, :, 0] = t[:, 0] + lay * t[:, 5]
    out[:, :, 1] = t[:, 1] + lay * t[:, 5]
    out[:, :, 2] = torch.where(t[:, 2] != 0, t[:, 2] + lay * t[:, 6], torch.zeros_like(t[:, 2]))
    out[:, :, 3] = t[:, 3]
    out[:, :, 4] = t[:, 4]
    return out.to(device)


def decode_workspace_bytes(Bz, H, G, D, max_len) -> int:
    return lib.ckv_decode_workspace_bytes(Bz, H, G, D, max_len)


def decode_attn(views: torch.Tensor, H: int, G: int, q: torch.Tensor, out: torch.Tensor, scale: float, max_len: int,
                workspace: torch.Tensor):
    """ckv_decode_attn on the current stream.  views: layer_views(...); q, out: [Bz, H*G, D]."""
    Bz, HG, D = q.shape
    assert HG == H * G and q.is_contiguous() and out.is_contiguous()
    _check(lib.ckv_decode_attn(views.data_ptr(), Bz, H, G, D, dtype_code(q.dtype), q.data_ptr(), out.data_ptr(), scale,
                               max_len, workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream_ptr()))


def decode_attn_static(views: torch.Tensor, H: int, G: int, q: torch.Tensor, out: torch.Tensor, scale: float, max_len: int):
    """ckv_decode_attn_static on the current stream: decode attention without a caller workspace, for callers
    that cannot allocate device memory; the split partials use a fixed 4 MiB array inside the library."""
    Bz, HG, D = q.shape
    assert HG == H * G and q.is_contiguous() and out.is_contiguous()
    _check(lib.ckv_decode_attn_static(views.data_ptr(), Bz, H, G, D, dtype_code(q.dtype), q.data_ptr(), out.data_ptr(),
                                      scale, max_len, _stream_ptr()))


# ---- paged cache: one layer's pool k_pages, v_pages [n_pages, H, P, D], deg_pages int32 / logdeg_pages fp32 [n_pages, H, P]

def _ptr(t):
    return t.data_ptr() if t is not None else None


def paged_views(block_tables, lens, device="cuda") -> torch.Tensor:
    """Device array of ckv_paged_view (two int64 words each) from per-sequence block-table tensors on the GPU."""
    return torch.tensor([[t.data_ptr(), n] for t, n in zip(block_tables, lens)], dtype=torch.int64).to(device)


def decode_attn_paged(views: torch.Tensor, k_pages, v_pages, logdeg_pages, H: int, G: int, q, out, scale: float, max_len: int,
                      workspace: torch.Tensor):
    """ckv_decode_attn_paged on the current stream."""
    Bz, HG, D = q.shape
    assert HG == H * G and q.is_contiguous() and out.is_contiguous() and k_pages.is_contiguous() and v_pages.is_contiguous()
    _check(lib.ckv_decode_attn_paged(views.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), _ptr(logdeg_pages), k_pages.shape[2],
                                     Bz, H, G, D, dtype_code(q.dtype), q.data_ptr(), out.data_ptr(), scale, max_len,
                                     workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream_ptr()))


def decode_append_attn_paged(views: torch.Tensor, k_pages, v_pages, deg_pages, logdeg_pages, H: int, G: int, k_new, v_new, q, out,
                             scale: float, max_len: int, workspace: torch.Tensor):
    """ckv_decode_append_attn_paged on the current stream: k_new, v_new [Bz, H, D] are written to slot views[b].len of
    every sequence's pages and attended to in the same launch; max_len bounds every len + 1."""
    Bz, HG, D = q.shape
    assert HG == H * G and q.is_contiguous() and out.is_contiguous() and k_new.is_contiguous() and v_new.is_contiguous()
    assert k_new.shape == (Bz, H, D) and v_new.shape == (Bz, H, D)
    _check(lib.ckv_decode_append_attn_paged(views.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), deg_pages.data_ptr(),
                                            _ptr(logdeg_pages), k_pages.shape[2], Bz, H, G, D, dtype_code(q.dtype), k_new.data_ptr(),
                                            v_new.data_ptr(), q.data_ptr(), out.data_ptr(), scale, max_len, workspace.data_ptr(),
                                            workspace.numel() * workspace.element_size(), _stream_ptr()))


def pages_gather(block_table, length, k_pages, v_pages, deg_pages, k, v, deg, logdeg=None):
    """ckv_pages_gather: pages -> contiguous slab k, v [H, cap, D], deg [H, cap] of one layer."""
    _, H, P, D = k_pages.shape
    _check(lib.ckv_pages_gather(block_table.data_ptr(), length, k_pages.data_ptr(), v_pages.data_ptr(), _ptr(deg_pages), P, H, D,
                                dtype_code(k_pages.dtype), k.data_ptr(), v.data_ptr(), _ptr(deg), _ptr(logdeg), k.shape[1], _stream_ptr()))


def pages_scatter(block_table, length, k, v, deg, k_pages, v_pages, deg_pages, logdeg_pages):
    """ckv_pages_scatter: contiguous slab -> pages (degrees and log-degrees included)."""
    _, H, P, D = k_pages.shape
    _check(lib.ckv_pages_scatter(block_table.data_ptr(), length, k.data_ptr(), v.data_ptr(), _ptr(deg), k.shape[1], P, H, D,
                                 dtype_code(k_pages.dtype), k_pages.data_ptr(), v_pages.data_ptr(), _ptr(deg_pages),
                                 _ptr(logdeg_pages), _stream_ptr()))



# ---- block tables and slot maps, attention over selected pages, four-bit pages
# (Calls of a few microseconds on the GPU: what is checked of a tensor is what a wrong read or write could come from: its device,
# its size in bytes and that it is contiguous, and the type of everything but a pool's codes and scales and the workspace, which
# are bytes.)

_raw_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_i32, _i64, _f32 = torch.int32, torch.int64, torch.float32
_ROWS = struct.Struct("@PPPqqqqqqiii4x")   # ckv_token_rows
_POOL = struct.Struct("@PPPPPP")           # ckv_quant_pool


def _stream_for(first: torch.Tensor, *others: torch.Tensor | None):
    """The current stream, for a call whose tensors are all on the current device (the library launches there and takes every
    pointer for one of that device's: the host's and other devices' are refused)."""
    dev = first.get_device()
    for t in others:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"tensors are on {first.device} and on {t.device}")
    if dev < 0 or dev != _raw_device():
        raise ValueError(f"tensors are on {first.device}, which is not the current CUDA device")
    return _raw_stream(dev) if _raw_stream is not None else torch.cuda.current_stream().cuda_stream


def pages_resize(lens: torch.Tensor, new_lens: torch.Tensor, block_tables: torch.Tensor, ring: torch.Tensor, ring_state: torch.Tensor,
                 slots: torch.Tensor, slot_begin: torch.Tensor, lens_out: torch.Tensor, ring_state_out: torch.Tensor, status: torch.Tensor,
                 page_tokens: int, views: torch.Tensor | None = None):
    """ckv_pages_resize on the current stream: one step of a batch's block tables, free list, slot map and views, from lengths
    on the device.  lens, new_lens, lens_out int64 [Bz]; block_tables int32 [Bz, row]; ring int32 [n_pages]; ring_state,
    ring_state_out int64 [2] (head, count); slots int64 [n]; slot_begin int64 [Bz + 1]; status int32 [1] (RESIZE_*);
    views int64 [Bz, 2] (paged_views' layout)."""
    Bz, row = block_tables.shape
    n_pages, n_slots = ring.numel(), slots.numel()
    assert lens.dtype is new_lens.dtype is lens_out.dtype is slot_begin.dtype is _i64, "lengths"
    assert lens.nbytes == new_lens.nbytes == lens_out.nbytes == slot_begin.nbytes - 8 == 8 * Bz, "lengths"
    assert lens.is_contiguous() and new_lens.is_contiguous() and lens_out.is_contiguous() and slot_begin.is_contiguous(), "lengths"
    assert ring_state.dtype is ring_state_out.dtype is _i64 and ring_state.nbytes == ring_state_out.nbytes == 16, "ring"
    assert ring_state.is_contiguous() and ring_state_out.is_contiguous(), "ring"
    assert ring.dtype is _i32 and ring.is_contiguous() and status.dtype is _i32 and status.nbytes == 4, "ring"
    assert block_tables.dtype is _i32 and block_tables.is_contiguous() and slots.dtype is _i64 and slots.is_contiguous(), "tables"
    assert views is None or views.dtype is _i64 and views.nbytes == 16 * Bz and views.is_contiguous(), "views"
    _check(lib.ckv_pages_resize(lens.data_ptr(), new_lens.data_ptr(), Bz, page_tokens, block_tables.data_ptr(), row, ring.data_ptr(),
                                n_pages, ring_state.data_ptr(), slots.data_ptr(), n_slots, slot_begin.data_ptr(),
                                lens_out.data_ptr(), ring_state_out.data_ptr(), status.data_ptr(), _ptr(views),
                                _stream_for(lens, new_lens, block_tables, ring, ring_state, slots, slot_begin, lens_out, ring_state_out, status, views)))


def _token_rows(slots: torch.Tensor, k: torch.Tensor, v: torch.Tensor, deg: torch.Tensor | None, heads: int) -> bytes:
    """ckv_token_rows of k, v [n, H, D] with any strides but contiguous rows (a slab [H, cap, D] is passed transposed); deg
    int32 [n, H] with any strides."""
    (n, H, D), (kt, kh, k1), (vt, vh, v1), dt = k.shape, k.stride(), v.stride(), k.dtype
    assert k1 == v1 == 1 and v.dtype is dt and v.shape == (n, H, D) and H == heads, "rows"
    assert slots.dtype is _i64 and slots.nbytes == 8 * n and slots.is_contiguous(), "slots"
    ts, hs, dp = 0, 0, 0
    if deg is not None:
        assert deg.dtype is _i32 and deg.shape == (n, H), "degrees"
        (ts, hs), dp = deg.stride(), deg.data_ptr()
    return _ROWS.pack(k.data_ptr(), v.data_ptr(), dp, kt, kh, vt, vh, ts, hs, H, D, _DTYPE_CODES[dt])


def pages_write(slots: torch.Tensor, k: torch.Tensor, v: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor,
                deg_pages: torch.Tensor | None = None, logdeg_pages: torch.Tensor | None = None, deg: torch.Tensor | None = None):
    """ckv_pages_write on the current stream: k, v [n, H, D] to the slots of one layer's pool, degrees with them."""
    n_pages, H, P, D = k_pages.shape
    rows, per_row = _token_rows(slots, k, v, deg, H), 4 * n_pages * H * P
    assert k_pages.dtype is v_pages.dtype is k.dtype and k_pages.nbytes == v_pages.nbytes and k.shape[2] == D, "pages"
    assert k_pages.is_contiguous() and v_pages.is_contiguous(), "pages"
    assert deg_pages is None or deg_pages.dtype is _i32 and deg_pages.nbytes == per_row and deg_pages.is_contiguous(), "degree pages"
    assert logdeg_pages is None or logdeg_pages.dtype is _f32 and logdeg_pages.nbytes == per_row and logdeg_pages.is_contiguous(), "log-degree pages"
    _check(lib.ckv_pages_write(rows, slots.data_ptr(), slots.numel(), k_pages.data_ptr(), v_pages.data_ptr(), _ptr(deg_pages),
                               _ptr(logdeg_pages), n_pages, P, _stream_for(slots, k, v, k_pages, v_pages, deg_pages, logdeg_pages, deg)))


def pages_summarize(views: torch.Tensor, k_pages: torch.Tensor, deg_pages: torch.Tensor | None, c_pages: torch.Tensor, clog_pages: torch.Tensor,
                    max_blocks: int, from_lens: torch.Tensor | None = None):
    """ckv_pages_summarize on the current stream: mean keys c_pages [n_pages, H, D] and log-degrees clog_pages [n_pages, H] of
    the batch's pages, from the one that holds token from_lens[b] on (of a sequence that is now shorter: its last page)."""
    n_pages, H, P, D = k_pages.shape
    Bz, dt, heads = views.numel() // 2, k_pages.dtype, n_pages * H
    assert views.dtype is _i64 and views.is_contiguous(), "views"
    assert from_lens is None or from_lens.dtype is _i64 and from_lens.nbytes == 8 * Bz and from_lens.is_contiguous(), "lengths"
    assert k_pages.is_contiguous(), "pages"
    assert deg_pages is None or deg_pages.dtype is _i32 and deg_pages.nbytes == 4 * heads * P and deg_pages.is_contiguous(), "degree pages"
    assert c_pages.dtype is dt and c_pages.numel() == heads * D and c_pages.is_contiguous(), "summaries"
    assert clog_pages.dtype is _f32 and clog_pages.nbytes == 4 * heads and clog_pages.is_contiguous(), "summaries"
    _check(lib.ckv_pages_summarize(views.data_ptr(), _ptr(from_lens), Bz, k_pages.data_ptr(), _ptr(deg_pages), P, H, D, _DTYPE_CODES[dt],
                                   max_blocks, c_pages.data_ptr(), clog_pages.data_ptr(),
                                   _stream_for(views, k_pages, deg_pages, c_pages, clog_pages, from_lens)))


def pages_select(views: torch.Tensor, c_pages: torch.Tensor, clog_pages: torch.Tensor | None, page_tokens: int, G: int, q: torch.Tensor,
                 scale: float, max_len: int, selected: torch.Tensor, n_first: int = 0, n_last: int = 0):
    """ckv_pages_select on the current stream: the best blocks of every (sequence, KV head) into selected int32 [Bz, H, n_select]."""
    n_pages, H, D = c_pages.shape
    Bz, heads, n_select = selected.shape
    dt = q.dtype
    assert heads == H and q.shape == (Bz, H * G, D) and q.is_contiguous(), "queries"
    assert views.dtype is _i64 and views.nbytes == 16 * Bz and views.is_contiguous(), "views"
    assert c_pages.dtype is dt and c_pages.is_contiguous(), "summaries"
    assert clog_pages is None or clog_pages.dtype is _f32 and clog_pages.nbytes == 4 * n_pages * H and clog_pages.is_contiguous(), "summaries"
    assert selected.dtype is _i32 and selected.is_contiguous(), "selected"
    _check(lib.ckv_pages_select(views.data_ptr(), c_pages.data_ptr(), _ptr(clog_pages), page_tokens, Bz, H, G, D, _DTYPE_CODES[dt], q.data_ptr(),
                                scale, max_len, n_first, n_last, n_select, selected.data_ptr(),
                                _stream_for(views, c_pages, clog_pages, q, selected)))


def decode_attn_selected(views: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, logdeg_pages: torch.Tensor | None,
                         selected: torch.Tensor, H: int, G: int, q: torch.Tensor, out: torch.Tensor, scale: float):
    """ckv_decode_attn_selected on the current stream: Eq. 3 over the blocks that selected [Bz, H, n_select] lists."""
    Bz, HG, D = q.shape
    n_pages, heads, P, width = k_pages.shape
    dt, n_select = q.dtype, selected.shape[2]
    assert HG == H * G and heads == H and width == D and q.is_contiguous(), "queries"
    assert views.dtype is _i64 and views.nbytes == 16 * Bz and views.is_contiguous(), "views"
    assert out.dtype is dt and out.numel() == Bz * HG * D and out.is_contiguous(), "out"
    assert k_pages.dtype is v_pages.dtype is dt and k_pages.nbytes == v_pages.nbytes and k_pages.is_contiguous() and v_pages.is_contiguous(), "pages"
    assert logdeg_pages is None or logdeg_pages.dtype is _f32 and logdeg_pages.nbytes == 4 * n_pages * H * P, "log-degree pages"
    assert logdeg_pages is None or logdeg_pages.is_contiguous(), "log-degree pages"
    assert selected.dtype is _i32 and selected.numel() == Bz * H * n_select and selected.is_contiguous(), "selected"
    _check(lib.ckv_decode_attn_selected(views.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), _ptr(logdeg_pages), P, selected.data_ptr(),
                                        n_select, Bz, H, G, D, _DTYPE_CODES[dt], q.data_ptr(), out.data_ptr(), scale,
                                        _stream_for(views, k_pages, v_pages, logdeg_pages, selected, q, out)))


@dataclass
class QuantPool:
    """One layer's four-bit pool: codes uint8 [n_pages, H, page_tokens, 64], scales uint8 [n_pages, H, page_tokens, 4], degrees
    int32 and log-degrees fp32 [n_pages, H, page_tokens].  Either may be None: the attention reads the log-degrees (None: all
    degrees one), pages_dequantize returns what is kept and refuses to return degrees that are kept as logarithms alone."""
    k_codes: torch.Tensor
    v_codes: torch.Tensor
    k_scales: torch.Tensor
    v_scales: torch.Tensor
    deg_pages: torch.Tensor | None = None
    logdeg_pages: torch.Tensor | None = None

    @classmethod
    def empty(cls, n_pages: int, H: int, page_tokens: int, device="cuda"):
        u8 = dict(dtype=torch.uint8, device=device)
        return cls(torch.zeros((n_pages, H, page_tokens, 64), **u8), torch.zeros((n_pages, H, page_tokens, 64), **u8),
                   torch.zeros((n_pages, H, page_tokens, 4), **u8), torch.zeros((n_pages, H, page_tokens, 4), **u8),
                   torch.zeros((n_pages, H, page_tokens), dtype=torch.int32, device=device),
                   torch.zeros((n_pages, H, page_tokens), dtype=torch.float32, device=device))

    def c(self):
        """(ckv_quant_pool, n_pages, H, page_tokens), checked; all tensors are on k_codes' device."""
        kc, vc, ks, vs, deg, logdeg = self.k_codes, self.v_codes, self.k_scales, self.v_scales, self.deg_pages, self.logdeg_pages
        n, H, P, width = kc.shape
        per_row = 4 * n * H * P
        assert width == 64 and kc.nbytes == vc.nbytes == 16 * per_row and kc.is_contiguous() and vc.is_contiguous(), "codes"
        assert ks.nbytes == vs.nbytes == per_row and ks.is_contiguous() and vs.is_contiguous(), "scales"
        assert deg is None or deg.dtype is _i32 and deg.nbytes == per_row and deg.is_contiguous(), "degree pages"
        assert logdeg is None or logdeg.dtype is _f32 and logdeg.nbytes == per_row and logdeg.is_contiguous(), "log-degree pages"
        dev = kc.get_device()
        if not (dev == vc.get_device() == ks.get_device() == vs.get_device() and (deg is None or deg.get_device() == dev) and
                (logdeg is None or logdeg.get_device() == dev)):
            raise ValueError("the pool's tensors are on different devices")
        return _POOL.pack(kc.data_ptr(), vc.data_ptr(), ks.data_ptr(), vs.data_ptr(), 0 if deg is None else deg.data_ptr(),
                          0 if logdeg is None else logdeg.data_ptr()), n, H, P


def pages_quantize(slots: torch.Tensor, k: torch.Tensor, v: torch.Tensor, pool: QuantPool, deg: torch.Tensor | None = None):
    """ckv_pages_quantize on the current stream: k, v [n, H, D] (bf16 or fp32) to the slots of a four-bit pool."""
    cp, n_pages, H, P = pool.c()
    _check(lib.ckv_pages_quantize(_token_rows(slots, k, v, deg, H), slots.data_ptr(), slots.numel(), cp, n_pages, P,
                                  _stream_for(slots, k, v, deg, pool.k_codes)))


def pages_dequantize(block_table: torch.Tensor, length: int, pool: QuantPool, k: torch.Tensor, v: torch.Tensor,
                     deg: torch.Tensor | None = None, logdeg: torch.Tensor | None = None):
    """ckv_pages_dequantize on the current stream: one sequence's four-bit pages to a slab k, v [H, cap, D], deg, logdeg [H, cap]."""
    cp, _, H, P = pool.c()
    (heads, cap, D), dt = k.shape, k.dtype
    assert block_table.dtype is _i32 and block_table.is_contiguous() and block_table.numel() * P >= length, "block table"
    assert heads == H and v.dtype is dt and v.nbytes == k.nbytes and k.is_contiguous() and v.is_contiguous(), "slab"
    assert deg is None or deg.dtype is _i32 and deg.nbytes == 4 * H * cap and deg.is_contiguous(), "degrees"
    assert logdeg is None or logdeg.dtype is _f32 and logdeg.nbytes == 4 * H * cap and logdeg.is_contiguous(), "log-degrees"
    _check(lib.ckv_pages_dequantize(block_table.data_ptr(), length, cp, P, H, D, _DTYPE_CODES[dt], k.data_ptr(), v.data_ptr(),
                                    _ptr(deg), _ptr(logdeg), cap, _stream_for(block_table, k, v, deg, logdeg, pool.k_codes)))


def decode_quantized_workspace_bytes(Bz, H, G, D, max_len) -> int:
    return lib.ckv_decode_quantized_workspace_bytes(Bz, H, G, D, max_len)


def decode_attn_quantized(views: torch.Tensor, pool: QuantPool, H: int, G: int, q: torch.Tensor, out: torch.Tensor, scale: float, max_len: int,
                          workspace: torch.Tensor):
    """ckv_decode_attn_quantized on the current stream: Eq. 3 over four-bit pages; q, out bf16 [Bz, H*G, D]."""
    Bz, HG, D = q.shape
    cp, _, heads, P = pool.c()
    dt = q.dtype
    assert HG == H * G and heads == H and q.is_contiguous(), "queries"
    assert views.dtype is _i64 and views.nbytes == 16 * Bz and views.is_contiguous(), "views"
    assert out.dtype is dt and out.numel() == Bz * HG * D and out.is_contiguous(), "out"
    _check(lib.ckv_decode_attn_quantized(views.data_ptr(), cp, P, Bz, H, G, D, _DTYPE_CODES[dt], q.data_ptr(), out.data_ptr(), scale, max_len,
                                         workspace.data_ptr(), workspace.nbytes, _stream_for(views, q, out, workspace, pool.k_codes)))
