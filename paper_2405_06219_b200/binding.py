"""Thin Python binding of libskvq (see ``include/skvq.h``): argument marshalling only.

Functions carry the names of the C entry points.  Tensors are torch CUDA tensors used purely
as device memory; every computation happens in the library's kernels.  The library is loaded
on first use; if it has not been built the call raises -- there is no fallback.
"""
from __future__ import annotations

import contextlib
import ctypes
import os

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libskvq.so")
_lib = None

SKVQ_OK = 0
SKVQ_ERR_INVALID_ARG, SKVQ_ERR_UNSUPPORTED, SKVQ_ERR_MISALIGNED = -1, -2, -3
SKVQ_ERR_CAPACITY, SKVQ_ERR_WORKSPACE, SKVQ_ERR_CUDA = -4, -5, -6
SKVQ_ERR_SCRATCH_LIMIT = -7
SKVQ_NOALLOC_SCRATCH_BYTES = 8 << 20
SKVQ_STATUS_OVERFLOW = 1
SKVQ_STATUS_COPY_TIMEOUT = 2
SKVQ_STATUS_BOUNDS = 4
SKVQ_STATUS_BAD_BATCH = 8
SKVQ_STATUS_BAD_PAGE = 16
SKVQ_STATUS_BAD_POSITION = 32
SKVQ_TOKEN_ALIGN = 64
SKVQ_GROUP_GRANULE = 32
SKVQ_BITS_TERNARY = 15
SKVQ_F16, SKVQ_BF16, SKVQ_F32 = 0, 1, 2
SKVQ_ROPE_PLAIN, SKVQ_ROPE_LINEAR, SKVQ_ROPE_NTK, SKVQ_ROPE_YARN = 0, 1, 2, 3

EXPORTS = ["skvq_version", "skvq_strerror", "skvq_launch_count", "skvq_check_config", "skvq_quant_capacity",
           "skvq_cache_sizes", "skvq_sink_bytes", "skvq_quantize_append", "skvq_workspace_size", "skvq_decode_attention",
           "skvq_step_staging_size", "skvq_decode_step_host", "skvq_decode_attention_noalloc", "skvq_check_group_bounds",
           "skvq_rope_frequencies", "skvq_rope_table", "skvq_rope_apply", "skvq_check_paged_config", "skvq_paged_cache_sizes",
           "skvq_paged_append", "skvq_paged_read", "skvq_paged_workspace_size", "skvq_paged_attention", "skvq_rope_apply_axes",
           "skvq_paged_weights_workspace_size", "skvq_paged_weights", "skvq_paged_evict_workspace_size", "skvq_paged_evict"]


class SkvqConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "n_q_heads", "n_kv_heads", "head_dim", "k_bits", "v_bits",
                                              "group_size", "window", "max_tokens", "n_sink", "meta_fp8")]


class SkvqCacheStruct(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k_codes", "v_codes", "k_meta", "v_meta", "k_win", "v_win", "lengths",
                                               "reorder_k", "reorder_v", "alpha_k", "alpha_v", "status", "k_sink",
                                               "v_sink", "group_bounds_k", "group_bounds_v")]


class SkvqAttnArgs(ctypes.Structure):
    _fields_ = [("sm_scale", ctypes.c_float), ("max_len_hint", ctypes.c_int32), ("n_splits", ctypes.c_int32),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
                ("ev_begin", ctypes.c_void_p), ("ev_end", ctypes.c_void_p)]


class SkvqRopeScaling(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("original_positions", ctypes.c_int32)] + \
        [(n, ctypes.c_double) for n in ("base", "factor", "fast", "slow")]


class SkvqRope(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p)] + [(n, ctypes.c_int32) for n in ("rot_dim", "interleaved", "n_positions")]


class SkvqRopeTensor(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("y", ctypes.c_void_p)] + \
        [(n, ctypes.c_int64) for n in ("x_token_stride", "x_head_stride", "y_token_stride", "y_head_stride")] + \
        [("n_heads", ctypes.c_int32)]


class SkvqRopeAxes(ctypes.Structure):
    _fields_ = [("n_axes", ctypes.c_int32), ("axis", ctypes.c_uint8 * 128)]


class SkvqPagedConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_q_heads", "n_kv_heads", "head_dim", "group_size", "window", "ring_tokens",
                                              "page_tokens", "n_pages", "n_slots", "dtype")]


class SkvqPagedCacheStruct(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k_codes", "v_codes", "k_meta", "v_meta", "k_win", "v_win", "reorder_k",
                                               "reorder_v", "alpha_k", "alpha_v", "status")]


class SkvqPagedBatch(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("page_table", "lens", "starts", "slots")] + \
        [(n, ctypes.c_int32) for n in ("n_seqs", "max_pages", "n_tokens", "max_new", "max_len")] + [("ring_from", ctypes.c_void_p)]


class SkvqPagedAttnArgs(ctypes.Structure):
    _fields_ = [("sm_scale", ctypes.c_float), ("causal", ctypes.c_int32), ("n_splits", ctypes.c_int32),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class SkvqPagedWeightsArgs(ctypes.Structure):
    _fields_ = [("sm_scale", ctypes.c_float), ("causal", ctypes.c_int32), ("last", ctypes.c_int32), ("capacity", ctypes.c_int32),
                ("weights", ctypes.c_void_p), ("weights_out", ctypes.c_void_p), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t)]


class SkvqPagedEvictArgs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("keep", "first", "recent", "capacity")] + \
        [(n, ctypes.c_void_p) for n in ("weights", "weights_out", "page_table_out")] + [("max_pages_out", ctypes.c_int32)] + \
        [(n, ctypes.c_void_p) for n in ("slots_out", "lens_out", "ring_from_out", "kept", "workspace")] + [("workspace_bytes", ctypes.c_size_t)]


class SkvqError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {skvq_strerror(code)} ({code})")


def use_library(path: str | None) -> None:
    """Make the wrappers call the library at ``path`` from now on (None = the default libskvq.so): the debugging build
    libskvq_checked.so exports the same entry points."""
    global _lib, _LIB_PATH
    _LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libskvq.so") if path is None else path
    _lib = None


def lib() -> ctypes.CDLL:
    """Open libskvq.so (built in-tree by ``build.build_library``); raise if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} not found: build it with paper_2405_06219_b200.build.build_library(); "
                               "there is no fallback path")
        L = ctypes.CDLL(_LIB_PATH)
        P, c_int, c_sz, vp = ctypes.POINTER, ctypes.c_int, ctypes.c_size_t, ctypes.c_void_p
        L.skvq_version.restype = c_int
        L.skvq_strerror.restype = ctypes.c_char_p
        L.skvq_strerror.argtypes = [c_int]
        L.skvq_launch_count.restype = ctypes.c_uint64
        L.skvq_check_config.restype = c_int
        L.skvq_check_config.argtypes = [P(SkvqConfig)]
        L.skvq_check_group_bounds.restype = c_int
        L.skvq_check_group_bounds.argtypes = [P(SkvqConfig), vp]
        L.skvq_quant_capacity.restype = ctypes.c_int32
        L.skvq_quant_capacity.argtypes = [P(SkvqConfig)]
        L.skvq_cache_sizes.restype = c_int
        L.skvq_cache_sizes.argtypes = [P(SkvqConfig), P(c_sz)]
        L.skvq_sink_bytes.restype = c_sz
        L.skvq_sink_bytes.argtypes = [P(SkvqConfig)]
        L.skvq_quantize_append.restype = c_int
        L.skvq_quantize_append.argtypes = [P(SkvqConfig), P(SkvqCacheStruct), vp, vp, vp, ctypes.c_int32, vp]
        L.skvq_workspace_size.restype = c_sz
        L.skvq_workspace_size.argtypes = [P(SkvqConfig), ctypes.c_int32, ctypes.c_int32]
        L.skvq_decode_attention.restype = c_int
        L.skvq_decode_attention.argtypes = [P(SkvqConfig), P(SkvqCacheStruct), vp, vp, P(SkvqAttnArgs), vp]
        L.skvq_step_staging_size.restype = c_sz
        L.skvq_step_staging_size.argtypes = [P(SkvqConfig)]
        L.skvq_decode_step_host.restype = c_int
        L.skvq_decode_step_host.argtypes = [P(SkvqConfig), P(SkvqCacheStruct), vp, vp, vp, vp, vp, P(SkvqAttnArgs), vp]
        L.skvq_decode_attention_noalloc.restype = c_int
        L.skvq_decode_attention_noalloc.argtypes = [P(SkvqConfig), P(SkvqCacheStruct), vp, vp, ctypes.c_float,
                                                    ctypes.c_int32, ctypes.c_int32, vp]
        i32, i64, f64 = ctypes.c_int32, ctypes.c_int64, ctypes.c_double
        paged = [P(SkvqPagedConfig), P(SkvqPagedCacheStruct), P(SkvqPagedBatch)]
        L.skvq_rope_frequencies.restype = c_int
        L.skvq_rope_frequencies.argtypes = [i32, P(SkvqRopeScaling), P(f64), P(f64)]
        L.skvq_rope_table.restype = c_int
        L.skvq_rope_table.argtypes = [P(f64), i32, f64, i64, i32, vp, vp]
        L.skvq_rope_apply.restype = c_int
        L.skvq_rope_apply.argtypes = [P(SkvqRope), i32, i32, P(SkvqRopeTensor), P(SkvqRopeTensor), vp, i32, i32, vp, vp]
        L.skvq_check_paged_config.restype = c_int
        L.skvq_check_paged_config.argtypes = [P(SkvqPagedConfig)]
        L.skvq_paged_cache_sizes.restype = c_int
        L.skvq_paged_cache_sizes.argtypes = [P(SkvqPagedConfig), P(c_sz)]
        L.skvq_paged_append.restype = c_int
        L.skvq_paged_append.argtypes = [*paged, P(SkvqRope), vp, vp, i64, i64, vp]
        L.skvq_paged_read.restype = c_int
        L.skvq_paged_read.argtypes = [*paged, i32, vp, vp, i64, i64, vp]
        L.skvq_paged_workspace_size.restype = c_sz
        L.skvq_paged_workspace_size.argtypes = [P(SkvqPagedConfig), P(SkvqPagedBatch), i32]
        L.skvq_paged_attention.restype = c_int
        L.skvq_paged_attention.argtypes = [*paged, P(SkvqRope), vp, i64, vp, i64, vp, P(SkvqPagedAttnArgs), vp]
        L.skvq_rope_apply_axes.restype = c_int
        L.skvq_rope_apply_axes.argtypes = [P(SkvqRope), P(SkvqRopeAxes), i32, i32, P(SkvqRopeTensor), P(SkvqRopeTensor), vp, i64, i64, i32, i32,
                                           vp, vp]
        L.skvq_paged_weights_workspace_size.restype = c_sz
        L.skvq_paged_weights_workspace_size.argtypes = [P(SkvqPagedConfig), P(SkvqPagedBatch), i32]
        L.skvq_paged_weights.restype = c_int
        L.skvq_paged_weights.argtypes = [*paged, P(SkvqRope), vp, i64, vp, P(SkvqPagedWeightsArgs), vp]
        L.skvq_paged_evict_workspace_size.restype = c_sz
        L.skvq_paged_evict_workspace_size.argtypes = [P(SkvqPagedConfig), P(SkvqPagedBatch)]
        L.skvq_paged_evict.restype = c_int
        L.skvq_paged_evict.argtypes = [*paged, P(SkvqPagedEvictArgs), vp]
        _lib = L
    return _lib


def _check(code: int, where: str) -> None:
    if code != SKVQ_OK:
        raise SkvqError(code, where)


def _dptr(t) -> int | None:
    return None if t is None else t.data_ptr()


def _stream(stream) -> int:
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream


# ---------------------------------------------------------------- plain wrappers, same names as the C ABI
def skvq_version() -> int:
    return lib().skvq_version()


def skvq_strerror(code: int) -> str:
    return lib().skvq_strerror(code).decode()


def skvq_launch_count() -> int:
    return int(lib().skvq_launch_count())


def skvq_check_config(cfg: SkvqConfig) -> int:
    return lib().skvq_check_config(ctypes.byref(cfg))


def skvq_check_group_bounds(cfg: SkvqConfig, bounds_host) -> int:
    """bounds_host: contiguous int32 numpy array [Hkv, ng+1] in host memory."""
    return lib().skvq_check_group_bounds(ctypes.byref(cfg), bounds_host.ctypes.data)


def skvq_quant_capacity(cfg: SkvqConfig) -> int:
    return lib().skvq_quant_capacity(ctypes.byref(cfg))


def skvq_cache_sizes(cfg: SkvqConfig) -> list[int]:
    out = (ctypes.c_size_t * 6)()
    _check(lib().skvq_cache_sizes(ctypes.byref(cfg), out), "skvq_cache_sizes")
    return list(out)


def skvq_sink_bytes(cfg: SkvqConfig) -> int:
    return int(lib().skvq_sink_bytes(ctypes.byref(cfg)))


def skvq_workspace_size(cfg: SkvqConfig, max_len_hint: int, n_splits: int = 0) -> int:
    return int(lib().skvq_workspace_size(ctypes.byref(cfg), max_len_hint, n_splits))


def skvq_step_staging_size(cfg: SkvqConfig) -> int:
    return int(lib().skvq_step_staging_size(ctypes.byref(cfg)))


def skvq_quantize_append(cfg: SkvqConfig, cache: SkvqCacheStruct, k, v, n_new_per_seq, n_new: int, stream=None) -> None:
    _check(lib().skvq_quantize_append(ctypes.byref(cfg), ctypes.byref(cache), _dptr(k), _dptr(v),
                                      _dptr(n_new_per_seq), n_new, _stream(stream)), "skvq_quantize_append")


def skvq_decode_attention(cfg: SkvqConfig, cache: SkvqCacheStruct, q, out, args: SkvqAttnArgs, stream=None) -> None:
    _check(lib().skvq_decode_attention(ctypes.byref(cfg), ctypes.byref(cache), _dptr(q), _dptr(out),
                                       ctypes.byref(args), _stream(stream)), "skvq_decode_attention")


def skvq_decode_step_host(cfg, cache, k_new_host, v_new_host, q_host, out_host, staging, args, stream=None) -> None:
    _check(lib().skvq_decode_step_host(ctypes.byref(cfg), ctypes.byref(cache), k_new_host.data_ptr(),
                                       v_new_host.data_ptr(), q_host.data_ptr(), out_host.data_ptr(),
                                       _dptr(staging), ctypes.byref(args), _stream(stream)), "skvq_decode_step_host")


def skvq_decode_attention_noalloc(cfg, cache, q, out, sm_scale, max_len_hint, n_splits=0, stream=None) -> None:
    """Decode attention whose split scratch is the library's built-in device array: for callers that cannot
    allocate or lend a workspace.  Shapes beyond SKVQ_NOALLOC_SCRATCH_BYTES raise SkvqError(SKVQ_ERR_SCRATCH_LIMIT)."""
    _check(lib().skvq_decode_attention_noalloc(ctypes.byref(cfg), ctypes.byref(cache), _dptr(q), _dptr(out),
                                               float(sm_scale), int(max_len_hint), int(n_splits), _stream(stream)),
           "skvq_decode_attention_noalloc")


def skvq_rope_frequencies(rot_dim: int, scaling: SkvqRopeScaling) -> tuple[list[float], float]:
    """Frequencies (radians per position) of the rot_dim/2 pairs and the amplitude of cos and sin."""
    f, amplitude = (ctypes.c_double * max(rot_dim // 2, 1))(), ctypes.c_double()
    _check(lib().skvq_rope_frequencies(rot_dim, ctypes.byref(scaling), f, ctypes.byref(amplitude)), "skvq_rope_frequencies")
    return list(f), amplitude.value


def skvq_rope_table(frequencies, amplitude: float, first_position: int, n_positions: int, table, stream=None) -> None:
    f = (ctypes.c_double * len(frequencies))(*frequencies)
    _check(lib().skvq_rope_table(f, len(frequencies), amplitude, first_position, n_positions, _dptr(table), _stream(stream)),
           "skvq_rope_table")


def skvq_rope_apply(rope: SkvqRope, dtype: int, head_dim: int, a: SkvqRopeTensor, b, positions, n_tokens: int,
                    inverse: int = 0, status=None, stream=None) -> None:
    _check(lib().skvq_rope_apply(ctypes.byref(rope), dtype, head_dim, ctypes.byref(a), None if b is None else ctypes.byref(b),
                                 _dptr(positions), n_tokens, inverse, _dptr(status), _stream(stream)), "skvq_rope_apply")


def skvq_check_paged_config(cfg: SkvqPagedConfig) -> int:
    return lib().skvq_check_paged_config(ctypes.byref(cfg))


def skvq_paged_cache_sizes(cfg: SkvqPagedConfig) -> list[int]:
    out = (ctypes.c_size_t * 6)()
    _check(lib().skvq_paged_cache_sizes(ctypes.byref(cfg), out), "skvq_paged_cache_sizes")
    return list(out)


def skvq_paged_append(cfg, cache, batch, rope, k, v, k_stride: int, v_stride: int, stream=None) -> None:
    _check(lib().skvq_paged_append(ctypes.byref(cfg), ctypes.byref(cache), ctypes.byref(batch),
                                   None if rope is None else ctypes.byref(rope), _dptr(k), _dptr(v), k_stride, v_stride,
                                   _stream(stream)), "skvq_paged_append")


def skvq_paged_read(cfg, cache, batch, window: int, k, v, k_stride: int, v_stride: int, stream=None) -> None:
    _check(lib().skvq_paged_read(ctypes.byref(cfg), ctypes.byref(cache), ctypes.byref(batch), window, _dptr(k), _dptr(v),
                                 k_stride, v_stride, _stream(stream)), "skvq_paged_read")


def skvq_paged_workspace_size(cfg, batch, n_splits: int = 0) -> int:
    return int(lib().skvq_paged_workspace_size(ctypes.byref(cfg), ctypes.byref(batch), n_splits))


def skvq_paged_attention(cfg, cache, batch, rope, q, q_stride: int, out, out_stride: int, lse, args, stream=None) -> None:
    _check(lib().skvq_paged_attention(ctypes.byref(cfg), ctypes.byref(cache), ctypes.byref(batch),
                                      None if rope is None else ctypes.byref(rope), _dptr(q), q_stride, _dptr(out), out_stride,
                                      _dptr(lse), ctypes.byref(args), _stream(stream)), "skvq_paged_attention")


def skvq_rope_apply_axes(rope: SkvqRope, axes: SkvqRopeAxes, dtype: int, head_dim: int, a: SkvqRopeTensor, b, positions, axis_stride: int,
                         token_stride: int, n_tokens: int, inverse: int = 0, status=None, stream=None) -> None:
    _check(lib().skvq_rope_apply_axes(ctypes.byref(rope), ctypes.byref(axes), dtype, head_dim, ctypes.byref(a),
                                      None if b is None else ctypes.byref(b), _dptr(positions), axis_stride, token_stride, n_tokens,
                                      inverse, _dptr(status), _stream(stream)), "skvq_rope_apply_axes")


def skvq_paged_weights_workspace_size(cfg, batch, last: int = 0) -> int:
    return int(lib().skvq_paged_weights_workspace_size(ctypes.byref(cfg), ctypes.byref(batch), last))


def skvq_paged_weights(cfg, cache, batch, rope, q, q_stride: int, lse, args, stream=None) -> None:
    _check(lib().skvq_paged_weights(ctypes.byref(cfg), ctypes.byref(cache), ctypes.byref(batch), None if rope is None else ctypes.byref(rope),
                                    _dptr(q), q_stride, _dptr(lse), ctypes.byref(args), _stream(stream)), "skvq_paged_weights")


def skvq_paged_evict_workspace_size(cfg, batch) -> int:
    return int(lib().skvq_paged_evict_workspace_size(ctypes.byref(cfg), ctypes.byref(batch)))


def skvq_paged_evict(cfg, cache, batch, args, stream=None) -> None:
    _check(lib().skvq_paged_evict(ctypes.byref(cfg), ctypes.byref(cache), ctypes.byref(batch), ctypes.byref(args), _stream(stream)),
           "skvq_paged_evict")


# ---------------------------------------------------------------- device-memory holder
class SkvqCache:
    """Allocates the cache buffers as torch tensors (device memory only) and keeps the C structs.

    reorder_k/_v: int32 [Hkv, D]; alpha_k/_v: float32 [Hkv, D/G] (host arrays or tensors); bounds_k/_v: optional
    int32 [Hkv, D/G + 1] group boundaries (host arrays), checked with skvq_check_group_bounds before the upload.
    """

    def __init__(self, batch, n_q_heads, n_kv_heads, head_dim, k_bits, v_bits, group_size, window, max_tokens,
                 reorder_k, reorder_v, alpha_k, alpha_v, device="cuda:0", n_sink=0, meta_fp8=False, bounds_k=None,
                 bounds_v=None):
        self.cfg = SkvqConfig(batch, n_q_heads, n_kv_heads, head_dim, k_bits, v_bits, group_size, window, max_tokens,
                              n_sink, 1 if meta_fp8 else 0)
        _check(skvq_check_config(self.cfg), "skvq_check_config")
        self.device = torch.device(device)
        self.cap = skvq_quant_capacity(self.cfg)
        self.ng = head_dim // group_size
        sizes = skvq_cache_sizes(self.cfg)
        B, H, W, D = batch, n_kv_heads, window, head_dim
        dev = self.device
        rows = B * H * self.cap
        self.k_codes = torch.zeros((B, H, self.cap, sizes[0] // rows), dtype=torch.uint8, device=dev)
        self.v_codes = torch.zeros((B, H, self.cap, sizes[1] // rows), dtype=torch.uint8, device=dev)
        meta_t = torch.uint8 if meta_fp8 else torch.float16      # {h, z} per (token, group): E4M3 bytes or fp16
        self.k_meta = torch.zeros((B, H, self.cap, self.ng, 2), dtype=meta_t, device=dev)
        self.v_meta = torch.zeros((B, H, self.cap, self.ng, 2), dtype=meta_t, device=dev)
        self.k_win = torch.zeros((B, H, max(W, 1), D), dtype=torch.float16, device=dev)
        self.v_win = torch.zeros((B, H, max(W, 1), D), dtype=torch.float16, device=dev)
        got = [t.numel() * t.element_size() for t in (self.k_codes, self.v_codes, self.k_meta, self.v_meta)]
        assert got == sizes[:4], (got, sizes)
        self.k_sink = torch.zeros((B, H, max(n_sink, 1), D), dtype=torch.float16, device=dev)
        self.v_sink = torch.zeros((B, H, max(n_sink, 1), D), dtype=torch.float16, device=dev)
        assert n_sink == 0 or self.k_sink.numel() * 2 == skvq_sink_bytes(self.cfg)
        self.lengths = torch.zeros((B,), dtype=torch.int32, device=dev)
        self.status = torch.zeros((4,), dtype=torch.int32, device=dev)
        self.reorder_k = torch.as_tensor(reorder_k, dtype=torch.int32).reshape(H, D).contiguous().to(dev)
        self.reorder_v = torch.as_tensor(reorder_v, dtype=torch.int32).reshape(H, D).contiguous().to(dev)
        self.alpha_k = torch.as_tensor(alpha_k, dtype=torch.float32).reshape(H, self.ng).contiguous().to(dev)
        self.alpha_v = torch.as_tensor(alpha_v, dtype=torch.float32).reshape(H, self.ng).contiguous().to(dev)
        self.bounds_k = self._upload_bounds(bounds_k)
        self.bounds_v = self._upload_bounds(bounds_v)
        self.struct = SkvqCacheStruct(*[t.data_ptr() for t in (
            self.k_codes, self.v_codes, self.k_meta, self.v_meta, self.k_win, self.v_win, self.lengths,
            self.reorder_k, self.reorder_v, self.alpha_k, self.alpha_v, self.status, self.k_sink, self.v_sink)],
            _dptr(self.bounds_k), _dptr(self.bounds_v))
        self._workspace = None

    def _upload_bounds(self, bounds):
        if bounds is None:
            return None
        import numpy as np
        b = np.ascontiguousarray(bounds, dtype=np.int32).reshape(self.cfg.n_kv_heads, self.ng + 1)
        _check(skvq_check_group_bounds(self.cfg, b), "skvq_check_group_bounds")
        return torch.from_numpy(b).to(self.device)

    @classmethod
    def for_workload(cls, w, max_tokens=None, device="cuda:0"):
        """Cache for a ``workloads.Workload`` with its reorder index and clip factors."""
        mt = w.context if max_tokens is None else max_tokens
        return cls(w.batch, w.n_q_heads, w.n_kv_heads, w.head_dim, w.k_bits, w.v_bits, w.group_size, w.window, mt,
                   w.reorder_index("k"), w.reorder_index("v"), w.alphas(), w.alphas(), device=device, n_sink=w.n_sink,
                   meta_fp8=w.meta_fp8, bounds_k=w.bounds(), bounds_v=w.bounds())

    def nbytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in (self.k_codes, self.v_codes, self.k_meta, self.v_meta,
                                                          self.k_win, self.v_win)) + \
            (2 * self.k_sink.numel() * 2 if self.cfg.n_sink else 0)

    def append(self, k, v, n_new_per_seq=None, stream=None) -> None:
        """k, v: half [B, n, Hkv, D] CUDA tensors; n_new_per_seq: optional int32 [B] CUDA tensor."""
        assert k.is_cuda and v.is_cuda and k.dtype == torch.float16 and k.is_contiguous() and v.is_contiguous()
        assert k.shape == v.shape and k.shape[0] == self.cfg.batch and tuple(k.shape[2:]) == (self.cfg.n_kv_heads,
                                                                                             self.cfg.head_dim)
        skvq_quantize_append(self.cfg, self.struct, k, v, n_new_per_seq, int(k.shape[1]), stream)

    def attn_args(self, sm_scale, max_len_hint, n_splits=0, ev_begin=None, ev_end=None) -> SkvqAttnArgs:
        need = skvq_workspace_size(self.cfg, max_len_hint, n_splits)
        if self._workspace is None or self._workspace.numel() * 4 < need:
            self._workspace = torch.empty((max(need, 16) + 3) // 4, dtype=torch.float32, device=self.device)
        return SkvqAttnArgs(float(sm_scale), int(max_len_hint), int(n_splits), self._workspace.data_ptr(),
                            self._workspace.numel() * 4,
                            None if ev_begin is None else ev_begin.cuda_event,
                            None if ev_end is None else ev_end.cuda_event)

    def attention(self, q, sm_scale, max_len_hint, out=None, n_splits=0, stream=None):
        """q: half [B, Hq, D] CUDA tensor -> half [B, Hq, D]."""
        assert q.is_cuda and q.dtype == torch.float16 and q.is_contiguous()
        if out is None:
            out = torch.empty_like(q)
        skvq_decode_attention(self.cfg, self.struct, q, out, self.attn_args(sm_scale, max_len_hint, n_splits), stream)
        return out


# ---------------------------------------------------------------- rotary positions and the paged cache
_DTYPES = {torch.float16: SKVQ_F16, torch.bfloat16: SKVQ_BF16, torch.float32: SKVQ_F32}


_HERE = contextlib.nullcontext()
_evict_sizes: dict[int, int] = {}      # workspace bytes of an eviction by its number of sequences


def _on(index: int):
    """The calls launch on the current device: make it the tensors' own."""
    return _HERE if torch.cuda.current_device() == index else torch.cuda.device(index)


def _raw_stream(index: int, stream) -> int:
    return torch._C._cuda_getCurrentRawStream(index) if stream is None else stream.cuda_stream


def _ref(struct):
    return None if struct is None else ctypes.byref(struct)


def _rope_operand(x, y, dtype, T: int, D: int, index: int) -> SkvqRopeTensor:
    assert x.get_device() == y.get_device() == index and x.dtype == y.dtype == dtype, "tensors of one type on the table's device"
    shape = x.shape
    xs, ys = x.stride(), y.stride()
    assert len(shape) == 3 and y.shape == shape and shape[0] == T and shape[2] == D and (D == 1 or (xs[2] == 1 and ys[2] == 1)), "rows [T, heads, D]"
    return SkvqRopeTensor(x.data_ptr(), y.data_ptr(), xs[0], xs[1], ys[0], ys[1], shape[1])


class RopeAxes:
    """Which axis of a position turns which pair of a head: ``of_pair[j]`` is the axis of pair j (0..3), one entry per pair.

    RopeAxes.runs([16, 24, 24]) gives the first 16 pairs to axis 0, the next 24 to axis 1, the last 24 to axis 2."""

    def __init__(self, of_pair):
        of_pair = [int(a) for a in of_pair]
        assert 1 <= len(of_pair) <= 128 and 0 <= min(of_pair) and max(of_pair) < 4, "an axis below 4 for each of up to 128 pairs"
        self.pairs, self.n_axes = len(of_pair), max(of_pair) + 1
        self.struct = SkvqRopeAxes(self.n_axes, (ctypes.c_uint8 * 128)(*of_pair))

    @classmethod
    def runs(cls, lengths):
        return cls([a for a, n in enumerate(lengths) for _ in range(n)])


class RopeTable:
    """A rotation: its cos/sin table (fp32 [positions, rot_dim/2, 2] on the GPU) and the pairing of channels."""

    def __init__(self, table, rot_dim: int, interleaved: bool = False):
        assert table.is_cuda and table.dtype == torch.float32 and table.is_contiguous()
        assert table.dim() == 3 and tuple(table.shape[1:]) == (rot_dim // 2, 2), "table: [positions, rot_dim/2, 2]"
        self.table, self.rot_dim, self.interleaved, self.device = table, rot_dim, bool(interleaved), table.device
        self.struct = SkvqRope(table.data_ptr(), rot_dim, 1 if interleaved else 0, table.shape[0])
        self.index = table.get_device()

    @classmethod
    def build(cls, rot_dim: int, n_positions: int, interleaved: bool = False, base: float = 10000.0,
              kind: int = SKVQ_ROPE_PLAIN, factor: float = 1.0, original_positions: int = 0, fast: float = 32.0,
              slow: float = 1.0, device="cuda:0"):
        """The table of positions 0..n_positions-1 for one of the SKVQ_ROPE_* scalings."""
        f, amplitude = skvq_rope_frequencies(rot_dim, SkvqRopeScaling(kind, original_positions, base, factor, fast, slow))
        table = torch.empty((n_positions, rot_dim // 2, 2), dtype=torch.float32, device=device)
        with _on(table.get_device()):
            skvq_rope_table(f, amplitude, 0, n_positions, table)
        return cls(table, rot_dim, interleaved)

    def apply(self, positions, q, q_out=None, k=None, k_out=None, inverse: bool = False, status=None, stream=None) -> None:
        """Rotate q [T, heads, D] and, in the same launch, k: into q_out/k_out, in place without them.  positions: int32 [T]."""
        T, _, D = q.shape
        index, dtype = self.index, q.dtype
        assert positions.dtype == torch.int32 and positions.is_contiguous() and positions.numel() == T and positions.get_device() == index
        assert status is None or (status.dtype == torch.int32 and status.numel() >= 1 and status.get_device() == index), "status: int32 on the table's device"
        a = _rope_operand(q, q if q_out is None else q_out, dtype, T, D, index)
        b = None if k is None else _rope_operand(k, k if k_out is None else k_out, dtype, T, D, index)
        with _on(index):
            _check(lib().skvq_rope_apply(_ref(self.struct), _DTYPES[dtype], D, _ref(a), _ref(b), positions.data_ptr(), T,
                                         1 if inverse else 0, _dptr(status), _raw_stream(index, stream)), "skvq_rope_apply")


    def apply_axes(self, axes: RopeAxes, positions, q, q_out=None, k=None, k_out=None, inverse: bool = False, status=None, stream=None) -> None:
        """apply() for tokens with a position on each of several axes.  positions: int32 [n_axes, T], any strides (a transposed [T, n_axes]
        tensor does); pair j of a head turns by the table's row positions[axis of j].  inverse=True is the gradient of the rotation."""
        T, _, D = q.shape
        index, dtype = self.index, q.dtype
        assert axes.pairs == self.rot_dim // 2, "axes: one entry per pair of the rotation"
        assert positions.dtype == torch.int32 and positions.shape == (axes.n_axes, T) and positions.get_device() == index, "positions: int32 [n_axes, T]"
        assert status is None or (status.dtype == torch.int32 and status.numel() >= 1 and status.get_device() == index), "status: int32 on the table's device"
        a = _rope_operand(q, q if q_out is None else q_out, dtype, T, D, index)
        b = None if k is None else _rope_operand(k, k if k_out is None else k_out, dtype, T, D, index)
        ps = positions.stride()
        with _on(index):
            _check(lib().skvq_rope_apply_axes(_ref(self.struct), _ref(axes.struct), _DTYPES[dtype], D, _ref(a), _ref(b), positions.data_ptr(), ps[0],
                                              ps[1], T, 1 if inverse else 0, _dptr(status), _raw_stream(index, stream)), "skvq_rope_apply_axes")


class SkvqPagedCache:
    """The pool of a paged 4-bit cache (torch tensors as device memory) and the C structs.

    dtype: torch.float16 or torch.bfloat16; reorder_k/_v: int32 [Hkv, D] or None; alpha_k/_v: float32 [Hkv, D/G] or None;
    ring_tokens: rows per ring slot (default: window); buffers: an engine's own tensors for any of k_codes, v_codes, k_meta,
    v_meta, k_win, v_win instead of new ones.  status[0] (int32, on the GPU) collects the SKVQ_STATUS_* bits of all calls: sequences
    and tokens that a call skipped are reported there and nowhere else; the caller reads and clears it."""

    def __init__(self, n_q_heads, n_kv_heads, head_dim, group_size, window, page_tokens, n_pages, n_slots, dtype=torch.float16,
                 reorder_k=None, reorder_v=None, alpha_k=None, alpha_v=None, ring_tokens=None, buffers=None, device="cuda:0"):
        self.cfg = SkvqPagedConfig(n_q_heads, n_kv_heads, head_dim, group_size, window, window if ring_tokens is None else ring_tokens,
                                   page_tokens, n_pages, n_slots, _DTYPES[dtype])
        _check(skvq_check_paged_config(self.cfg), "skvq_check_paged_config")
        self.dtype = dtype
        H, D, ng, R = n_kv_heads, head_dim, head_dim // group_size, self.cfg.ring_tokens if window else 0
        shapes = {"k_codes": (n_pages, H, page_tokens, D // 2), "k_meta": (n_pages, H, page_tokens, ng, 2), "k_win": (n_slots, H, R, D)}
        kinds = {"codes": torch.uint8, "meta": torch.float16, "win": dtype}
        given = dict(buffers or {})
        self.device = next(iter(given.values())).device if given else torch.empty(0, device=device).device      # with its index
        for name in ("k_codes", "v_codes", "k_meta", "v_meta", "k_win", "v_win"):
            shape, kind = shapes["k" + name[1:]], kinds[name[2:]]
            t = given.pop(name, None)
            if t is None:
                t = torch.zeros(shape, dtype=kind, device=self.device)
            assert t.is_cuda and t.device == self.device and t.dtype == kind and tuple(t.shape) == shape and t.is_contiguous(), name
            setattr(self, name, t)
        assert not given, f"unknown buffers {sorted(given)}"
        assert [t.numel() * t.element_size() for t in (self.k_codes, self.v_codes, self.k_meta, self.v_meta, self.k_win, self.v_win)] == \
            skvq_paged_cache_sizes(self.cfg)
        self.status = torch.zeros((4,), dtype=torch.int32, device=self.device)

        def small(x, kind, shape):
            return None if x is None else torch.as_tensor(x, dtype=kind).reshape(shape).contiguous().to(self.device)
        self.reorder_k, self.reorder_v = small(reorder_k, torch.int32, (H, D)), small(reorder_v, torch.int32, (H, D))
        self.alpha_k, self.alpha_v = small(alpha_k, torch.float32, (H, ng)), small(alpha_v, torch.float32, (H, ng))
        self.struct = SkvqPagedCacheStruct(*[_dptr(t) if t is None or t.numel() else None for t in (
            self.k_codes, self.v_codes, self.k_meta, self.v_meta, self.k_win, self.v_win, self.reorder_k, self.reorder_v,
            self.alpha_k, self.alpha_v, self.status)])
        self.index = self.k_codes.get_device()

    def batch(self, page_table, lens, starts, n_tokens: int, max_new: int, max_len: int, slots=None, ring_from=None) -> SkvqPagedBatch:
        """The sequences of a step: page_table int32 [n, max_pages], lens int32 [n] (tokens including the new ones), starts
        int32 [n + 1] (their rows among the n_tokens packed ones), slots int32 [n] or None; max_new and max_len bound them.  ring_from int32
        [n] or None: the first token that was appended to the sequence's present slot, for sequences that begin on kept pages or came
        back in another slot; the window's older tokens are then read from their pages."""
        n = page_table.shape[0]
        for t, count in ((page_table, page_table.numel()), (lens, n), (starts, n + 1), (slots, n), (ring_from, n)):
            assert t is None or (t.device == self.device and t.dtype == torch.int32 and t.is_contiguous() and t.numel() == count)
        b = SkvqPagedBatch(page_table.data_ptr(), lens.data_ptr(), starts.data_ptr(), _dptr(slots), n, page_table.shape[1],
                           n_tokens, max_new, max_len, _dptr(ring_from))
        b.keep = (page_table, lens, starts, slots, ring_from)
        b.index = self.index
        return b

    def _rows(self, x, batch, heads) -> int:
        """Checks packed rows [T, heads, D] and gives their token stride."""
        shape, stride = x.shape, x.stride()
        D = self.cfg.head_dim
        assert x.get_device() == self.index and x.dtype == self.dtype and len(shape) == 3 and shape[0] >= batch.n_tokens
        assert shape[1] == heads and shape[2] == D and stride[2] == 1 and (heads == 1 or stride[1] == D), "rows: heads and channels contiguous"
        return stride[0] if shape[0] > 1 else heads * D

    def _operands(self, batch, rope=None):
        """Batch and rotation have to lie on the cache's device; the rotation's struct."""
        assert getattr(batch, "index", self.index) == self.index, "a batch on the cache's device"
        if rope is None:
            return None
        assert rope.index == self.index, "a rotation on the cache's device"
        return _ref(rope.struct)

    def append(self, batch, k, v, rope=None, stream=None) -> None:
        """k, v: [T, Hkv, D] in the cache's type, any token stride that is a multiple of 8."""
        H, index, rotation = self.cfg.n_kv_heads, self.index, self._operands(batch, rope)
        ks, vs = self._rows(k, batch, H), self._rows(v, batch, H)
        with _on(index):
            _check(lib().skvq_paged_append(_ref(self.cfg), _ref(self.struct), _ref(batch), rotation, k.data_ptr(),
                                           v.data_ptr(), ks, vs, _raw_stream(index, stream)), "skvq_paged_append")

    def read(self, batch, k=None, v=None, window: bool = True, stream=None):
        """The new tokens' rows of the cache as values [T, Hkv, D], in source order; into k and v where they are given.
        Rows of skipped sequences and tokens, and rows behind the last sequence, are not written: in tensors made here they hold
        whatever lay in that memory.  What was skipped shows in the cache's `status`."""
        H, index = self.cfg.n_kv_heads, self.index
        self._operands(batch)
        with _on(index), (_HERE if stream is None else torch.cuda.stream(stream)):
            if k is None and v is None:
                k, v = torch.empty((2, batch.n_tokens, H, self.cfg.head_dim), dtype=self.dtype, device=self.device).unbind(0)
            elif k is None or v is None:
                other = torch.empty((batch.n_tokens, H, self.cfg.head_dim), dtype=self.dtype, device=self.device)
                k, v = (other, v) if k is None else (k, other)
            ks, vs = self._rows(k, batch, H), self._rows(v, batch, H)
            _check(lib().skvq_paged_read(_ref(self.cfg), _ref(self.struct), _ref(batch), 1 if window else 0, k.data_ptr(), v.data_ptr(), ks, vs,
                                         _raw_stream(index, stream)), "skvq_paged_read")
        return k, v

    def attention(self, batch, q, sm_scale, out=None, causal: bool = True, rope=None, lse=None, n_splits: int = 0,
                  workspace=None, stream=None):
        """q [T, Hq, D] -> out [T, Hq, D]; lse: optional float32 [T, Hq].  Without a workspace (a tensor of at least
        skvq_paged_workspace_size bytes) each call takes one of its own from torch's allocator on the stream it runs on, so calls
        on several streams and captured graphs never share it.  Rows of skipped sequences, and rows behind the last sequence, are not
        written: without `out` they hold whatever lay in that memory.  What was skipped shows in the cache's `status`."""
        c, index, rotation = self.cfg, self.index, self._operands(batch, rope)
        H = c.n_q_heads
        qs = self._rows(q, batch, H)
        with _on(index), (_HERE if stream is None else torch.cuda.stream(stream)):
            if out is None:
                out, os_ = torch.empty((batch.n_tokens, H, c.head_dim), dtype=self.dtype, device=self.device), H * c.head_dim
            else:
                os_ = self._rows(out, batch, H)
            if workspace is None:
                size = skvq_paged_workspace_size(c, batch, n_splits)
                workspace = torch.empty(size, dtype=torch.uint8, device=self.device) if size else None
            else:
                assert workspace.get_device() == index and workspace.is_contiguous()
                size = workspace.numel() * workspace.element_size()
            assert lse is None or (lse.dtype == torch.float32 and lse.is_contiguous() and lse.get_device() == index and lse.numel() >= batch.n_tokens * H)
            args = SkvqPagedAttnArgs(sm_scale, 1 if causal else 0, n_splits, _dptr(workspace), size)
            _check(lib().skvq_paged_attention(_ref(c), _ref(self.struct), _ref(batch), rotation, q.data_ptr(), qs,
                                              out.data_ptr(), os_, _dptr(lse), _ref(args), _raw_stream(index, stream)), "skvq_paged_attention")
        return out

    def new_weights(self, capacity: int):
        """Attention weights of every slot, for accumulate_weights and evict: float32 [n_slots, Hkv, capacity], capacity >= the longest
        sequence."""
        return torch.zeros((self.cfg.n_slots, self.cfg.n_kv_heads, capacity), dtype=torch.float32, device=self.device)

    def _weights(self, w) -> int:
        shape = w.shape
        assert w.get_device() == self.index and w.dtype == torch.float32 and w.is_contiguous() and len(shape) == 3
        assert shape[0] == self.cfg.n_slots and shape[1] == self.cfg.n_kv_heads, "weights: [n_slots, Hkv, capacity]"
        return shape[2]

    def _words(self, t, count) -> int:
        """Checks an int32 tensor of the cache's device and gives its address."""
        assert t.get_device() == self.index and t.dtype == torch.int32 and t.is_contiguous() and (count is None or t.numel() == count)
        return t.data_ptr()

    def accumulate_weights(self, batch, q, lse, weights, sm_scale, out=None, causal: bool = True, rope=None, last: int = 0, workspace=None,
                           stream=None):
        """Adds to the weight of every token what this step's rows gave it: exp(score - lse) over the query heads of its KV head.
        q [T, Hq, D] and lse [T, Hq] float32 as attention(..., lse=lse) had them, with the same sm_scale, causal and rope; weights float32
        [n_slots, Hkv, capacity] (None: zeros), updated in place or into `out`.  last: only the last so many new tokens of a sequence
        count.  Entries at or beyond a sequence's length are left alone.  Without a workspace each call takes one of its own."""
        c, index, rotation = self.cfg, self.index, self._operands(batch, rope)
        out = weights if out is None else out
        assert out is not None, "weights, or out"
        capacity = self._weights(out)
        assert weights is None or self._weights(weights) == capacity, "weights and out of one capacity"
        qs = self._rows(q, batch, c.n_q_heads)
        assert lse.dtype == torch.float32 and lse.is_contiguous() and lse.get_device() == index and lse.numel() >= batch.n_tokens * c.n_q_heads
        with _on(index), (_HERE if stream is None else torch.cuda.stream(stream)):
            if workspace is None:
                size = skvq_paged_weights_workspace_size(c, batch, last)
                workspace = torch.empty(size, dtype=torch.uint8, device=self.device) if size else None
            else:
                assert workspace.get_device() == index and workspace.is_contiguous()
                size = workspace.numel() * workspace.element_size()
            args = SkvqPagedWeightsArgs(sm_scale, 1 if causal else 0, last, capacity, _dptr(weights), out.data_ptr(), _dptr(workspace), size)
            _check(lib().skvq_paged_weights(_ref(c), _ref(self.struct), _ref(batch), rotation, q.data_ptr(), qs, lse.data_ptr(), _ref(args),
                                            _raw_stream(index, stream)), "skvq_paged_weights")
        return out

    def evict(self, batch, weights, keep: int, first: int = 0, recent=None, weights_out=None, page_table_out=None, slots_out=None, lens_out=None,
              ring_from_out=None, kept=None, stream=None):
        """Shortens every sequence of the batch to `keep` tokens: per KV head the `first` oldest, the `recent` newest (default: the
        window) and the heaviest of those between.  Gives (kept int32 [n, Hkv, keep]: the old number of every token, -1 behind the last;
        the lengths int32 [n]; ring_from int32 [n] for later batches).  In place, or into other pages (page_table_out int32
        [n, max_pages]), slots (slots_out int32 [n]) and weights (weights_out).  lens_out and ring_from_out may be the batch's own."""
        c, index = self.cfg, self.index
        self._operands(batch)
        n, H = batch.n_seqs, c.n_kv_heads
        capacity, w = self._weights(weights), weights.data_ptr()
        w_out = w
        if weights_out is not None:
            assert self._weights(weights_out) == capacity, "weights of one capacity"
            w_out = weights_out.data_ptr()
        pages, max_pages = None, 0
        if page_table_out is not None:
            pages, max_pages = self._words(page_table_out, None), page_table_out.shape[-1]
            assert page_table_out.shape == (n, max_pages), "page_table_out: [n, max_pages]"
        with _on(index), (_HERE if stream is None else torch.cuda.stream(stream)):
            size = _evict_sizes.get(n)
            if size is None:
                size = _evict_sizes[n] = skvq_paged_evict_workspace_size(c, batch)      # depends on the number of sequences alone
            if kept is None:
                kept = torch.empty((n, H, keep), dtype=torch.int32, device=self.device)
            # one piece of memory for the workspace and the two results
            rows = size // (4 * n) if n else 0
            small = torch.empty((rows + 2, n), dtype=torch.int32, device=self.device)
            if lens_out is None:
                lens_out = small[rows]
            if ring_from_out is None:
                ring_from_out = small[rows + 1]
            args = SkvqPagedEvictArgs(keep, first, c.window if recent is None else recent, capacity, w, w_out, pages, max_pages,
                                      None if slots_out is None else self._words(slots_out, n), self._words(lens_out, n),
                                      self._words(ring_from_out, n), self._words(kept, n * H * keep), small.data_ptr(), size)
            _check(lib().skvq_paged_evict(_ref(c), _ref(self.struct), _ref(batch), _ref(args), _raw_stream(index, stream)), "skvq_paged_evict")
        return kept, lens_out, ring_from_out
