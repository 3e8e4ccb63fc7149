"""Thin binding of libpackkv.so -- argument marshalling only: ctypes, and for the calls of a decode step and of an append
a native module (csrc/binding_native.cpp) that is tried first and leaves every argument it does not expect to the code here,
which makes every call where that module cannot be built or loaded.

Function names follow the C ABI (include/packkv.h).  PyTorch is used for
device memory and streams; every step of the path runs in the HIP kernels.
There is no CPU fallback: if the library is missing the import of the symbols
fails loudly.
"""
from __future__ import annotations

import ctypes as C
import importlib.util
import math
import os
import subprocess
import warnings

import torch

from . import build as _build

KV_OK, KV_ERR_ARG, KV_ERR_UNSUPPORTED, KV_ERR_CAPACITY, KV_ERR_HIP = 0, -1, -2, -3, -4
HEAD_DIM = 128
BLOCK_TOKENS = 64
CHUNK_MAX_BYTES = 512 + 512 * 8


class kv_config_t(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_kv_heads", C.c_int32), ("n_q_heads", C.c_int32),
                ("head_dim", C.c_int32), ("block_tokens", C.c_int32), ("pack_size", C.c_int32),
                ("repack", C.c_int32), ("tail_capacity", C.c_int32),
                ("k_rel_scale", C.c_float), ("v_rel_scale", C.c_float),
                ("max_tokens", C.c_int64)]


_BUFFER_NAMES = ("k_arena", "v_arena", "k_index", "v_index", "k_token_meta", "v_token_meta",
                 "k_tail", "v_tail", "workspace", "token_order", "k_pages", "v_pages")
PAGE_BYTES = 65536
REPACK_NONE, REPACK_V_MEDIAN = 0, 1


class kv_sizes_t(C.Structure):
    _fields_ = [(n, C.c_size_t) for n in _BUFFER_NAMES]


class kv_buffers_t(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in _BUFFER_NAMES]


class kv_stats_t(C.Structure):
    _fields_ = [("tokens", C.c_int64), ("packed_tokens", C.c_int64), ("tail_tokens", C.c_int64),
                ("n_chunks", C.c_int64), ("k_bytes", C.c_int64), ("v_bytes", C.c_int64),
                ("index_bytes", C.c_int64), ("token_meta_bytes", C.c_int64),
                ("overflow", C.c_int32),
                ("k_header_bytes", C.c_int64), ("k_payload_bytes", C.c_int64), ("k_padding_bytes", C.c_int64),
                ("v_header_bytes", C.c_int64), ("v_payload_bytes", C.c_int64), ("v_padding_bytes", C.c_int64)]


FP4_PAGE_TOKENS, FP4_GROUP = 64, 32
KV_TYPE_FP16, KV_TYPE_BF16, KV_TYPE_FP32 = 0, 1, 2


class kv_fp4_config_t(C.Structure):
    _fields_ = [("n_kv_heads", C.c_int32), ("n_q_heads", C.c_int32), ("head_dim", C.c_int32), ("n_pages", C.c_int64)]


class kv_fp4_sizes_t(C.Structure):
    _fields_ = [("pages", C.c_size_t), ("workspace", C.c_size_t)]


class kv_rotary_t(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("dims", C.c_int32), ("interleaved", C.c_int32), ("magnitude", C.c_float),
                ("turns", C.c_void_p)]


class kv_fp4_batch_t(C.Structure):
    _fields_ = [("batch", C.c_int32), ("max_new", C.c_int32), ("table_pages", C.c_int32),
                ("lens", C.c_void_p), ("new_rows", C.c_void_p), ("first_row", C.c_void_p), ("page_table", C.c_void_p)]


EXPORTS = ("kv_query_sizes", "kv_cache_create", "kv_cache_destroy", "kv_compress_append", "kv_compress_append_bf16",
           "kv_k_matvec", "kv_v_matvec", "kv_v_matvec_noalloc", "kv_softmax", "kv_decode_attention", "kv_cache_stats", "kv_cache_restore", "kv_cache_tokens",
           "kv_strerror", "kv_fp16_k_matvec", "kv_fp16_v_matvec", "kv_fp16_v_workspace_bytes",
           "kv_stream_read", "kv_page_pool_state_bytes", "kv_page_pool_create", "kv_page_pool_destroy",
           "kv_page_pool_free_pages", "kv_query_sizes_paged", "kv_cache_create_paged", "kv_cache_release",
           "kv_fp4_query_sizes", "kv_fp4_cache_create", "kv_fp4_cache_destroy", "kv_fp4_append", "kv_fp4_read",
           "kv_fp4_attention", "kv_fp4_weights", "kv_fp4_select", "kv_fp4_compact", "kv_rotary")
# entry points the native module calls, in its order
_NATIVE_CALLS = ("kv_compress_append", "kv_compress_append_bf16", "kv_k_matvec", "kv_softmax", "kv_v_matvec",
                 "kv_decode_attention", "kv_cache_restore", "kv_cache_release", "kv_cache_tokens", "kv_fp4_append", "kv_fp4_read",
                 "kv_fp4_attention", "kv_fp4_weights", "kv_fp4_select", "kv_fp4_compact", "kv_rotary")

_lib = None
_native = None


def library_path() -> str:
    return _build.LIB


def _load_native(L):
    """The native module on top of the library L, built first only if it does not exist; None where it cannot be had."""
    try:
        path = _build.native_path()
        if not os.path.exists(path):
            _build.build_native()
        spec = importlib.util.spec_from_file_location(__package__ + "._native", path)
        native = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(native)
        native.bind(tuple(C.cast(getattr(L, name), C.c_void_p).value for name in _NATIVE_CALLS), _check,
                    _current_device, _current_raw_stream, getattr(torch._C, "_cuda_isInBadFork", None))
        return native
    except (ImportError, OSError, subprocess.CalledProcessError) as e:
        warnings.warn("the binding's native part is not available, calls are marshalled in Python: %s" % e, RuntimeWarning)
        return None


class _PythonCalls:
    """In the place of the native module's Calls: leaves every call to the Python code."""

    def set_handle(self, address):
        pass

    def append(self, *args):
        return NotImplemented

    k_matvec = softmax = v_matvec = attention = restore = release = read = append
    read_into = weights = select = compact = turn = append


def lib():
    """Load libpackkv.so and the native module; build them first only if they do not exist."""
    global _lib, _native
    if _lib is None:
        if not os.path.exists(_build.LIB):
            _build.build()
        L = C.CDLL(_build.LIB)
        vp, i32, i64, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float
        L.kv_query_sizes.argtypes = [C.POINTER(kv_config_t), C.c_double, C.POINTER(kv_sizes_t)]
        L.kv_cache_create.argtypes = [C.POINTER(kv_config_t), C.POINTER(kv_buffers_t),
                                      C.POINTER(kv_sizes_t), C.POINTER(vp)]
        L.kv_cache_destroy.argtypes = [vp]
        L.kv_page_pool_state_bytes.argtypes = [i64]
        L.kv_page_pool_state_bytes.restype = C.c_size_t
        L.kv_page_pool_create.argtypes = [vp, i64, vp, vp, C.POINTER(vp)]
        L.kv_page_pool_destroy.argtypes = [vp]
        L.kv_page_pool_free_pages.argtypes = [vp, C.POINTER(i64), vp]
        L.kv_query_sizes_paged.argtypes = [C.POINTER(kv_config_t), C.POINTER(kv_sizes_t)]
        L.kv_cache_create_paged.argtypes = [C.POINTER(kv_config_t), vp, C.POINTER(kv_buffers_t),
                                            C.POINTER(kv_sizes_t), C.POINTER(vp)]
        L.kv_cache_release.argtypes = [vp, vp]
        L.kv_compress_append.argtypes = [vp, vp, vp, i32, vp]
        L.kv_compress_append_bf16.argtypes = [vp, vp, vp, i32, vp]
        L.kv_k_matvec.argtypes = [vp, vp, f32, vp, i64, vp]
        L.kv_v_matvec.argtypes = [vp, vp, i64, vp, vp]
        L.kv_v_matvec_noalloc.argtypes = [vp, vp, i64, vp, vp]
        L.kv_decode_attention.argtypes = [vp, vp, f32, vp, vp]
        L.kv_softmax.argtypes = [vp, vp, i64, vp]
        L.kv_cache_stats.argtypes = [vp, C.POINTER(kv_stats_t), vp]
        L.kv_cache_restore.argtypes = [vp, i64]
        L.kv_cache_tokens.argtypes = [vp]
        L.kv_cache_tokens.restype = i64
        L.kv_strerror.argtypes = [C.c_int]
        L.kv_strerror.restype = C.c_char_p
        L.kv_fp16_k_matvec.argtypes = [vp, vp, f32, vp, i64, i32, i32, i32, i64, vp]
        L.kv_fp16_v_matvec.argtypes = [vp, vp, i64, vp, i32, i32, i32, i64, vp, vp]
        L.kv_fp16_v_workspace_bytes.argtypes = [i32, i32]
        L.kv_fp16_v_workspace_bytes.restype = C.c_size_t
        L.kv_stream_read.argtypes = [vp, C.c_size_t, vp, vp]
        batch = C.POINTER(kv_fp4_batch_t)
        L.kv_fp4_query_sizes.argtypes = [C.POINTER(kv_fp4_config_t), C.POINTER(kv_fp4_sizes_t)]
        L.kv_fp4_cache_create.argtypes = [C.POINTER(kv_fp4_config_t), vp, vp, C.POINTER(kv_fp4_sizes_t), C.POINTER(vp)]
        L.kv_fp4_cache_destroy.argtypes = [vp]
        L.kv_fp4_append.argtypes = [vp, batch, vp, i64, vp, i64, i32, i64, vp]
        L.kv_fp4_read.argtypes = [vp, batch, vp, vp, i32, i64, vp]
        L.kv_fp4_attention.argtypes = [vp, batch, vp, i64, i32, i64, f32, i32, i32, vp, i32, vp, vp]
        L.kv_fp4_weights.argtypes = [vp, batch, vp, i64, i32, i64, f32, i32, i32, vp, vp, vp, i64, vp]
        L.kv_fp4_select.argtypes = [vp, batch, vp, i64, i32, vp, i32, i32, vp, vp, vp]
        L.kv_fp4_compact.argtypes = [vp, batch, batch, vp, i32, vp, vp, i64, vp, i64, vp]
        L.kv_rotary.argtypes = [C.POINTER(kv_rotary_t), vp, i64, i32, i32, vp, i64, i32, vp, i64, vp, i64, i32, vp, i64, vp]
        for name in EXPORTS:
            if name not in ("kv_cache_tokens", "kv_strerror", "kv_fp16_v_workspace_bytes",
                            "kv_page_pool_state_bytes"):
                getattr(L, name).restype = C.c_int
        _lib, _native = L, _load_native(L)
    return _lib


class PackKVError(RuntimeError):
    """A library call returned an error code (kept in .code)."""

    def __init__(self, message, code=None):
        super().__init__(message)
        self.code = code


def _check(rc: int, what: str) -> None:
    if rc != KV_OK:
        raise PackKVError("%s: %s (%d)" % (what, lib().kv_strerror(rc).decode(), rc), rc)


# torch's current stream as a raw pointer, without building a Stream object around it (2 us per call
# of the decode entry points, which launch kernels of a few microseconds)
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream_ptr(stream=None):
    """stream: None (torch's current stream), a torch stream, or a raw hipStream_t as int."""
    if stream is None:
        if _current_raw_stream is not None and _current_device is not None and torch.cuda.is_initialized():
            return _current_raw_stream(_current_device())
        return torch.cuda.current_stream().cuda_stream
    return stream if isinstance(stream, int) else stream.cuda_stream


def make_config(batch, n_kv_heads, n_q_heads, max_tokens, k_rel_scale=0.1, v_rel_scale=0.2,
                repack=REPACK_NONE, pack_size=16):
    return kv_config_t(batch, n_kv_heads, n_q_heads, HEAD_DIM, BLOCK_TOKENS, pack_size, repack, BLOCK_TOKENS,
                       k_rel_scale, v_rel_scale, max_tokens)


def kv_query_sizes(cfg: kv_config_t, bits_per_element_budget: float = 0.0) -> kv_sizes_t:
    out = kv_sizes_t()
    _check(lib().kv_query_sizes(C.byref(cfg), bits_per_element_budget, C.byref(out)), "kv_query_sizes")
    return out


def kv_query_sizes_paged(cfg: kv_config_t) -> kv_sizes_t:
    out = kv_sizes_t()
    _check(lib().kv_query_sizes_paged(C.byref(cfg), C.byref(out)), "kv_query_sizes_paged")
    return out


class PagePool:
    """Owns the pages and the bookkeeping words (torch tensors) and the kv_page_pool_t handle."""

    def __init__(self, n_pages, device="cuda:0"):
        self.device = torch.device(device)
        self.n_pages = n_pages
        state_bytes = lib().kv_page_pool_state_bytes(n_pages)
        if state_bytes == 0:
            raise PackKVError("kv_page_pool_state_bytes: invalid argument", KV_ERR_ARG)
        with torch.cuda.device(self.device):
            self.pages = torch.empty(n_pages * PAGE_BYTES, dtype=torch.uint8, device=self.device)
            self.state = torch.empty(state_bytes, dtype=torch.uint8, device=self.device)
            torch.cuda.synchronize()
            handle = C.c_void_p()
            _check(lib().kv_page_pool_create(self.pages.data_ptr(), n_pages, self.state.data_ptr(),
                                             _stream_ptr(None), C.byref(handle)), "kv_page_pool_create")
        self.handle = handle

    def kv_page_pool_free_pages(self, stream=None) -> int:
        n = C.c_int64()
        _check(lib().kv_page_pool_free_pages(self.handle, C.byref(n), _stream_ptr(stream)),
               "kv_page_pool_free_pages")
        return int(n.value)

    def close(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.kv_page_pool_destroy(self.handle)
        self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class PackedKVCache:
    """Owns the device buffers (torch tensors) and the kv_cache_t handle.  With `pool` (a PagePool)
    the cache is paged: it has no arenas of its own and keeps its chunks in pages of the pool."""

    def __init__(self, batch, n_kv_heads, n_q_heads, max_tokens, k_rel_scale=0.1, v_rel_scale=0.2,
                 bits_per_element_budget=0.0, device="cuda:0", repack=REPACK_NONE, pack_size=16, pool=None):
        self.cfg = make_config(batch, n_kv_heads, n_q_heads, max_tokens, k_rel_scale, v_rel_scale, repack,
                               pack_size)
        self.device = torch.device(device)
        self.pool = pool
        self.sizes = (kv_query_sizes_paged(self.cfg) if pool is not None
                      else kv_query_sizes(self.cfg, bits_per_element_budget))
        self.tensors = {}
        bufs = kv_buffers_t()
        with torch.cuda.device(self.device):
            for name in _BUFFER_NAMES:
                t = torch.empty(getattr(self.sizes, name), dtype=torch.uint8, device=self.device)
                assert t.numel() == 0 or t.data_ptr() % 256 == 0
                self.tensors[name] = t
                setattr(bufs, name, t.data_ptr() if t.numel() else None)
            torch.cuda.synchronize()
            handle = C.c_void_p()
            if pool is not None:
                _check(lib().kv_cache_create_paged(C.byref(self.cfg), pool.handle, C.byref(bufs),
                                                   C.byref(self.sizes), C.byref(handle)), "kv_cache_create_paged")
            else:
                _check(lib().kv_cache_create(C.byref(self.cfg), C.byref(bufs), C.byref(self.sizes),
                                             C.byref(handle)), "kv_cache_create")
        self._calls = _native.Calls(batch, n_kv_heads, n_q_heads, str(self.device)) if _native else _PythonCalls()
        self.handle = handle
        self.batch, self.n_kv_heads, self.n_q_heads = batch, n_kv_heads, n_q_heads
        self._q_shape, self._row_shape = (batch, n_q_heads, HEAD_DIM), (batch, n_q_heads)
        self._token_shape = (n_kv_heads, HEAD_DIM)

    def close(self):
        if getattr(self, "handle", None) and _lib is not None:
            # a paged cache returns its pages to the pool here: the pool must still exist
            # (if it was closed first, the handle is dropped without the call)
            if getattr(self, "pool", None) is None or self.pool.handle:
                _lib.kv_cache_destroy(self.handle)
        self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def handle(self):
        """The kv_cache_t of the library (ctypes.c_void_p), None once closed."""
        return self._handle

    @handle.setter
    def handle(self, value):
        self._handle = value
        calls = getattr(self, "_calls", None)
        if calls is not None:
            calls.set_handle((value.value if isinstance(value, C.c_void_p) else value) or 0)

    @property
    def tokens(self) -> int:
        return _lib.kv_cache_tokens(self.handle)

    def kv_compress_append(self, k_new: torch.Tensor, v_new: torch.Tensor, stream=None):
        """k_new, v_new: fp16 (or both bf16: kv_compress_append_bf16) [B, n, H_kv, 128] contiguous device tensors."""
        if self._calls.append(k_new, v_new, stream) is not NotImplemented:
            return
        dtype, shape = k_new.dtype, k_new.shape
        assert dtype == v_new.dtype and dtype in (torch.float16, torch.bfloat16)
        assert k_new.is_contiguous() and v_new.is_contiguous() and shape == v_new.shape
        assert shape[0] == self.batch and shape[2:] == self._token_shape
        if dtype == torch.bfloat16:
            rc = _lib.kv_compress_append_bf16(self.handle, k_new.data_ptr(), v_new.data_ptr(), shape[1],
                                              _stream_ptr(stream))
            if rc != KV_OK:
                _check(rc, "kv_compress_append_bf16")
            return
        rc = _lib.kv_compress_append(self.handle, k_new.data_ptr(), v_new.data_ptr(), shape[1], _stream_ptr(stream))
        if rc != KV_OK:
            _check(rc, "kv_compress_append")

    def kv_k_matvec(self, q: torch.Tensor, sm_scale: float, scores: torch.Tensor = None, stream=None):
        """q: fp16 [B, Hq, 128] -> scores fp32 [B, Hq, ld] (ld >= tokens)."""
        done = self._calls.k_matvec(q, sm_scale, scores, stream)
        if done is not NotImplemented:
            return done
        assert q.dtype == torch.float16 and q.is_contiguous()
        assert q.shape == self._q_shape
        if scores is None:
            scores = torch.empty(self.batch, self.n_q_heads, self.tokens, dtype=torch.float32,
                                 device=self.device)
        else:
            assert scores.dtype == torch.float32 and scores.is_contiguous()
        rc = _lib.kv_k_matvec(self.handle, q.data_ptr(), sm_scale, scores.data_ptr(), scores.shape[2],
                              _stream_ptr(stream))
        if rc != KV_OK:
            _check(rc, "kv_k_matvec")
        return scores

    def kv_v_matvec(self, p: torch.Tensor, out: torch.Tensor = None, stream=None):
        """p: fp32 [B, Hq, ld] -> out fp32 [B, Hq, 128]."""
        if out is None:
            done = self._calls.v_matvec(p, stream)
            if done is not NotImplemented:
                return done
        assert p.dtype == torch.float32 and p.is_contiguous()
        assert p.shape[:2] == self._row_shape
        if out is None:
            out = torch.empty(self._q_shape, dtype=torch.float32, device=self.device)
        rc = _lib.kv_v_matvec(self.handle, p.data_ptr(), p.shape[2], out.data_ptr(), _stream_ptr(stream))
        if rc != KV_OK:
            _check(rc, "kv_v_matvec")
        return out

    def kv_v_matvec_noalloc(self, p: torch.Tensor, out: torch.Tensor, stream=None):
        """As kv_v_matvec, through the entry point that allocates nothing; `out` is the caller's."""
        assert p.dtype == torch.float32 and p.is_contiguous()
        assert tuple(p.shape[:2]) == (self.batch, self.n_q_heads)
        assert out.dtype == torch.float32 and out.is_contiguous()
        assert tuple(out.shape) == (self.batch, self.n_q_heads, HEAD_DIM)
        _check(lib().kv_v_matvec_noalloc(self.handle, p.data_ptr(), p.shape[2], out.data_ptr(),
                                         _stream_ptr(stream)), "kv_v_matvec_noalloc")
        return out

    def kv_softmax(self, scores: torch.Tensor, stream=None):
        """In-place softmax over the cached tokens of scores fp32 [B, Hq, ld]; returns scores."""
        done = self._calls.softmax(scores, stream)
        if done is not NotImplemented:
            return done
        assert scores.dtype == torch.float32 and scores.is_contiguous()
        assert scores.shape[:2] == self._row_shape
        rc = _lib.kv_softmax(self.handle, scores.data_ptr(), scores.shape[2], _stream_ptr(stream))
        if rc != KV_OK:
            _check(rc, "kv_softmax")
        return scores

    def kv_decode_attention(self, q: torch.Tensor, sm_scale: float, out: torch.Tensor = None, stream=None):
        """q: fp16 [B, Hq, 128] -> out fp32 [B, Hq, 128] = softmax(sm_scale * q K^T) V over the whole cache."""
        if out is None:
            done = self._calls.attention(q, sm_scale, stream)
            if done is not NotImplemented:
                return done
        assert q.dtype == torch.float16 and q.is_contiguous()
        assert q.shape == self._q_shape
        if out is None:
            out = torch.empty(self._q_shape, dtype=torch.float32, device=self.device)
        rc = _lib.kv_decode_attention(self.handle, q.data_ptr(), sm_scale, out.data_ptr(), _stream_ptr(stream))
        if rc != KV_OK:
            _check(rc, "kv_decode_attention")
        return out

    def kv_cache_stats(self, stream=None) -> kv_stats_t:
        st = kv_stats_t()
        _check(lib().kv_cache_stats(self.handle, C.byref(st), _stream_ptr(stream)), "kv_cache_stats")
        return st

    def kv_cache_release(self, stream=None):
        if self._calls.release(stream) is not NotImplemented:
            return
        rc = _lib.kv_cache_release(self.handle, _stream_ptr(stream))
        if rc != KV_OK:
            _check(rc, "kv_cache_release")

    def kv_cache_restore(self, tokens: int):
        if self._calls.restore(tokens) is not NotImplemented:
            return
        rc = _lib.kv_cache_restore(self.handle, tokens)
        if rc != KV_OK:
            _check(rc, "kv_cache_restore")

    # typed views of the raw buffers, for tests and tools
    def view(self, name, dtype):
        return self.tensors[name].view(dtype)


_TYPES = {torch.float16: KV_TYPE_FP16, torch.bfloat16: KV_TYPE_BF16, torch.float32: KV_TYPE_FP32}


def _refuse(what, why):
    raise PackKVError("%s: %s" % (what, why), KV_ERR_ARG)


class FP4Batch:
    """What a call on an FP4KVCache is about (kv_fp4_batch_t): sequence b holds lens[b] tokens, the last new_rows[b] of which
    are rows first_row[b], first_row[b] + 1, ... of the call's tensors.  lens, new_rows, first_row: int32 device tensors
    [batch]; page_table: int32 [batch, pages of a sequence at most].  Without new_rows every sequence has max_new of them, without first_row
    sequence b's begin at row b * max_new, without page_table sequence b has pages b * table_pages .. of the cache.
    The tensors are kept and read when a call's kernels run: a program changes their contents from step to step.
    What the batch was made of stays: its attributes are read-only."""

    def __init__(self, lens, max_new, page_table=None, new_rows=None, first_row=None, table_pages=None):
        what = "FP4Batch"
        if lens.dim() != 1 or lens.shape[0] < 1:
            _refuse(what, "lens is [batch]")
        batch, max_new, device = lens.shape[0], int(max_new), lens.device
        for name, t in (("lens", lens), ("new_rows", new_rows), ("first_row", first_row)):
            if t is not None and (t.dtype != torch.int32 or tuple(t.shape) != (batch,) or not t.is_contiguous()):
                _refuse(what, "%s is int32 [batch], contiguous" % name)
        if page_table is not None:
            if page_table.dtype != torch.int32 or page_table.dim() != 2 or page_table.shape[0] != batch or \
                    not page_table.is_contiguous() or table_pages not in (None, page_table.shape[1]):
                _refuse(what, "page_table is int32 [batch, table_pages], contiguous")
            table_pages = page_table.shape[1]
        elif table_pages is None:
            _refuse(what, "page_table or table_pages")
        if any(t is not None and t.device != device for t in (new_rows, first_row, page_table)):
            _refuse(what, "tensors of one device")
        table_pages = int(table_pages)
        if not (0 <= max_new < 2 ** 31 and 1 <= table_pages < 2 ** 31):
            _refuse(what, "max_new is 0 or more, table_pages 1 or more")
        self._tensors = (lens, new_rows, first_row, page_table)   # whose addresses the structure holds
        self._c = kv_fp4_batch_t(batch, max_new, table_pages,
                                 *(None if t is None else t.data_ptr() for t in (lens, new_rows, first_row, page_table)))
        self._ref, self._address, self._on = C.byref(self._c), C.addressof(self._c), device.index

    batch = property(lambda self: self._c.batch)
    max_new = property(lambda self: self._c.max_new)
    table_pages = property(lambda self: self._c.table_pages)
    device = property(lambda self: self._tensors[0].device)
    lens = property(lambda self: self._tensors[0])
    new_rows = property(lambda self: self._tensors[1])
    first_row = property(lambda self: self._tensors[2])
    page_table = property(lambda self: self._tensors[3])


class _Operators:
    """What calls on tensors of one device (self.device) have in common."""

    def _row_pitch(self, what, t, heads, dim, types):
        """Rows and row stride of t: [rows, heads, dim] or [batch, n, heads, dim], the heads of a row next to each other."""
        if t.device != self.device or t.dtype not in types:
            _refuse(what, "tensors of %s on %s" % (" or ".join(map(str, types)), self.device))
        shape, stride = t.shape, t.stride()
        if t.dim() not in (3, 4) or shape[-2:] != (heads, dim) or \
                stride[-1] != 1 or (heads > 1 and stride[-2] != dim):
            _refuse(what, "[rows, %d, %d], the heads of a row next to each other" % (heads, dim))
        if t.dim() == 3:
            rows, pitch = shape[0], stride[0]
        else:
            rows, pitch = shape[0] * shape[1], stride[1] if shape[1] > 1 else stride[0]
            if shape[0] > 1 and shape[1] > 1 and stride[0] != shape[1] * stride[1]:
                _refuse(what, "rows at even distances")
        return rows, pitch if rows > 1 else heads * dim

    def _made(self, what, function, *args):
        """function(*args) with the operators' device the current one."""
        if _current_device is not None and _current_device() == self.device.index:
            rc = function(*args[:-1], _stream_ptr(args[-1]))
        else:
            with torch.cuda.device(self.device):
                rc = function(*args[:-1], _stream_ptr(args[-1]))
        if rc != KV_OK:
            _check(rc, what)

    def _stream(self, stream):
        return torch.cuda.ExternalStream(stream, device=self.device) if isinstance(stream, int) else stream

    def _new(self, shape, dtype, stream, zeros=False):
        """An output, in memory that the stream which writes it may write at once; the current stream is taken to read it."""
        make = torch.zeros if zeros else torch.empty
        if stream is None:
            return make(shape, dtype=dtype, device=self.device)
        with torch.cuda.stream(stream):
            made = make(shape, dtype=dtype, device=self.device)
        made.record_stream(torch.cuda.current_stream(self.device))
        return made


class FP4KVCache(_Operators):
    """A 4-bit paged cache (packkv.h: MXFP4 rows in pages of 64 tokens): owns the pages and the workspace (torch tensors)
    and the kv_fp4_cache_t handle.  Which pages a sequence has, and how long it is, is the program's (FP4Batch).

    There is no backward pass: results carry no gradient, whatever k, v and q require.

    Calls run on torch's current stream, or on `stream` (a torch stream, or a hipStream_t as int).  On another stream than the current
    one the program sees to the order, as with torch's own operators: that stream waits for what made the inputs, and whoever reads
    the outputs for it.  Tensors of such a call may be dropped as soon as it returns: their memory is not reused before that stream is done.
    Calls on the current stream record nothing: a program that makes another stream current for some of them keeps the cache, and
    tensors made on other streams, until that one is done."""

    def __init__(self, n_pages, n_kv_heads, n_q_heads, head_dim=HEAD_DIM, device="cuda:0"):
        self.cfg = kv_fp4_config_t(n_kv_heads, n_q_heads, head_dim, n_pages)
        self.device = torch.device(device)
        sizes = kv_fp4_sizes_t()
        _check(lib().kv_fp4_query_sizes(C.byref(self.cfg), C.byref(sizes)), "kv_fp4_query_sizes")
        self.pages = torch.empty(sizes.pages, dtype=torch.uint8, device=self.device)
        self.workspace = torch.empty(sizes.workspace, dtype=torch.uint8, device=self.device)
        self.device = self.pages.device
        handle = C.c_void_p()
        with torch.cuda.device(self.device):
            torch.cuda.synchronize()
            _check(lib().kv_fp4_cache_create(C.byref(self.cfg), self.pages.data_ptr(), self.workspace.data_ptr(),
                                             C.byref(sizes), C.byref(handle)), "kv_fp4_cache_create")
        self._calls = _native.FP4Calls(n_kv_heads, n_q_heads, head_dim, str(self.device)) if _native else _PythonCalls()
        self.handle = handle
        self._calls.set_handle(handle.value)
        self.n_pages, self.n_kv_heads, self.n_q_heads, self.head_dim = n_pages, n_kv_heads, n_q_heads, head_dim

    def close(self):
        if getattr(self, "handle", None) and _lib is not None:
            self._calls.set_handle(0)
            _lib.kv_fp4_cache_destroy(self.handle)
        self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _rows(self, what, t, heads, types):
        return self._row_pitch(what, t, heads, self.head_dim, types)

    def _call(self, what, function, batch, stream, *args):
        if not self.handle:
            _refuse(what, "the cache is closed")
        if batch.device != self.device:
            _refuse(what, "the batch is on %s, the cache on %s" % (batch.device, self.device))
        self._made(what, function, self.handle, batch._ref, *args, stream)

    def _plain(self, what, name, t, dtype, shape):
        """t's address; None: null."""
        if t is None:
            return None
        if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous() or t.device != self.device:
            _refuse(what, "%s is contiguous %s %s on %s" % (name, dtype, tuple(shape), self.device))
        return t.data_ptr()

    def _keep(self, stream, batch, *tensors):
        """What a call on `stream` uses is not reused before `stream` is done with it, even if the program drops it now."""
        if stream is not None:
            for t in (*tensors, *batch._tensors, self.pages, self.workspace):
                if t is not None:
                    t.record_stream(stream)

    def kv_fp4_append(self, k, v, batch, stream=None):
        """k, v: fp16 or bf16 [rows, H_kv, D] (or [batch, n, H_kv, D]); may be parts of wider rows."""
        if self._calls.append(k, v, batch._address, batch._on, stream) is not NotImplemented:
            return
        half = (torch.float16, torch.bfloat16)
        rows, k_stride = self._rows("kv_fp4_append", k, self.n_kv_heads, half)
        v_rows, v_stride = self._rows("kv_fp4_append", v, self.n_kv_heads, half)
        if rows != v_rows or k.dtype != v.dtype:
            _refuse("kv_fp4_append", "k and v of as many rows and of one type")
        self._call("kv_fp4_append", _lib.kv_fp4_append, batch, stream, k.data_ptr(), k_stride, v.data_ptr(), v_stride,
                   _TYPES[k.dtype], rows)
        self._keep(self._stream(stream), batch, k, v)

    def kv_fp4_read(self, batch, n_rows, dtype=torch.float16, k=None, v=None, stream=None):
        """The batch's new rows as the cache holds them: (k, v), [n_rows, H_kv, D] of dtype; rows of no sequence are not written."""
        if k is None and v is None:
            done = self._calls.read(batch._address, batch._on, n_rows, dtype, stream)
            if done is not NotImplemented:
                return done
        elif k is not None and v is not None and k.dtype == dtype:
            done = self._calls.read_into(batch._address, batch._on, n_rows, k, v, stream)
            if done is not NotImplemented:
                return done
        what, shape = "kv_fp4_read", (n_rows, self.n_kv_heads, self.head_dim)
        if dtype not in _TYPES:
            _refuse(what, "dtype is float16, bfloat16 or float32")
        on = self._stream(stream)
        made = [self._new(shape, dtype, on) if t is None else t for t in (k, v)]
        for t in made:
            if t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous() or t.device != self.device:
                _refuse(what, "k and v are contiguous %s %s on %s" % (shape, dtype, self.device))
        self._call(what, _lib.kv_fp4_read, batch, stream, made[0].data_ptr(), made[1].data_ptr(), _TYPES[dtype], n_rows)
        self._keep(on, batch, *made)
        return tuple(made)

    def kv_fp4_attention(self, q, batch, sm_scale, window=0, sinks=0, out=None, lse=None, stream=None):
        """q: fp16 or bf16 [rows, H_q, D] (or [batch, n, H_q, D]) -> out [rows, H_q, D] of q's type (or of out's: fp16, bf16,
        fp32); lse: fp32 [rows, H_q] that gets the logarithms of the softmax sums.  Rows of no sequence are not written."""
        if out is None and lse is None:
            done = self._calls.attention(q, batch._address, batch._on, sm_scale, window, sinks, stream)
            if done is not NotImplemented:
                return done
        what = "kv_fp4_attention"
        rows, q_stride = self._rows(what, q, self.n_q_heads, (torch.float16, torch.bfloat16))
        on = self._stream(stream)
        if out is None:
            out = self._new(q.shape, q.dtype, on)
        elif out.dtype not in _TYPES or out.shape != q.shape or not out.is_contiguous() or out.device != self.device:
            _refuse(what, "out is contiguous, of q's shape and on its device")
        if lse is not None and (lse.dtype != torch.float32 or lse.shape != q.shape[:-1] or not lse.is_contiguous() or
                                lse.device != self.device):
            _refuse(what, "lse is contiguous fp32, of q's shape without the last axis")
        if not (0 <= window < 2 ** 31 and 0 <= sinks < 2 ** 31):
            _refuse(what, "window and sinks are 0 or more")
        self._call(what, _lib.kv_fp4_attention, batch, stream, q.data_ptr(), q_stride, _TYPES[q.dtype], rows, sm_scale,
                   window, sinks, out.data_ptr(), _TYPES[out.dtype], None if lse is None else lse.data_ptr())
        self._keep(on, batch, q, out, lse)
        return out

    def kv_fp4_weights(self, q, lse, batch, sm_scale, window=0, sinks=0, past=None, out=None, stream=None):
        """The attention weight that every cached token gets from the batch's new rows, on top of `past`: fp32 [batch, H_kv, tokens].
        q, sm_scale, window and sinks as kv_fp4_attention had them, lse as it gave them; past: of out's shape, or out
        itself; it counts for the tokens before the new rows.  Without out a new tensor of past's shape, or of the page table's
        width, zeros where the sequences have no tokens; places of out behind a sequence's tokens are not written."""
        if out is not None:
            done = self._calls.weights(q, lse, batch._address, batch._on, sm_scale, window, sinks, past, out, stream)
            if done is not NotImplemented:
                return done
        what, tokens = "kv_fp4_weights", 64 * batch.table_pages
        rows, q_stride = self._rows(what, q, self.n_q_heads, (torch.float16, torch.bfloat16))
        on = self._stream(stream)
        lse_at = self._plain(what, "lse", lse, torch.float32, q.shape[:-1])
        for t in (past, out):
            if t is not None:
                if t.dim() != 3:
                    _refuse(what, "past and out are [batch, H_kv, tokens]")
                tokens = t.shape[2]
        shape = (batch.batch, self.n_kv_heads, tokens)
        past_at = self._plain(what, "past", past, torch.float32, shape)
        if not (0 <= window < 2 ** 31 and 0 <= sinks < 2 ** 31):
            _refuse(what, "window and sinks are 0 or more")
        if out is None:
            out = self._new(shape, torch.float32, on, zeros=True)
        self._call(what, _lib.kv_fp4_weights, batch, stream, q.data_ptr(), q_stride, _TYPES[q.dtype], rows, sm_scale, window, sinks,
                   lse_at, past_at, self._plain(what, "out", out, torch.float32, shape), tokens)
        self._keep(on, batch, q, lse, past, out)
        return out

    def kv_fp4_select(self, mass, batch, keep, sinks=0, recent=0, budgets=None, kept=None, n_kept=None, stream=None):
        """Which tokens the batch's sequences keep, of mass [batch, H_kv, tokens] (kv_fp4_weights): (kept, n_kept), int32 [batch, H_kv,
        keep], positions in ascending order and -1 behind them, and int32 [batch].  All of a sequence of no more than keep (or
        budgets[b], int32 [batch]) tokens; else the first `sinks`, the last `recent` and the others of the largest mass.  kept, n_kept: where to;
        not the batch's lens, which the call reads."""
        if budgets is None and kept is None:
            done = self._calls.select(mass, batch._address, batch._on, keep, sinks, recent, n_kept, stream)
            if done is not NotImplemented:
                return done
        what = "kv_fp4_select"
        keep = int(keep)
        if mass.dim() != 3 or not (1 <= keep < 2 ** 31 and 0 <= sinks < 2 ** 31 and 0 <= recent < 2 ** 31):
            _refuse(what, "mass is [batch, H_kv, tokens], keep 1 or more, sinks and recent are 0 or more")
        tokens, on = mass.shape[2], self._stream(stream)
        mass_at = self._plain(what, "mass", mass, torch.float32, (batch.batch, self.n_kv_heads, tokens))
        budgets_at = self._plain(what, "budgets", budgets, torch.int32, (batch.batch,))
        shape = (batch.batch, self.n_kv_heads, keep)
        kept = self._new(shape, torch.int32, on) if kept is None else kept
        n_kept = self._new(shape[:1], torch.int32, on) if n_kept is None else n_kept
        self._call(what, _lib.kv_fp4_select, batch, stream, mass_at, tokens, keep, budgets_at, sinks, recent,
                   self._plain(what, "kept", kept, torch.int32, shape), self._plain(what, "n_kept", n_kept, torch.int32, shape[:1]))
        self._keep(on, batch, mass, budgets, kept, n_kept)
        return kept, n_kept

    def kv_fp4_compact(self, kept, n_kept, batch, to, mass=None, mass_out=None, stream=None):
        """Moves the tokens `kept` (int32 [batch, H_kv, keep]; the first n_kept[b], int32 [batch], of each) of batch's sequences together into
        the pages of `to`, an FP4Batch of as many sequences whose pages the call does not read (its lens may be n_kept).  mass: weights
        that go with them, [batch, H_kv, tokens], into mass_out, [batch, H_kv, any number] (without it new, [batch, H_kv, keep], zeros
        behind the kept ones), which is returned."""
        done = self._calls.compact(kept, n_kept, batch._address, batch._on, to._address, to._on, mass, mass_out, stream)
        if done is not NotImplemented:
            return done
        what, keep = "kv_fp4_compact", kept.shape[-1]
        shape, on = (batch.batch, self.n_kv_heads, keep), self._stream(stream)
        kept_at = self._plain(what, "kept", kept, torch.int32, shape)
        n_at = self._plain(what, "n_kept", n_kept, torch.int32, shape[:1])
        if keep >= 2 ** 31:
            _refuse(what, "kept has fewer than 2^31 positions to a head")
        if to.device != self.device or to.batch != batch.batch:
            _refuse(what, "both batches are on %s, of as many sequences" % self.device)
        if any(t is not None and t.dim() != 3 for t in (mass, mass_out)) or (mass is None and mass_out is not None):
            _refuse(what, "mass and mass_out are [batch, H_kv, tokens]")
        if mass is not None and mass_out is None:
            mass_out = self._new(shape, torch.float32, on, zeros=True)
        sizes = [0 if t is None else t.shape[2] for t in (mass, mass_out)]
        at = [self._plain(what, name, t, torch.float32, (*shape[:2], n)) for name, t, n in zip(("mass", "mass_out"), (mass, mass_out), sizes)]
        self._call(what, _lib.kv_fp4_compact, batch, stream, to._ref, kept_at, keep, n_at, at[0], sizes[0], at[1], sizes[1])
        self._keep(on, batch, kept, n_kept, mass, mass_out, *to._tensors)
        return mass_out


class Rotary(_Operators):
    """Rotary positions of query and key rows, before keys are appended to a cache and queries attend: the first `dims` channels of a
    head (all without it) in pairs (i, i + dims / 2), or (2i, 2i + 1) where interleaved, pair i turned by position * f_i.

    f_i = base^(-2i / dims), for contexts of `original` tokens; scaling makes them serve contexts `factor` times as long:
      "linear"  f_i / factor
      "base"    the base times factor^(dims / (dims - 2)): the last pair is turned factor times as slowly, the first as before
      "bands"   f_i / factor of pairs that turn less than `low` times over `original` tokens, f_i from `high` turns on, in between a
                blend that is linear in the turns
      "ramp"    f_i / factor of pairs that turn less than `slow` times, f_i of those that do more than `fast` times, in between a blend that is
                linear in i; the turned channels are multiplied by 0.1 ln(factor) + 1
    frequencies: all f_i, in radians, instead; magnitude: what the turned channels are multiplied by, instead.  Frequencies are
    doubles: an angle position * f_i is right to some 2^-52 of its size (5e-7 radians for f_i = 1 at the last of positions) before it is reduced.

    There is no backward pass; inverse=True is the transposed operation, which takes gradients back.  Streams as of FP4KVCache."""

    def __init__(self, head_dim, dims=None, base=10000.0, interleaved=False, scaling="none", factor=1.0, original=8192, low=1.0, high=4.0,
                 slow=1.0, fast=32.0, frequencies=None, magnitude=None, device="cuda:0"):
        what, dims = "Rotary", head_dim if dims is None else dims
        if head_dim % 2 or dims % 2 or not 2 <= dims <= head_dim:
            _refuse(what, "head_dim and dims are even, dims 2 .. head_dim")
        if frequencies is None:
            frequencies = self._frequencies(what, dims, base, scaling, factor, original, low, high, slow, fast)
            if magnitude is None:
                magnitude = 0.1 * math.log(factor) + 1.0 if scaling == "ramp" else 1.0
        frequencies = [float(f) for f in frequencies]
        magnitude = 1.0 if magnitude is None else float(magnitude)
        if len(frequencies) != dims // 2 or not all(map(math.isfinite, [*frequencies, magnitude])):
            _refuse(what, "dims / 2 finite frequencies, a finite magnitude")
        # 2^-64 of a turn, modulo a turn, as the signed numbers that torch has
        turns = [round(math.ldexp(math.fmod(f / (2.0 * math.pi), 1.0), 64)) % 2 ** 64 for f in frequencies]
        lib()
        self.head_dim, self.dims, self.interleaved, self.frequencies, self.magnitude = head_dim, dims, bool(interleaved), frequencies, magnitude
        self._turns = torch.tensor([t - 2 ** 64 if t >= 2 ** 63 else t for t in turns], dtype=torch.int64).to(device)
        self.device = self._turns.device
        self._c = kv_rotary_t(head_dim, dims, int(self.interleaved), magnitude, self._turns.data_ptr())
        self._ref = C.byref(self._c)
        self._calls = _native.RotaryCalls(C.addressof(self._c), head_dim, str(self.device)) if _native else _PythonCalls()

    @staticmethod
    def _frequencies(what, dims, base, scaling, factor, original, low, high, slow, fast):
        if not (base > 1.0 and factor > 0.0 and original > 0):
            _refuse(what, "base above 1, factor and original above 0")
        if scaling == "base":
            if dims == 2:
                _refuse(what, 'scaling "base" takes dims of 4 or more')
            base = base * factor ** (dims / (dims - 2))
        f = [base ** (-2.0 * i / dims) for i in range(dims // 2)]
        if scaling == "linear":
            return [x / factor for x in f]
        if scaling == "bands":
            if not 0.0 <= low < high:
                _refuse(what, "low is below high")
            own = [min(max((original * x / (2.0 * math.pi) - low) / (high - low), 0.0), 1.0) for x in f]   # what stays of f
        elif scaling == "ramp":
            if not 0.0 < slow <= fast:
                _refuse(what, "slow is at most fast")
            first, last = (dims * math.log(original / (2.0 * math.pi * turns)) / (2.0 * math.log(base)) for turns in (fast, slow))
            first, last = max(math.floor(first), 0), min(math.ceil(last), dims - 1)
            own = [1.0 - min(max((i - first) / max(last - first, 0.001), 0.0), 1.0) for i in range(dims // 2)]
        elif scaling in ("none", "base"):
            return f
        else:
            _refuse(what, 'scaling is "none", "linear", "base", "bands" or "ramp"')
        return [x * (w + (1.0 - w) / factor) for x, w in zip(f, own)]

    def kv_rotary(self, q, positions, k=None, out=None, k_out=None, inverse=False, stream=None):
        """q, k: fp16, bf16 or fp32 [rows, heads, head_dim] (or [batch, n, heads, head_dim]), both of one type; may be parts of wider rows.
        positions: int32, of q's shape without the last two axes.  Returns what became of q, or of (q, k); out and k_out: where to, which
        may be q and k themselves, and else nothing that overlaps what is read.  inverse: turned the other way."""
        done = self._calls.turn(q, positions, k, out, k_out, inverse, stream)
        if done is not NotImplemented:
            return done
        what, types = "kv_rotary", (torch.float16, torch.bfloat16, torch.float32)
        on, args, kept = self._stream(stream), [], [positions]
        if positions.dtype != torch.int32 or positions.device != self.device or not positions.is_contiguous() or \
                positions.shape != q.shape[:-2]:
            _refuse(what, "positions are contiguous int32 on %s, one to a row of q" % self.device)
        made = []
        for t, to in ((q, out), (k, k_out)):
            if t is None:
                if to is not None:
                    _refuse(what, "k_out without k")
                args += [None, 0, 0, None, 0]
                continue
            heads = t.shape[-2] if t.dim() > 2 else 0
            rows, pitch = self._row_pitch(what, t, heads, self.head_dim, types)
            if t.dtype != q.dtype or rows != positions.numel():
                _refuse(what, "q and k of one type, as many rows as positions")
            to = self._new(t.shape, t.dtype, on) if to is None else to
            to_rows, to_pitch = self._row_pitch(what, to, heads, self.head_dim, (t.dtype,))
            if to.shape != t.shape:
                _refuse(what, "an output is of its input's shape")
            args += [t.data_ptr(), pitch, min(heads, 65536), to.data_ptr(), to_pitch]     # (65535 at most: the library says so)
            made.append(to)
            kept += [t, to]
        self._made(what, _lib.kv_rotary, self._ref, positions.data_ptr(), positions.numel(), _TYPES[q.dtype], int(inverse), *args, stream)
        if on is not None:
            for t in (*kept, self._turns):
                t.record_stream(on)
        return made[0] if k is None else tuple(made)


def kv_fp16_k_matvec(k_cache, q, sm_scale, n_kv_heads, scores=None, stream=None):
    """k_cache: fp16 [B, H_kv, L, 128]; q: fp16 [B, Hq, 128] -> fp32 [B, Hq, L]."""
    B, H, L, Dd = k_cache.shape
    Hq = q.shape[1]
    if scores is None:
        scores = torch.empty(B, Hq, L, dtype=torch.float32, device=k_cache.device)
    _check(lib().kv_fp16_k_matvec(k_cache.data_ptr(), q.data_ptr(), sm_scale, scores.data_ptr(),
                                  scores.shape[2], B, H, Hq, L, _stream_ptr(stream)), "kv_fp16_k_matvec")
    return scores


def kv_fp16_v_matvec(v_cache, p, out=None, workspace=None, stream=None):
    """v_cache: fp16 [B, H_kv, L, 128]; p: fp32 [B, Hq, ld] -> fp32 [B, Hq, 128]."""
    B, H, L, Dd = v_cache.shape
    Hq = p.shape[1]
    if out is None:
        out = torch.empty(B, Hq, Dd, dtype=torch.float32, device=v_cache.device)
    if workspace is None:
        workspace = torch.empty(lib().kv_fp16_v_workspace_bytes(B, Hq), dtype=torch.uint8,
                                device=v_cache.device)
    _check(lib().kv_fp16_v_matvec(v_cache.data_ptr(), p.data_ptr(), p.shape[2], out.data_ptr(), B, H,
                                  Hq, L, workspace.data_ptr(), _stream_ptr(stream)), "kv_fp16_v_matvec")
    return out


def kv_stream_read(buf: torch.Tensor, checksum: torch.Tensor, stream=None):
    nbytes = buf.numel() * buf.element_size()
    _check(lib().kv_stream_read(buf.data_ptr(), nbytes - nbytes % 16, checksum.data_ptr(),
                                _stream_ptr(stream)), "kv_stream_read")
