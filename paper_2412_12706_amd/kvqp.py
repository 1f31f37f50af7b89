"""Thin ctypes binding of libkvqp.so (declarations: include/kvqp.h).

Argument marshalling only: every step of the path runs in the library's HIP
kernels.  PyTorch supplies device memory and streams.  There is no fallback:
if the library is missing, loading raises.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os
import struct as _struct
from dataclasses import dataclass, field
from operator import lt as _less

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libkvqp.so")

KVQP_OK = 0
KEY_PER_CHANNEL = 0
KEY_PER_TOKEN = 1
CACHE_AUTO, CACHE_STREAM, CACHE_KEEP = 0, 1, 2     # kvqp_cfg.decode_cache_hint
EXPORTS = ["kvqp_cache_sizes", "kvqp_cache_sizes_cap", "kvqp_outlier_sizes", "kvqp_workspace_bytes", "kvqp_compress",
           "kvqp_compress_ragged", "kvqp_quantize_selected", "kvqp_quantize_selected_ragged", "kvqp_append_tail", "kvqp_append_tail_ragged", "kvqp_decode_attn", "kvqp_decode_attn_static", "kvqp_decode_workspace_init",
           "kvqp_tree_workspace_bytes", "kvqp_tree_workspace_init", "kvqp_tree_attn", "kvqp_accumulate_weights", "kvqp_evict_workspace_bytes", "kvqp_evict",
           "kvqp_rope_frequencies", "kvqp_rope_table", "kvqp_rotate", "kvqp_paged_append", "kvqp_paged_workspace_bytes", "kvqp_paged_workspace_init",
           "kvqp_paged_attn", "kvqp_paged_read",
           "kvqp_strerror", "kvqp_version"]
MOST_ROWS = 256     # KVQP_MOST_ROWS
ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE, ROPE_PARTS = 0, 1, 2, 3     # scalings of rope_frequencies


class KvqpError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        super().__init__(f"{where}: {strerror(code)} ({code})")


class CfgStruct(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("batch", "n_q_heads", "n_kv_heads", "head_dim", "seq_len", "window",
                                         "pool_kernel", "budget", "bits", "group_size", "key_axis",
                                         "decode_splits")] + [("sm_scale", C.c_float), ("outlier_threshold", C.c_float),
                                                            ("decode_cache_hint", C.c_int32),
                                                            ("outlier_overflow_cap", C.c_int32)]


class CacheStruct(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k_codes", "v_codes", "k_scale", "k_zero", "v_scale", "v_zero",
                                          "tail_k", "tail_v")] + [(n, C.c_int32) for n in
                                                                  ("n_kept", "tail_len", "tail_cap", "n_cap")] + [
        ("head_n_kept", C.c_void_p), ("k_out", C.c_void_p), ("v_out", C.c_void_p), ("k_ovf", C.c_void_p),
        ("v_ovf", C.c_void_p)]


# The structs' bytes in one go (host order and alignment, as ctypes lays them out): a struct object with a field
# converted at a time takes 2.4 (cfg) and 3.6 us (cache) where these take 0.6 and 1.5.
_pack_cfg = _struct.Struct("12i2f2i").pack
_pack_cache = _struct.Struct("8P4i5P").pack
assert _struct.calcsize("12i2f2i") == C.sizeof(CfgStruct) and _struct.calcsize("8P4i5P") == C.sizeof(CacheStruct)
_pack_rope = _struct.Struct("P3i4x").pack           # kvqp_rope
_pack_rows = _struct.Struct("P3q").pack             # kvqp_rows
_pack_pages = _struct.Struct("6i9P").pack           # kvqp_pages

_lib = None
# Entry points once more, for this module's own calls: a cfg (and a cache that is only read) goes in as its bytes, a pointer as a number.
_fn = {}
_fn_rows = {}       # ... those of several query rows, and eviction


def lib():
    """Load the library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} not built; run `python -m paper_2412_12706_amd.build`")
        L = C.CDLL(LIB_PATH)
        L.kvqp_strerror.restype = C.c_char_p
        L.kvqp_strerror.argtypes = [C.c_int]
        L.kvqp_cache_sizes.argtypes = [C.POINTER(CfgStruct), C.c_int32, C.POINTER(C.c_size_t)]
        L.kvqp_cache_sizes_cap.argtypes = [C.POINTER(CfgStruct), C.c_int32, C.c_int32, C.POINTER(C.c_size_t)]
        L.kvqp_outlier_sizes.argtypes = [C.POINTER(CfgStruct), C.c_int32, C.POINTER(C.c_size_t)]
        L.kvqp_append_tail.argtypes = [C.POINTER(CfgStruct), C.POINTER(CacheStruct), C.c_int32, C.c_void_p]
        L.kvqp_append_tail_ragged.argtypes = [C.POINTER(CfgStruct), C.POINTER(CacheStruct), C.c_int32, C.POINTER(C.c_int32), C.c_void_p]
        L.kvqp_workspace_bytes.argtypes = [C.POINTER(CfgStruct), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]
        L.kvqp_compress.argtypes = [C.POINTER(CfgStruct), C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(CacheStruct),
                                    C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.kvqp_compress_ragged.argtypes = [C.POINTER(CfgStruct), C.c_void_p, C.c_void_p, C.c_void_p,
                                           C.POINTER(C.c_int32), C.POINTER(CacheStruct), C.c_void_p, C.c_void_p,
                                           C.c_void_p, C.c_size_t, C.c_void_p]
        L.kvqp_quantize_selected.argtypes = [C.POINTER(CfgStruct), C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32,
                                             C.POINTER(CacheStruct), C.c_void_p]
        L.kvqp_quantize_selected_ragged.argtypes = [C.POINTER(CfgStruct), C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32,
                                                    C.POINTER(C.c_int32), C.POINTER(CacheStruct), C.c_void_p]
        L.kvqp_decode_attn.argtypes = [C.POINTER(CfgStruct), C.c_void_p, C.POINTER(CacheStruct), C.c_void_p,
                                       C.c_void_p, C.c_size_t, C.c_void_p]
        L.kvqp_decode_attn_static.argtypes = [C.POINTER(CfgStruct), C.c_void_p, C.POINTER(CacheStruct), C.c_void_p, C.c_void_p]
        L.kvqp_decode_workspace_init.argtypes = [C.POINTER(CfgStruct), C.c_void_p, C.c_size_t, C.c_void_p]
        L.kvqp_tree_workspace_bytes.argtypes = L.kvqp_evict_workspace_bytes.argtypes = [C.POINTER(CfgStruct), C.c_int32, C.POINTER(C.c_size_t)]
        L.kvqp_tree_workspace_init.argtypes = [C.c_void_p, C.c_size_t, C.c_void_p]
        L.kvqp_tree_attn.argtypes = [C.POINTER(CfgStruct), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32,
                                     C.POINTER(CacheStruct), C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.kvqp_accumulate_weights.argtypes = [C.POINTER(CfgStruct), C.c_void_p, C.c_void_p, C.c_int32, C.POINTER(CacheStruct),
                                              C.c_void_p, C.c_int32, C.c_float, C.c_void_p]
        L.kvqp_evict.argtypes = [C.POINTER(CfgStruct), C.POINTER(CacheStruct), C.c_void_p, C.c_int32, C.c_int32, C.c_int32,
                                 C.POINTER(CacheStruct), C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        cfg, ptr, size, i32 = C.c_char_p, C.c_void_p, C.c_size_t, C.c_int32
        for name, args in {"kvqp_compress": (cfg, ptr, ptr, ptr, ptr, ptr, ptr, ptr, size, ptr),
                           "kvqp_append_tail": (cfg, ptr, i32, ptr),
                           "kvqp_decode_attn": (cfg, ptr, C.c_char_p, ptr, ptr, size, ptr),
                           "kvqp_decode_attn_static": (cfg, ptr, C.c_char_p, ptr, ptr)}.items():
            entry = L[name]
            entry.argtypes = args       # (before another thread, which may have loaded the library already, can find it)
            _fn[name] = entry
        for name, args in {"kvqp_tree_attn": (cfg, ptr, ptr, ptr, ptr, i32, i32, C.c_char_p, ptr, ptr, ptr, size, ptr),
                           "kvqp_accumulate_weights": (cfg, ptr, ptr, i32, C.c_char_p, ptr, i32, C.c_float, ptr),
                           "kvqp_evict": (cfg, C.c_char_p, ptr, i32, i32, i32, ptr, ptr, i32, ptr, ptr, size, ptr)}.items():
            entry = L[name]
            entry.argtypes = args
            _fn_rows[name] = entry
        dbl, i64 = C.c_double, C.c_int64
        L.kvqp_rope_frequencies.argtypes = [i32, dbl, i32, dbl, dbl, dbl, dbl, C.POINTER(dbl)]
        L.kvqp_rope_table.argtypes = [C.POINTER(dbl), i32, i32, dbl, ptr, ptr]
        L.kvqp_paged_workspace_bytes.argtypes = [C.POINTER(CfgStruct), i32, C.POINTER(size)]
        L.kvqp_paged_workspace_init.argtypes = [ptr, size, ptr]
        for name, args in {"kvqp_rotate": (cfg, i32, i32, i32, i32, cfg, cfg, ptr, i32, i32, i32, ptr),
                           "kvqp_paged_append": (cfg, cfg, cfg, ptr, i64, ptr, i64, ptr, i64, i32, ptr, ptr, ptr, ptr),
                           "kvqp_paged_attn": (cfg, cfg, ptr, i64, i32, ptr, i32, ptr, ptr, ptr, size, ptr),
                           "kvqp_paged_read": (cfg, cfg, i32, i32, ptr, ptr, ptr)}.items():
            entry = L[name]
            entry.argtypes = args
            _fn_rows[name] = entry
        _lib = L
    return _lib


def strerror(code: int) -> str:
    return lib().kvqp_strerror(code).decode()


def version() -> int:
    return int(lib().kvqp_version())


@dataclass
class Cfg:
    batch: int
    n_q_heads: int
    n_kv_heads: int
    head_dim: int = 128
    seq_len: int = 0
    window: int = 32
    pool_kernel: int = 7
    budget: int = 0
    bits: int = 4
    group_size: int = 32
    key_axis: int = KEY_PER_CHANNEL
    decode_splits: int = 0
    sm_scale: float = 128 ** -0.5
    outlier_threshold: float = 0.0
    decode_cache_hint: int = 0      # CACHE_AUTO / CACHE_STREAM / CACHE_KEEP
    outlier_overflow_cap: int = 0   # entries of one head's overflow list (outlier filtering)

    def _bytes(self) -> bytes:
        fields = (self.batch, self.n_q_heads, self.n_kv_heads, self.head_dim, self.seq_len, self.window,
                  self.pool_kernel, self.budget, self.bits, self.group_size, self.key_axis,
                  self.decode_splits, self.sm_scale, self.outlier_threshold, self.decode_cache_hint,
                  self.outlier_overflow_cap)
        try:
            return _pack_cfg(*fields)
        except (_struct.error, OverflowError):      # (numbers that do not fit are cut down by ctypes; the library judges the rest)
            return bytes(CfgStruct(*fields))

    def struct(self) -> CfgStruct:
        return CfgStruct.from_buffer_copy(self._bytes())

    @property
    def n_kept(self) -> int:
        return min(self.budget, self.seq_len - self.window)


def cache_sizes(cfg: Cfg, tail_cap: int):
    out = (C.c_size_t * 8)()
    rc = lib().kvqp_cache_sizes(C.byref(cfg.struct()), tail_cap, out)
    if rc:
        raise KvqpError(rc, "kvqp_cache_sizes")
    return list(out)


def cache_sizes_cap(cfg: Cfg, n_cap: int, tail_cap: int):
    out = (C.c_size_t * 8)()
    rc = lib().kvqp_cache_sizes_cap(C.byref(cfg.struct()), n_cap, tail_cap, out)
    if rc:
        raise KvqpError(rc, "kvqp_cache_sizes_cap")
    return list(out)


def outlier_sizes(cfg: Cfg, n_cap: int = 0):
    out = (C.c_size_t * 4)()
    rc = lib().kvqp_outlier_sizes(C.byref(cfg.struct()), n_cap, out)
    if rc:
        raise KvqpError(rc, "kvqp_outlier_sizes")
    return list(out)


def workspace_bytes(cfg: Cfg):
    a, b = C.c_size_t(), C.c_size_t()
    rc = lib().kvqp_workspace_bytes(C.byref(cfg.struct()), C.byref(a), C.byref(b))
    if rc:
        raise KvqpError(rc, "kvqp_workspace_bytes")
    return a.value, b.value


_NAMES = ("k_codes", "v_codes", "k_scale", "k_zero", "v_scale", "v_zero", "tail_k", "tail_v")


@dataclass
class Cache:
    """Device buffers of one layer's compressed cache (byte tensors) plus the ABI struct."""
    buffers: dict
    n_kept: int = 0
    tail_len: int = 0
    tail_cap: int = 0
    n_cap: int = 0      # tokens the packed buffers are laid out for; 0 = n_kept (compact)
    head_n_kept: object = None   # int32 device tensor [batch * Hkv] of a cache with head-level counts
    _keep: list = field(default_factory=list)

    def _bytes(self) -> bytes:
        # (an empty tensor's address is 0, which is NULL.  Written out: this runs on every call)
        b = self.buffers
        outs = (0, 0, 0, 0) if len(b) == 8 else [b[n].data_ptr() if n in b else 0 for n in ("k_out", "v_out", "k_ovf", "v_ovf")]
        fields = (b["k_codes"].data_ptr(), b["v_codes"].data_ptr(), b["k_scale"].data_ptr(), b["k_zero"].data_ptr(),
                  b["v_scale"].data_ptr(), b["v_zero"].data_ptr(), b["tail_k"].data_ptr(), b["tail_v"].data_ptr(),
                  self.n_kept, self.tail_len, self.tail_cap, self.n_cap,
                  0 if self.head_n_kept is None else self.head_n_kept.data_ptr(), *outs)
        try:
            return _pack_cache(*fields)
        except (_struct.error, OverflowError):      # (as in Cfg)
            return bytes(CacheStruct(*fields))

    def struct(self) -> CacheStruct:
        return CacheStruct.from_buffer_copy(self._bytes())

    def nbytes(self) -> int:
        return sum(t.numel() for t in self.buffers.values())


def alloc_cache(cfg: Cfg, tail_cap: int | None = None, device="cuda", n_cap: int = 0, ragged: bool = False) -> Cache:
    """Buffers for cfg's budget (compact) or, with n_cap, laid out for n_cap tokens per head;
    ragged adds the device array of head-level token counts."""
    import torch
    tail_cap = cfg.window if tail_cap is None else tail_cap
    sizes = cache_sizes_cap(cfg, n_cap, tail_cap) if n_cap else cache_sizes(cfg, tail_cap)
    bufs = {n: torch.empty(max(s, 0), dtype=torch.uint8, device=device) for n, s in zip(_NAMES, sizes)}
    if cfg.outlier_threshold > 0:
        for n, s in zip(("k_out", "v_out", "k_ovf", "v_ovf"), outlier_sizes(cfg, n_cap)):
            bufs[n] = torch.empty(s, dtype=torch.uint8, device=device)
    counts = torch.zeros(cfg.batch * cfg.n_kv_heads, dtype=torch.int32, device=device) if ragged else None
    return Cache(bufs, 0, 0, tail_cap, n_cap, counts)


def _stream_handle(stream) -> int:
    import torch
    if stream is None:
        try:                # the handle alone: the object that torch.cuda.current_stream() makes costs 3 us a call
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        except AttributeError:      # (undocumented names: a torch without them takes the public way)
            stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _stream_ptr(stream):
    return C.c_void_p(_stream_handle(stream))


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _addr(t):
    return None if t is None else t.data_ptr()


def _entry(name):
    if _lib is None:
        lib()
    return _fn[name]


def _memory_of(stream):
    """What is allocated in this context is the stream's: memory that is free on the current one may still have work pending there."""
    import torch
    if stream is None:
        return contextlib.nullcontext()
    return torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(stream.cuda_stream))


def _empty_output(like, stream):
    """Memory for a call's output; with a stream of its own it is that stream's, and kept until the current one, too, is done with it."""
    import torch
    if stream is None:
        return torch.empty_like(like)
    with _memory_of(stream):
        out = torch.empty_like(like)
    if out.is_cuda:
        out.record_stream(torch.cuda.current_stream(out.device))
    return out


def alloc_workspace(nbytes: int, device="cuda"):
    import torch
    return torch.empty(max(nbytes, 16), dtype=torch.uint8, device=device)


def decode_workspace_init(cfg: Cfg, workspace, stream=None):
    """kvqp_decode_workspace_init: zero the arrival counters at the head of a decode workspace."""
    rc = lib().kvqp_decode_workspace_init(C.byref(cfg.struct()), _ptr(workspace), workspace.numel(), _stream_ptr(stream))
    if rc:
        raise KvqpError(rc, "kvqp_decode_workspace_init")
    return workspace


def alloc_decode_workspace(cfg: Cfg, device="cuda", stream=None):
    """A decode workspace of kvqp_workspace_bytes' size, prepared for its first use; with a stream it is for calls on that one."""
    with _memory_of(stream):
        workspace = alloc_workspace(workspace_bytes(cfg)[1], device)
    return decode_workspace_init(cfg, workspace, stream)


def compress(cfg: Cfg, q_obs, k, v, cache: Cache, idx_out=None, workspace=None, stream=None, unrefined_out=None):
    """kvqp_compress: q_obs [B,Hq,W,D], k/v [B,Hkv,L,D] half tensors on the device;
    unrefined_out: int32 device tensor [B*Hkv] or None."""
    if workspace is None:
        with _memory_of(stream):
            workspace = alloc_workspace(workspace_bytes(cfg)[0], k.device)
    cs = cache.struct()
    rc = _entry("kvqp_compress")(cfg._bytes(), _addr(q_obs), _addr(k), _addr(v), C.byref(cs), _addr(idx_out),
                                 _addr(unrefined_out), workspace.data_ptr(), workspace.numel(), _stream_handle(stream))
    if rc:
        raise KvqpError(rc, "kvqp_compress")
    cache.n_kept, cache.tail_len = cs.n_kept, cs.tail_len
    return cache


def compress_ragged(cfg: Cfg, q_obs, k, v, head_budget, cache: Cache, idx_out=None, workspace=None, stream=None,
                    unrefined_out=None):
    """kvqp_compress_ragged: head_budget is a host sequence of batch * Hkv token counts."""
    if workspace is None:
        with _memory_of(stream):
            workspace = alloc_workspace(workspace_bytes(cfg)[0], k.device)
    n = cfg.batch * cfg.n_kv_heads
    if len(head_budget) != n:
        raise ValueError(f"head_budget needs {n} entries")
    hb = (C.c_int32 * n)(*[int(x) for x in head_budget])
    cs = cache.struct()
    rc = lib().kvqp_compress_ragged(C.byref(cfg.struct()), _ptr(q_obs), _ptr(k), _ptr(v), hb, C.byref(cs),
                                    _ptr(idx_out), _ptr(unrefined_out), _ptr(workspace), workspace.numel(),
                                    _stream_ptr(stream))
    if rc:
        raise KvqpError(rc, "kvqp_compress_ragged")
    cache.n_kept, cache.tail_len = cs.n_kept, cs.tail_len
    return cache


def quantize_selected(cfg: Cfg, k, v, idx, cache: Cache, stream=None):
    """kvqp_quantize_selected: idx int32 [B,Hkv,n_kept] ascending."""
    n_kept = int(idx.shape[-1])
    cs = cache.struct()
    rc = lib().kvqp_quantize_selected(C.byref(cfg.struct()), _ptr(k), _ptr(v), _ptr(idx) if n_kept else None, n_kept,
                                      C.byref(cs), _stream_ptr(stream))
    if rc:
        raise KvqpError(rc, "kvqp_quantize_selected")
    cache.n_kept, cache.tail_len = cs.n_kept, cs.tail_len
    return cache


def quantize_selected_ragged(cfg: Cfg, k, v, idx, head_count, cache: Cache, stream=None):
    """kvqp_quantize_selected_ragged: idx int32 [B,Hkv,n_kept]; head h uses its first head_count[h] entries."""
    n_kept = int(idx.shape[-1])
    n = cfg.batch * cfg.n_kv_heads
    if len(head_count) != n:
        raise ValueError(f"head_count needs {n} entries")
    hc = (C.c_int32 * n)(*[int(x) for x in head_count])
    cs = cache.struct()
    rc = lib().kvqp_quantize_selected_ragged(C.byref(cfg.struct()), _ptr(k), _ptr(v), _ptr(idx) if n_kept else None,
                                             n_kept, hc, C.byref(cs), _stream_ptr(stream))
    if rc:
        raise KvqpError(rc, "kvqp_quantize_selected_ragged")
    cache.n_kept, cache.tail_len = cs.n_kept, cs.tail_len
    return cache


def append_tail(cfg: Cfg, cache: Cache, n_tokens: int, stream=None):
    """kvqp_append_tail: the n_tokens oldest tail rows join the low-precision part."""
    cs = cache.struct()
    rc = _entry("kvqp_append_tail")(cfg._bytes(), C.byref(cs), n_tokens, _stream_handle(stream))
    if rc:
        raise KvqpError(rc, "kvqp_append_tail")
    cache.n_kept, cache.tail_len = cs.n_kept, cs.tail_len
    return cache


def append_tail_ragged(cfg: Cfg, cache: Cache, n_tokens: int, head_count, stream=None):
    """kvqp_append_tail_ragged: every head takes the n_tokens oldest tail rows at its own count
    (head_count: the heads' current counts, a host sequence)."""
    n = cfg.batch * cfg.n_kv_heads
    if len(head_count) != n:
        raise ValueError(f"head_count needs {n} entries")
    hc = (C.c_int32 * n)(*[int(x) for x in head_count])
    cs = cache.struct()
    rc = lib().kvqp_append_tail_ragged(C.byref(cfg.struct()), C.byref(cs), n_tokens, hc, _stream_ptr(stream))
    if rc:
        raise KvqpError(rc, "kvqp_append_tail_ragged")
    cache.n_kept, cache.tail_len = cs.n_kept, cs.tail_len
    return cache


def decode_attn(cfg: Cfg, q, cache: Cache, out=None, workspace=None, stream=None):
    """kvqp_decode_attn: q [B,Hq,D] half -> out [B,Hq,D] half."""
    if out is None:
        out = _empty_output(q, stream)
    if workspace is None:
        workspace = alloc_decode_workspace(cfg, q.device, stream)
    rc = _entry("kvqp_decode_attn")(cfg._bytes(), _addr(q), cache._bytes(), out.data_ptr(), workspace.data_ptr(),
                                    workspace.numel(), _stream_handle(stream))
    if rc:
        raise KvqpError(rc, "kvqp_decode_attn")
    return out


def decode_attn_static(cfg: Cfg, q, cache: Cache, out, stream=None):
    """kvqp_decode_attn_static: the decode step on the library's own scratch array; out is the caller's."""
    rc = _entry("kvqp_decode_attn_static")(cfg._bytes(), _addr(q), cache._bytes(), _addr(out), _stream_handle(stream))
    if rc:
        raise KvqpError(rc, "kvqp_decode_attn_static")
    return out


# ---- several query rows per call, and eviction ----

def _want(what, t, dtype, shape, device):
    """A tensor argument as the library takes it: its type and shape, contiguous, on the GPU of the others (its number)."""
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != device or device < 0:
        raise ValueError(f"{what}: a contiguous {dtype} tensor of shape {tuple(shape)} on GPU {device} is needed, not {t.dtype} {tuple(t.shape)}"
                         f"{'' if t.is_contiguous() else ', strided'} on {t.device}")


def _same_device(name, device, *tensors):
    for t in tensors:
        if t.numel() and t.get_device() != device:
            raise ValueError(f"{name}: a buffer on {t.device} and tensors on GPU {device}")


def _check_room(what, cfg: Cfg, cache: Cache, rows: int, device):
    """A cache that a call fills: its buffers hold so many packed tokens per head, and the tail rows that they state."""
    b, heads, bits, group = cache.buffers, cfg.batch * cfg.n_kv_heads, cfg.bits, max(cfg.group_size, 1)      # (what a cfg may not hold the library refuses)
    block = 64 if bits == 2 else 32
    codes = heads * 16 * bits
    per_token = 0 if bits == 16 else heads * rows * (cfg.head_dim // group) * 2
    key = per_token if bits == 16 or cfg.key_axis == KEY_PER_TOKEN else heads * -(-rows // group) * cfg.head_dim * 2
    tail = heads * cache.tail_cap * cfg.head_dim * 2
    need = (codes * rows, codes * block * -(-rows // block), key, key, per_token, per_token, tail, tail)
    have = (b["k_codes"].nbytes, b["v_codes"].nbytes, b["k_scale"].nbytes, b["k_zero"].nbytes, b["v_scale"].nbytes, b["v_zero"].nbytes,
            b["tail_k"].nbytes, b["tail_v"].nbytes)        # (written out: this runs on every call)
    if any(map(_less, have, need)):
        name, n, m = next(x for x in zip(_NAMES, have, need) if x[1] < x[2])
        raise ValueError(f"{what} has no room for {rows} packed tokens and {cache.tail_cap} tail rows per head: {name} holds {n} bytes of {m}")
    counts = cache.head_n_kept
    if counts is not None:
        import torch
        _want(f"{what}.head_n_kept", counts, torch.int32, counts.shape if counts.numel() == heads else (heads,), device)


_raw = None         # torch's current device, and its current stream's handle on one, as plain functions (the public ones take 3 us more)


def _raw_functions():
    global _raw
    import torch
    try:
        _raw = (torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream)
    except AttributeError:      # (undocumented names: a torch without them takes the public way)
        _raw = (torch.cuda.current_device, lambda device: torch.cuda.current_stream(device).cuda_stream)
    return _raw


def _call(name, device, stream, args):
    """Calls an entry point with that GPU as the current one."""
    if _lib is None:
        lib()
    current, handle = _raw or _raw_functions()
    if current() != device:
        import torch
        with torch.cuda.device(device):
            rc = _fn_rows[name](*args, _stream_handle(stream))
    else:
        rc = _fn_rows[name](*args, handle(device) if stream is None else stream.cuda_stream)
    if rc:
        raise KvqpError(rc, name)


def _sized(entry, cfg: Cfg, n: int) -> int:
    out = C.c_size_t()
    rc = getattr(lib(), entry)(C.byref(cfg.struct()), n, C.byref(out))
    if rc:
        raise KvqpError(rc, entry)
    return out.value


def tree_workspace_bytes(cfg: Cfg, n_rows: int) -> int:
    return _sized("kvqp_tree_workspace_bytes", cfg, n_rows)


def tree_workspace_init(workspace, stream=None):
    """kvqp_tree_workspace_init: zero the arrival counters at the head of a workspace of tree_attn."""
    import torch
    with torch.cuda.device(workspace.device):
        rc = lib().kvqp_tree_workspace_init(_ptr(workspace), workspace.numel() * workspace.element_size(), _stream_ptr(stream))
    if rc:
        raise KvqpError(rc, "kvqp_tree_workspace_init")
    return workspace


def alloc_tree_workspace(cfg: Cfg, n_rows: int, device="cuda", stream=None):
    """A workspace for tree_attn calls of at most n_rows rows on caches of any token count, prepared for its first use; with a stream it is for calls
    on that one."""
    nbytes = tree_workspace_bytes(cfg, n_rows)
    with _memory_of(stream):
        workspace = alloc_workspace(nbytes, device)
    return tree_workspace_init(workspace, stream) if nbytes else workspace


def evict_workspace_bytes(cfg: Cfg, n_kept: int) -> int:
    return _sized("kvqp_evict_workspace_bytes", cfg, n_kept)


def alloc_evict_workspace(cfg: Cfg, cache: Cache, device="cuda"):
    """A workspace for evictions from caches of at most this one's count of packed tokens."""
    return alloc_workspace(evict_workspace_bytes(cfg, cache.n_kept), device)


def tree_mask(parents, device="cuda"):
    """The mask of a drafted tree: parents[i] is the number of the drafted token that token i follows, or -1 where it follows the
    sequence itself; a sequence of such sequences makes one mask per batch item.  Every token sees itself and its ancestors.
    int32 [n, ceil(n / 32)] or [batch, n, ceil(n / 32)]."""
    import torch
    if hasattr(parents, "tolist"):      # (an element of a tensor is a tensor, too)
        parents = parents.tolist()
    several = len(parents) > 0 and hasattr(parents[0], "__len__")
    out = []
    for tree in (parents if several else [parents]):
        seen = []
        for i, p in enumerate(tree):
            p = int(p)
            if not -1 <= p < i:
                raise ValueError(f"token {i} cannot follow token {p}: a parent comes before its children")
            seen.append((seen[p] if p >= 0 else 0) | 1 << i)
        words = (len(seen) + 31) // 32
        out.append([[_signed32(s >> 32 * w & 0xFFFFFFFF) for w in range(words)] for s in seen])
    return torch.tensor(out if several else out[0], dtype=torch.int32).to(device)


def _signed32(u: int) -> int:
    return u - (1 << 32) if u >> 31 else u


def tree_attn(cfg: Cfg, q, k_new, v_new, mask, cache: Cache, out=None, lse=None, workspace=None, stream=None):
    """kvqp_tree_attn: q [B,Hq,N,D], k_new / v_new [B,Hkv,N,D] half -> out [B,Hq,N,D] half; mask int32 [N,ceil(N/32)] or
    [B,N,ceil(N/32)] (tree_mask makes one), or None for a chain; lse float32 [B,Hq,N] or None."""
    import torch
    b, half, device = cfg.batch, torch.float16, q.get_device()
    n = q.shape[2] if q.dim() == 4 else 0
    _want("q", q, half, (b, cfg.n_q_heads, n, cfg.head_dim), device)
    kv = (b, cfg.n_kv_heads, n, cfg.head_dim)
    _want("k_new", k_new, half, kv, device)
    _want("v_new", v_new, half, kv, device)
    per_batch = 0
    if mask is not None:
        per_batch = int(mask.dim() == 3)
        words = (n + 31) // 32
        _want("mask", mask, torch.int32, (b, n, words) if per_batch else (n, words), device)
    if lse is not None:
        _want("lse", lse, torch.float32, (b, cfg.n_q_heads, n), device)
    if out is None:
        out = _empty_output(q, stream)
    else:
        _want("out", out, half, q.shape, device)
    if workspace is None:
        workspace = alloc_tree_workspace(cfg, n, q.device, stream)
    _same_device("tree_attn", device, workspace, cache.buffers["k_codes"])
    _call("kvqp_tree_attn", device, stream,
          (cfg._bytes(), q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), _addr(mask), per_batch, n, cache._bytes(), out.data_ptr(), _addr(lse),
           workspace.data_ptr(), workspace.numel() * workspace.element_size()))
    return out


def accumulate_weights(cfg: Cfg, q, lse, cache: Cache, weights, decay: float = 1.0, stream=None):
    """kvqp_accumulate_weights: q [B,Hq,N,D] half and lse [B,Hq,N] float32 of the last N tail rows' queries; weights float32
    [B,Hkv,w_cap] is updated in place and returned."""
    import torch
    b, device = cfg.batch, q.get_device()
    n, cap = (q.shape[2] if q.dim() == 4 else 0), weights.shape[-1]
    _want("q", q, torch.float16, (b, cfg.n_q_heads, n, cfg.head_dim), device)
    _want("lse", lse, torch.float32, (b, cfg.n_q_heads, n), device)
    _want("weights", weights, torch.float32, (b, cfg.n_kv_heads, cap), device)
    _same_device("accumulate_weights", device, cache.buffers["k_codes"])
    _call("kvqp_accumulate_weights", device, stream,
          (cfg._bytes(), q.data_ptr(), lse.data_ptr(), n, cache._bytes(), weights.data_ptr(), cap, decay))
    return weights


def evict(cfg: Cfg, cache: Cache, weights, n_keep: int, dst: Cache, weights_out=None, unit: int = 1, idx_out=None, workspace=None,
          stream=None):
    """kvqp_evict: the n_keep packed tokens per head with the highest weights (float32 [B,Hkv,w_cap]) go to dst, a cache with
    buffers of its own, with the tail; weights_out float32 [B,Hkv,w_cap_out], idx_out int32 [B,Hkv,kept] or None.  Returns dst."""
    import torch
    heads, device, cap, cap_out = (cfg.batch, cfg.n_kv_heads), weights.get_device(), weights.shape[-1], 0
    _want("weights", weights, torch.float32, (*heads, cap), device)
    if weights_out is not None:
        cap_out = weights_out.shape[-1]
        _want("weights_out", weights_out, torch.float32, (*heads, cap_out), device)
    n_keep = max(-1, min(n_keep, (1 << 31) - 1))          # (as many as a C integer holds)
    kept = min(n_keep, cache.n_kept)
    if cache.head_n_kept is None and n_keep < cache.n_kept and unit > 1:
        short = cache.n_kept % unit
        kept = short + (n_keep - short) // unit * unit
    if idx_out is not None:
        _want("idx_out", idx_out, torch.int32, (*heads, kept), device)
    _check_room("evict: dst", cfg, dst, dst.n_cap or (kept + 31) // 32 * 32, device)
    if workspace is None:
        with _memory_of(stream):
            workspace = alloc_evict_workspace(cfg, cache, weights.device)
    _same_device("evict", device, workspace, cache.buffers["k_codes"], dst.buffers["k_codes"])
    cs = dst.struct()
    _call("kvqp_evict", device, stream,
          (cfg._bytes(), cache._bytes(), weights.data_ptr(), cap, n_keep, unit, C.byref(cs), _addr(weights_out), cap_out, _addr(idx_out),
           workspace.data_ptr(), workspace.numel() * workspace.element_size()))
    dst.n_kept, dst.tail_len = cs.n_kept, cs.tail_len
    return dst


# ---- rotary positions, and the paged cache of 8-bit codes ----

def rope_frequencies(rot_dim: int = 128, base: float = 10000.0, scaling: int = ROPE_PLAIN, factor: float = 1.0, context: float = 1.0,
                     low: float = 1.0, high: float = 32.0):
    """kvqp_rope_frequencies: the rot_dim / 2 frequencies, a list of floats."""
    out = (C.c_double * (max(rot_dim, 2) // 2))()
    rc = lib().kvqp_rope_frequencies(rot_dim, base, scaling, factor, context, low, high, out)
    if rc:
        raise KvqpError(rc, "kvqp_rope_frequencies")
    return list(out)


class _Described:
    """An object whose fields describe device memory: they are checked and packed for the library once, and again after one of them is assigned
    or has other memory than it had.  (Calls of other threads may go on meanwhile: what they packed carries the state that they began with.)"""
    _packed = None      # (state, where the memory is, bytes)

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        object.__setattr__(self, "_state", object())

    def _pack(self, fits, *of):
        packed = (self._state, fits, self._checked(*of))
        object.__setattr__(self, "_packed", packed)
        return packed


@dataclass
class Rope(_Described):
    """A table of cosines and sines [n_positions, rot_dim / 2, 2] (float32, on the device) and how it turns a row.  The table may be replaced; its
    shape does not change in place."""
    table: object
    rot_dim: int = 128
    interleaved: bool = False

    def _bytes(self, device) -> bytes:
        fits, packed = (device, self.table.data_ptr()), self._packed
        if packed is None or packed[0] is not self._state or packed[1] != fits:
            packed = self._pack(fits, device)
        return packed[2]

    def _checked(self, device) -> bytes:
        import torch
        t = self.table
        _want("rope.table", t, torch.float32, (t.shape[0], self.rot_dim // 2, 2), device)
        return _pack_rope(t.data_ptr(), t.shape[0], self.rot_dim, bool(self.interleaved))


def rope_table(n_positions: int, inv_freq, magnitude: float = 1.0, interleaved: bool = False, device="cuda", stream=None) -> Rope:
    """kvqp_rope_table: a Rope for positions 0 .. n_positions - 1 with these frequencies (rope_frequencies gives some)."""
    import torch
    pairs = len(inv_freq)
    table = _empty_rows((max(n_positions, 1), pairs, 2), torch.float32, device, stream)
    with torch.cuda.device(table.device):
        rc = lib().kvqp_rope_table((C.c_double * pairs)(*inv_freq), 2 * pairs, n_positions, magnitude, table.data_ptr(), _stream_ptr(stream))
    if rc:
        raise KvqpError(rc, "kvqp_rope_table")
    return Rope(table, 2 * pairs, interleaved)


def _row_type(what, t, device, dtype=None):
    """0 or 1 (KVQP_HALF, KVQP_BFLOAT16) of a tensor [B, H, N, 128] of rows, whose channels lie next to each other; and its other strides."""
    import torch
    kind = t.dtype
    if t.get_device() == device >= 0 and (kind is dtype if dtype is not None else kind is torch.float16 or kind is torch.bfloat16) and t.dim() == 4 and t.shape[3] == 128:
        a, b, c, one = t.stride()
        if one == 1:
            return int(kind is torch.bfloat16), (a, b, c)
    raise ValueError(f"{what}: a tensor [B, H, N, 128] of {dtype or 'float16 or bfloat16'} on GPU {device} is needed, with adjacent channels, not {t.dtype} "
                     f"{tuple(t.shape)} with strides {t.stride()} on {t.device}")


def _empty_rows(shape, dtype, device, stream):
    """Memory for a call's output, as _empty_output."""
    import torch
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with _memory_of(stream):
        out = torch.empty(shape, dtype=dtype, device=device)
    if out.is_cuda:
        out.record_stream(torch.cuda.current_stream(out.device))
    return out


def rotate(rope: Rope, x, positions=None, first: int = 0, out=None, inverse: bool = False, stream=None):
    """kvqp_rotate: x [B,H,N,128] float16 or bfloat16, strided as it may be, -> out (contiguous unless given; x itself is allowed).
    positions int32 [N] or [B,N], or None for first, first + 1, ..."""
    device = x.get_device()
    kind, x_strides = _row_type("x", x, device)
    turn = rope._bytes(device)
    shape = x.shape
    b, h, n, _ = shape
    at = per_batch = 0
    if positions is not None:
        import torch
        per_batch = int(positions.dim() == 2)
        _want("positions", positions, torch.int32, (b, n) if per_batch else (n,), device)
        at = positions.data_ptr()
    if out is None:
        out = _empty_rows(shape, x.dtype, x.device, stream)
    _, out_strides = _row_type("out", out, device, x.dtype)
    if out.shape != shape:
        raise ValueError(f"out: shape {tuple(shape)} is needed, not {tuple(out.shape)}")
    if b == 0 or h == 0 or n == 0:
        return out
    _call("kvqp_rotate", device, stream,
          (turn, kind, b, h, n, _pack_rows(x.data_ptr(), *x_strides), _pack_rows(out.data_ptr(), *out_strides), at, per_batch, first, 1 if inverse else 0))
    return out


@dataclass
class Pages(_Described):
    """Device buffers of one layer's paged cache (kvqp_pages): k_codes [n_pages,Hkv,P,128] and v_codes [n_pages,Hkv,128,P], both float8_e4m3fn or both int8;
    k_scale, v_scale float32 [n_pages,Hkv]; open_k, open_v [n_open,Hkv,2P,128] float16 or bfloat16; table int32 [B,max_pages]; lengths int32 [B]; open_slot
    int32 [B] or None.  Their contents change as they may, and any may be replaced; shapes do not change in place."""
    k_codes: object
    v_codes: object
    k_scale: object
    v_scale: object
    open_k: object
    open_v: object
    table: object
    lengths: object
    open_slot: object = None

    @property
    def page_tokens(self) -> int:
        return self.k_codes.shape[2]

    def _bytes(self, cfg: Cfg, device) -> bytes:
        """kvqp_pages, with all buffers as it states them."""
        slot = self.open_slot
        fits = (device, cfg.n_kv_heads, cfg.batch, self.k_codes.data_ptr(), self.v_codes.data_ptr(), self.k_scale.data_ptr(), self.v_scale.data_ptr(), self.open_k.data_ptr(),
                self.open_v.data_ptr(), self.table.data_ptr(), self.lengths.data_ptr(), None if slot is None else slot.data_ptr())
        packed = self._packed
        if packed is None or packed[0] is not self._state or packed[1] != fits:
            packed = self._pack(fits, cfg, device)
        return packed[2]

    def _checked(self, cfg: Cfg, device) -> bytes:
        import torch
        k = self.k_codes
        n, _, p, _ = k.shape
        half, form = self.open_k.dtype, k.dtype
        if form not in (torch.float8_e4m3fn, torch.int8) or half not in (torch.float16, torch.bfloat16):
            raise ValueError(f"pages: codes of float8_e4m3fn or int8 and open rows of float16 or bfloat16 are needed, not {form} and {half}")
        kv, n_open, most = cfg.n_kv_heads, self.open_k.shape[0], self.table.shape[-1]
        _want("pages.k_codes", k, form, (n, kv, p, 128), device)
        _want("pages.v_codes", self.v_codes, form, (n, kv, 128, p), device)
        _want("pages.k_scale", self.k_scale, torch.float32, (n, kv), device)
        _want("pages.v_scale", self.v_scale, torch.float32, (n, kv), device)
        _want("pages.open_k", self.open_k, half, (n_open, kv, 2 * p, 128), device)
        _want("pages.open_v", self.open_v, half, (n_open, kv, 2 * p, 128), device)
        _want("pages.table", self.table, torch.int32, (cfg.batch, most), device)
        _want("pages.lengths", self.lengths, torch.int32, (cfg.batch,), device)
        if self.open_slot is not None:
            _want("pages.open_slot", self.open_slot, torch.int32, (cfg.batch,), device)
        return _pack_pages(half is torch.bfloat16, form is torch.int8, p, n, most, n_open, k.data_ptr(), self.v_codes.data_ptr(), self.k_scale.data_ptr(),
                           self.v_scale.data_ptr(), self.open_k.data_ptr(), self.open_v.data_ptr(), self.table.data_ptr(), self.lengths.data_ptr(),
                           _addr(self.open_slot) or 0)


def alloc_pages(cfg: Cfg, n_pages: int, max_pages: int, page_tokens: int = 16, dtype=None, form="e4m3", n_open: int | None = None, device="cuda") -> Pages:
    """Buffers for n_pages pages and cfg.batch sequences of at most max_pages of them: lengths 0, a table without pages (-1), for the caller to fill.
    dtype: of the rows (float16 unless given); form: "e4m3" or "int8"; n_open: places for open blocks (one per sequence unless given)."""
    import torch
    if form not in ("e4m3", "int8"):
        raise ValueError(f"form: \"e4m3\" or \"int8\", not {form!r}")
    heads, n_open = cfg.n_kv_heads, cfg.batch if n_open is None else n_open
    code = {"dtype": torch.float8_e4m3fn if form == "e4m3" else torch.int8, "device": device}
    row = {"dtype": dtype or torch.float16, "device": device}
    scale, count = {"dtype": torch.float32, "device": device}, {"dtype": torch.int32, "device": device}
    return Pages(torch.empty((n_pages, heads, page_tokens, 128), **code), torch.empty((n_pages, heads, 128, page_tokens), **code),
                 torch.empty((n_pages, heads), **scale), torch.empty((n_pages, heads), **scale),
                 torch.empty((n_open, heads, 2 * page_tokens, 128), **row), torch.empty((n_open, heads, 2 * page_tokens, 128), **row),
                 torch.full((cfg.batch, max_pages), -1, **count), torch.zeros(cfg.batch, **count))


def _packed_rows(what, t, heads, n, device, dtype):
    """The stride of the rows of a tensor [n, heads, 128] whose heads lie next to each other."""
    if t.dtype is dtype and t.get_device() == device >= 0 and t.shape == (n, heads, 128):
        stride = t.stride()
        if stride[2] == 1 and (stride[1] == 128 or heads == 1):
            return stride[0] if n > 1 else heads * 128
    raise ValueError(f"{what}: a {dtype} tensor of shape {(n, heads, 128)} on GPU {device} is needed, with adjacent heads and channels, not {t.dtype} "
                     f"{tuple(t.shape)} with strides {t.stride()} on {t.device}")


def _want_starts(cfg: Cfg, row_start, device):
    if row_start is not None:
        import torch
        _want("row_start", row_start, torch.int32, (cfg.batch + 1,), device)


def paged_append(cfg: Cfg, pages: Pages, k, v, row_start=None, q=None, rope: Rope | None = None, positions=None, q_out=None, stream=None):
    """kvqp_paged_append: k, v [n,Hkv,128] and q [n,Hq,128] or None, slices of a fused projection allowed; pages.lengths include the new rows.
    row_start int32 [B+1], or None for one row per sequence; positions int32 [n] or None.  Returns the rotated queries (q_out), or None."""
    import torch
    device, dtype, n = k.get_device(), pages.open_k.dtype, k.shape[0]
    layout = pages._bytes(cfg, device)
    ks, vs = _packed_rows("k", k, cfg.n_kv_heads, n, device, dtype), _packed_rows("v", v, cfg.n_kv_heads, n, device, dtype)
    _want_starts(cfg, row_start, device)
    qs = 0
    if q is not None:
        qs = _packed_rows("q", q, cfg.n_q_heads, n, device, dtype)
        if q_out is None:
            q_out = _empty_rows((n, cfg.n_q_heads, 128), dtype, q.device, stream)
        else:
            _want("q_out", q_out, dtype, (n, cfg.n_q_heads, 128), device)
    elif q_out is not None:
        raise ValueError("q_out: there is no q")
    turn = None if rope is None else rope._bytes(device)
    if positions is not None:
        _want("positions", positions, torch.int32, (n,), device)
    if n == 0 and row_start is not None:
        return q_out
    _call("kvqp_paged_append", device, stream,
          (cfg._bytes(), layout, turn, _addr(q), qs, k.data_ptr(), ks, v.data_ptr(), vs, n, _addr(row_start),
           _addr(positions), _addr(q_out)))
    return q_out


def paged_workspace_bytes(cfg: Cfg, n_rows: int) -> int:
    return _sized("kvqp_paged_workspace_bytes", cfg, n_rows)


def paged_workspace_init(workspace, stream=None):
    """kvqp_paged_workspace_init: zero the arrival counters at the head of a workspace of paged_attn."""
    import torch
    with torch.cuda.device(workspace.device):
        rc = lib().kvqp_paged_workspace_init(_ptr(workspace), workspace.numel() * workspace.element_size(), _stream_ptr(stream))
    if rc:
        raise KvqpError(rc, "kvqp_paged_workspace_init")
    return workspace


def alloc_paged_workspace(cfg: Cfg, n_rows: int, device="cuda", stream=None):
    """A workspace for paged_attn calls of at most n_rows rows, prepared for its first use; with a stream it is for calls on that one."""
    with _memory_of(stream):
        workspace = alloc_workspace(paged_workspace_bytes(cfg, n_rows), device)
    return paged_workspace_init(workspace, stream)


def paged_attn(cfg: Cfg, pages: Pages, q, row_start=None, window: int = 0, out=None, lse=None, workspace=None, stream=None):
    """kvqp_paged_attn: q [n,Hq,128] (rows apart as they may be) -> out [n,Hq,128]; row_start int32 [B+1], or None for one row per sequence;
    lse float32 [n,Hq] or None."""
    import torch
    device, dtype, n = q.get_device(), pages.open_k.dtype, q.shape[0]
    layout = pages._bytes(cfg, device)
    qs = _packed_rows("q", q, cfg.n_q_heads, n, device, dtype)
    _want_starts(cfg, row_start, device)
    if lse is not None:
        _want("lse", lse, torch.float32, (n, cfg.n_q_heads), device)
    if out is None:
        out = _empty_rows((n, cfg.n_q_heads, 128), dtype, q.device, stream)
    else:
        _want("out", out, dtype, (n, cfg.n_q_heads, 128), device)
    if n == 0 and row_start is not None:
        return out
    if workspace is None:
        workspace = alloc_paged_workspace(cfg, n, q.device, stream)
    _same_device("paged_attn", device, workspace)
    _call("kvqp_paged_attn", device, stream,
          (cfg._bytes(), layout, q.data_ptr(), qs, n, _addr(row_start), window, out.data_ptr(), _addr(lse), workspace.data_ptr(),
           workspace.numel() * workspace.element_size()))
    return out


def paged_read(cfg: Cfg, pages: Pages, count: int, first: int = 0, k_out=None, v_out=None, stream=None):
    """kvqp_paged_read: tokens first .. first + count - 1 of every sequence as k, v [B,Hkv,count,128]; float16 ones are what compress takes."""
    import torch
    device, dtype = pages.k_codes.get_device(), pages.open_k.dtype
    layout = pages._bytes(cfg, device)
    shape, outs = (cfg.batch, cfg.n_kv_heads, max(count, 0), 128), []
    for name, t in (("k_out", k_out), ("v_out", v_out)):
        if t is None:
            t = _empty_rows(shape, dtype, pages.k_codes.device, stream)
        else:
            _want(name, t, dtype, shape, device)
        outs.append(t)
    _call("kvqp_paged_read", device, stream, (cfg._bytes(), layout, first, count, outs[0].data_ptr(), outs[1].data_ptr()))
    return tuple(outs)
