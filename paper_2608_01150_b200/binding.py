"""ctypes binding of libzellige.so -- same names as the C ABI in include/zellige.h.

Argument marshalling only.  Tensors are torch CUDA tensors (device memory and streams come
from PyTorch); the functions pass their data pointers and the current stream to the
library.  Raw-pointer entry points (``*_ptr``) take integers so that callers holding host
buffers can drive the same C calls.
"""
from __future__ import annotations

import ctypes
import os
from typing import List, Optional, Sequence, Tuple

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libzellige.so")

STATUS_NAMES = {0: "ZL_OK", 1: "ZL_ERR_INVALID_ARG", 2: "ZL_ERR_OVERLAP", 3: "ZL_ERR_UNSUPPORTED",
                4: "ZL_ERR_WORKSPACE", 5: "ZL_ERR_CUDA", 6: "ZL_ERR_TIMEOUT"}


KERNEL_NAMES = ("fwd", "merge", "bwd_pre", "bwd_main", "bwd_post")


class ZlError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {STATUS_NAMES.get(status, status)}")


class ShardDesc(ctypes.Structure):
    _fields_ = [("q_off", ctypes.c_int32), ("q_len", ctypes.c_int32), ("kv_off", ctypes.c_int32),
                ("kv_len", ctypes.c_int32), ("seq_id", ctypes.c_int32)]


class WholeDesc(ctypes.Structure):
    _fields_ = [("off", ctypes.c_int32), ("len", ctypes.c_int32), ("head_begin", ctypes.c_int32),
                ("head_count", ctypes.c_int32)]


class HeadRange(ctypes.Structure):
    _fields_ = [("head_begin", ctypes.c_int32), ("head_count", ctypes.c_int32)]


class ShardPos(ctypes.Structure):
    _fields_ = [("q_pos", ctypes.c_int32), ("kv_pos", ctypes.c_int32), ("prefix", ctypes.c_int32)]


class ScoreDesc(ctypes.Structure):
    _fields_ = [("cap", ctypes.c_float), ("slopes", ctypes.c_void_p), ("bucket_bias", ctypes.c_void_p),
                ("bucket_of", ctypes.c_void_p), ("n_buckets", ctypes.c_int32), ("max_distance", ctypes.c_int32),
                ("masked", ctypes.c_int32)]


class KvCacheDesc(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("page_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("scale_page_stride", ctypes.c_int64), ("scale_token_stride", ctypes.c_int64), ("scale_head_stride", ctypes.c_int64),
                ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("format", ctypes.c_int32)]


class CacheBatchDesc(ctypes.Structure):
    _fields_ = [("cu_q", ctypes.c_void_p), ("kv_len", ctypes.c_void_p), ("pages", ctypes.c_void_p), ("prefix", ctypes.c_void_p),
                ("n_seqs", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("total_q", ctypes.c_int32), ("max_q", ctypes.c_int32)]


class TasksInfo(ctypes.Structure):
    _fields_ = [("n_tasks", ctypes.c_int32), ("n_merge_groups", ctypes.c_int32),
                ("n_kv_groups", ctypes.c_int32), ("n_fwd_items", ctypes.c_int32),
                ("n_bwd_items", ctypes.c_int32), ("partial_rows", ctypes.c_int64),
                ("o_partial_bytes", ctypes.c_size_t), ("lse_partial_bytes", ctypes.c_size_t),
                ("bwd_workspace_bytes", ctypes.c_size_t), ("n_fused_ranges", ctypes.c_int32)]


def library_path() -> str:
    return _LIB_PATH


def _load():
    if not os.path.exists(_LIB_PATH):
        raise ImportError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_2608_01150_b200.build` "
            "(nvcc, sm_100a). There is no fallback path.")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, i32, i64p = ctypes.c_void_p, ctypes.c_int32, ctypes.POINTER(ctypes.c_int64)
    lib.zl_build_tasks.restype = ctypes.c_int
    lib.zl_build_tasks.argtypes = [vp, i32, vp, i32, i32, i32, i32, i32, vp, ctypes.POINTER(vp)]
    lib.zl_build_tasks_ex.restype = ctypes.c_int
    lib.zl_build_tasks_ex.argtypes = [vp, i32, vp, i32, i32, i32, i32, i32, ctypes.c_uint32, vp, ctypes.POINTER(vp)]
    lib.zl_build_tasks_heads.restype = ctypes.c_int
    lib.zl_build_tasks_heads.argtypes = [vp, i32, vp, vp, i32, i32, i32, i32, i32, ctypes.c_uint32, vp, ctypes.POINTER(vp)]
    lib.zl_build_tasks_prefix.restype = ctypes.c_int
    lib.zl_build_tasks_prefix.argtypes = [vp, vp, i32, i32, i32, i32, i32, i32, vp, ctypes.POINTER(vp)]
    lib.zl_tasks_get_info.restype = ctypes.c_int
    lib.zl_tasks_get_info.argtypes = [vp, ctypes.POINTER(TasksInfo)]
    lib.zl_tasks_get_partial_slot.restype = ctypes.c_int
    lib.zl_tasks_get_partial_slot.argtypes = [vp, i32, i64p, i64p]
    for name in ("zl_tasks_get_fwd_items", "zl_tasks_get_bwd_items"):
        getattr(lib, name).restype = ctypes.c_int
        getattr(lib, name).argtypes = [vp, vp, i32, ctypes.POINTER(i32)]
    lib.zl_free_tasks.restype = None
    lib.zl_free_tasks.argtypes = [vp]
    lib.zl_coalesced_attn_fwd.restype = ctypes.c_int
    lib.zl_coalesced_attn_fwd.argtypes = [vp, vp, vp, vp, ctypes.c_float, vp, vp, vp, vp, vp]
    lib.zl_coalesced_attn_fwd_packed.restype = ctypes.c_int
    lib.zl_coalesced_attn_fwd_packed.argtypes = [vp, vp, ctypes.c_float, vp, vp, vp, vp, vp]
    lib.zl_coalesced_attn_bwd_packed.restype = ctypes.c_int
    lib.zl_coalesced_attn_bwd_packed.argtypes = [vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, ctypes.c_size_t, vp]
    lib.zl_lse_merge.restype = ctypes.c_int
    lib.zl_lse_merge.argtypes = [vp, vp, vp, vp, vp, vp]
    lib.zl_coalesced_attn_bwd.restype = ctypes.c_int
    lib.zl_coalesced_attn_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, vp, vp,
                                          ctypes.c_size_t, vp]
    for name in ("zl_set_fwd_phases", "zl_set_bwd_phases"):
        getattr(lib, name).restype = ctypes.c_int
        getattr(lib, name).argtypes = [vp, vp, vp, i32, vp]
    lib.zl_coalesced_attn_fwd_phase.restype = ctypes.c_int
    lib.zl_coalesced_attn_fwd_phase.argtypes = [vp, i32, vp, vp, vp, ctypes.c_float, vp, vp, vp, vp, vp]
    lib.zl_coalesced_attn_bwd_phase.restype = ctypes.c_int
    lib.zl_coalesced_attn_bwd_phase.argtypes = [vp, i32, vp, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, vp, vp,
                                                ctypes.c_size_t, vp]
    lib.zl_phase_info.restype = ctypes.c_int
    lib.zl_phase_info.argtypes = [vp, ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(i32)]
    lib.zl_set_sm_margin.restype = ctypes.c_int
    lib.zl_set_sm_margin.argtypes = [vp, i32]
    lib.zl_coalesced_attn_bwd_noalloc.restype = ctypes.c_int
    lib.zl_coalesced_attn_bwd_noalloc.argtypes = [vp, vp, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, vp, vp]
    sd = ctypes.POINTER(ScoreDesc)
    lib.zl_set_positions.restype = ctypes.c_int
    lib.zl_set_positions.argtypes = [vp, vp, vp, vp]
    lib.zl_scored_attn_fwd.restype = ctypes.c_int
    lib.zl_scored_attn_fwd.argtypes = [vp, sd, vp, vp, vp, ctypes.c_float, vp, vp, vp, vp, vp]
    lib.zl_scored_attn_fwd_packed.restype = ctypes.c_int
    lib.zl_scored_attn_fwd_packed.argtypes = [vp, sd, vp, ctypes.c_float, vp, vp, vp, vp, vp]
    lib.zl_scored_attn_bwd.restype = ctypes.c_int
    lib.zl_scored_attn_bwd.argtypes = [vp, sd, vp, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, vp, vp, vp,
                                       ctypes.c_size_t, vp]
    lib.zl_scored_attn_bwd_packed.restype = ctypes.c_int
    lib.zl_scored_attn_bwd_packed.argtypes = [vp, sd, vp, vp, vp, vp, ctypes.c_float, vp, vp, vp, ctypes.c_size_t, vp]
    lib.zl_scored_workspace_bytes.restype = ctypes.c_int
    lib.zl_scored_workspace_bytes.argtypes = [vp, sd, ctypes.POINTER(ctypes.c_size_t)]
    cd, bd = ctypes.POINTER(KvCacheDesc), ctypes.POINTER(CacheBatchDesc)
    lib.zl_cache_write.restype = ctypes.c_int
    lib.zl_cache_write.argtypes = [cd, bd, vp, vp, ctypes.c_int64, vp]
    lib.zl_cache_read.restype = ctypes.c_int
    lib.zl_cache_read.argtypes = [cd, bd, vp, vp, i32, vp, vp, vp]
    lib.zl_build_cached_attn.restype = ctypes.c_int
    lib.zl_build_cached_attn.argtypes = [i32, i32, i32, vp, ctypes.POINTER(vp)]
    lib.zl_free_cached_attn.restype = None
    lib.zl_free_cached_attn.argtypes = [vp]
    lib.zl_cached_attn_workspace_bytes.restype = ctypes.c_int
    lib.zl_cached_attn_workspace_bytes.argtypes = [vp, ctypes.POINTER(ctypes.c_size_t)]
    lib.zl_cached_attn_device_status.restype = ctypes.c_int
    lib.zl_cached_attn_device_status.argtypes = [vp, ctypes.POINTER(i32), ctypes.POINTER(i32)]
    lib.zl_cached_attn_fwd.restype = ctypes.c_int
    lib.zl_cached_attn_fwd.argtypes = [vp, cd, bd, vp, ctypes.c_int64, ctypes.c_float, vp, vp, vp, ctypes.c_size_t, vp]
    lib.zl_last_device_status.restype = ctypes.c_int
    lib.zl_last_device_status.argtypes = [vp, ctypes.POINTER(i32), ctypes.POINTER(i32)]
    lib.zl_set_kernel_timing.restype = ctypes.c_int
    lib.zl_set_kernel_timing.argtypes = [vp, i32]
    lib.zl_get_kernel_timing.restype = ctypes.c_int
    lib.zl_get_kernel_timing.argtypes = [vp, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(i32)]
    lib.zl_debug_set_fwd_order.restype = ctypes.c_int
    lib.zl_debug_set_fwd_order.argtypes = [vp, i32, vp]
    lib.zl_set_bwd_kernel.restype = ctypes.c_int
    lib.zl_set_bwd_kernel.argtypes = [vp, i32]
    lib.zl_selftest_bounded_wait.restype = ctypes.c_int
    lib.zl_selftest_bounded_wait.argtypes = [vp, i32, vp]
    lib.zl_status_str.restype = ctypes.c_char_p
    lib.zl_status_str.argtypes = [ctypes.c_int]
    lib.zl_launch_count.restype = ctypes.c_int64
    lib.zl_launch_count.argtypes = []
    return lib


_lib = _load()


def lib():
    return _lib


def _check(status: int, what: str):
    if status != 0:
        raise ZlError(status, what)


def _stream_ptr(stream=None) -> int:
    if stream is None:
        import torch
        if torch.cuda.is_initialized():
            # the current stream's handle without building a Stream object, which costs more than some of the launches
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        if not torch.cuda.is_available():
            return 0
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream) if hasattr(stream, "cuda_stream") else int(stream)


def _current_device() -> int:
    import torch
    return torch._C._cuda_getDevice()


def _ptr(t) -> Optional[int]:
    if t is None or isinstance(t, int):
        return t
    return t.data_ptr()


def _int32s(values) -> List[int]:
    """The values as ints that fit the ABI's int32; ctypes would keep the low 32 bits of others without a word."""
    out = [int(v) for v in values]
    if out and (min(out) < -2 ** 31 or max(out) >= 2 ** 31):
        raise ZlError(1, f"{max(out, key=abs)} does not fit 32 bits")
    return out


class TaskHandle:
    """Owns a ``zl_tasks*``.  Built once per placement, reused for every layer and step."""

    def __init__(self, ptr: int, n_heads: int, head_dim: int, total_q: int, total_kv: int, n_shards: int,
                 n_whole: int = 0):
        self._ptr = ctypes.c_void_p(ptr)
        self.n_heads, self.head_dim, self.total_q, self.total_kv = n_heads, head_dim, total_q, total_kv
        self.n_shards, self.n_whole = n_shards, n_whole
        info = TasksInfo()
        _check(_lib.zl_tasks_get_info(self._ptr, ctypes.byref(info)), "zl_tasks_get_info")
        self.info = info

    @property
    def ptr(self):
        return self._ptr

    def partial_slot(self, shard_idx: int) -> Tuple[int, int]:
        a, b = ctypes.c_int64(), ctypes.c_int64()
        _check(_lib.zl_tasks_get_partial_slot(self._ptr, shard_idx, ctypes.byref(a), ctypes.byref(b)),
               "zl_tasks_get_partial_slot")
        return a.value, b.value

    def _items(self, fn) -> List[Tuple[int, int, int, int]]:
        n = ctypes.c_int32()
        _check(fn(self._ptr, None, 0, ctypes.byref(n)), "items count")
        buf = (ctypes.c_int32 * (4 * max(1, n.value)))()
        _check(fn(self._ptr, buf, n.value, ctypes.byref(n)), "items")
        return [tuple(buf[4 * i:4 * i + 4]) for i in range(n.value)]

    def fwd_items(self):
        return self._items(_lib.zl_tasks_get_fwd_items)

    def bwd_items(self):
        return self._items(_lib.zl_tasks_get_bwd_items)

    def last_device_status(self) -> Tuple[int, int]:
        c, w = ctypes.c_int32(), ctypes.c_int32()
        _check(_lib.zl_last_device_status(self._ptr, ctypes.byref(c), ctypes.byref(w)), "zl_last_device_status")
        return c.value, w.value

    def set_kernel_timing(self, enable: bool):
        _check(_lib.zl_set_kernel_timing(self._ptr, 1 if enable else 0), "zl_set_kernel_timing")

    def get_kernel_timing(self):
        """{kernel name: (total ms, launches)} since the last read; synchronises the device."""
        ms = (ctypes.c_float * len(KERNEL_NAMES))()
        n = (ctypes.c_int32 * len(KERNEL_NAMES))()
        _check(_lib.zl_get_kernel_timing(self._ptr, ms, n), "zl_get_kernel_timing")
        return {name: (float(ms[i]), int(n[i])) for i, name in enumerate(KERNEL_NAMES)}

    def set_fwd_order(self, mode: int, stream=None):
        """0 longest-first (default), 1 placement order, 2 shortest-first (measurement aid)."""
        _check(_lib.zl_debug_set_fwd_order(self._ptr, mode, _stream_ptr(stream)), "zl_debug_set_fwd_order")

    @staticmethod
    def _phase_array(values):
        if values is None:
            return None, None
        arr = (ctypes.c_int32 * max(1, len(values)))(*_int32s(values))
        return arr, ctypes.cast(arr, ctypes.c_void_p)

    def set_fwd_phases(self, whole_phase, shard_phase, n_phases: int, stream=None):
        """zl_set_fwd_phases: one phase number per whole sequence / per shard (None = all zero)."""
        a, ap = self._phase_array(whole_phase)
        b, bp = self._phase_array(shard_phase)
        _check(_lib.zl_set_fwd_phases(self._ptr, ap, bp, n_phases, _stream_ptr(stream)), "zl_set_fwd_phases")

    def set_bwd_phases(self, whole_phase, shard_phase, n_phases: int, stream=None):
        """zl_set_bwd_phases."""
        a, ap = self._phase_array(whole_phase)
        b, bp = self._phase_array(shard_phase)
        _check(_lib.zl_set_bwd_phases(self._ptr, ap, bp, n_phases, _stream_ptr(stream)), "zl_set_bwd_phases")

    def set_positions(self, whole_prefix=None, shard_pos=None, stream=None):
        """zl_set_positions: visible prefix per whole sequence (None = 0), (q_pos, kv_pos, prefix) per shard."""
        if whole_prefix is not None and len(whole_prefix) != self.n_whole:
            raise ZlError(1, f"set_positions: {self.n_whole} whole sequences, {len(whole_prefix)} prefixes")
        if shard_pos is not None and len(shard_pos) != self.n_shards:
            raise ZlError(1, f"set_positions: {self.n_shards} shards, {len(shard_pos)} positions")
        a, ap = self._phase_array(whole_prefix)
        b = (ShardPos * max(1, self.n_shards))(*[ShardPos(*_int32s(s)) for s in shard_pos or ()])
        bp = ctypes.cast(b, ctypes.c_void_p) if shard_pos is not None else None
        _check(_lib.zl_set_positions(self._ptr, ap, bp, _stream_ptr(stream)), "zl_set_positions")

    def scored_workspace_bytes(self, score: "Score") -> int:
        """zl_scored_workspace_bytes: workspace of scored_attn_bwd with this score."""
        n = ctypes.c_size_t()
        _check(_lib.zl_scored_workspace_bytes(self._ptr, ctypes.byref(score.desc), ctypes.byref(n)),
               "zl_scored_workspace_bytes")
        return int(n.value)

    def phase_info(self):
        """zl_phase_info: (forward items per phase, backward items per phase)."""
        nf, nb = ctypes.c_int32(0), ctypes.c_int32(0)
        fi, bi = (ctypes.c_int32 * MAX_PHASES)(), (ctypes.c_int32 * MAX_PHASES)()
        _check(_lib.zl_phase_info(self._ptr, ctypes.byref(nf), ctypes.byref(nb), fi, bi), "zl_phase_info")
        return list(fi[:nf.value]), list(bi[:nb.value])

    def set_sm_margin(self, n_sms: int):
        """zl_set_sm_margin: SMs the persistent kernels leave free for kernels of other streams."""
        _check(_lib.zl_set_sm_margin(self._ptr, n_sms), "zl_set_sm_margin")

    def set_bwd_kernel(self, kernel: int):
        """0 library default, 1 one CTA per key tile, 2 CTA pairs (head_dim 128)."""
        _check(_lib.zl_set_bwd_kernel(self._ptr, kernel), "zl_set_bwd_kernel")

    def selftest_bounded_wait(self, limit_us: int = 1000, stream=None):
        """Launches a kernel whose bounded wait must expire; read the outcome with last_device_status()."""
        _check(_lib.zl_selftest_bounded_wait(self._ptr, limit_us, _stream_ptr(stream)), "zl_selftest_bounded_wait")

    def close(self):
        if self._ptr:
            _lib.zl_free_tasks(self._ptr)
            self._ptr = ctypes.c_void_p(0)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


BUILD_FUSE_LOCAL_CHUNKS = 1
MAX_PHASES = 64  # ZL_MAX_PHASES


def build_tasks(cu_seqlens: Sequence[int], shards: Sequence[Sequence[int]], total_q: int, total_kv: int,
                n_heads: int, head_dim: int, stream=None, flags: int = 0) -> TaskHandle:
    """zl_build_tasks / zl_build_tasks_ex: placement (cu_seqlens + shard descriptors) -> task handle.
    flags: 0 or BUILD_FUSE_LOCAL_CHUNKS."""
    n_whole = max(0, len(cu_seqlens) - 1)
    total_q, total_kv, n_heads, head_dim = _int32s((total_q, total_kv, n_heads, head_dim))
    cu = (ctypes.c_int32 * max(1, len(cu_seqlens)))(*_int32s(cu_seqlens))
    sh = (ShardDesc * max(1, len(shards)))(*[ShardDesc(*_int32s(s)) for s in shards])
    out = ctypes.c_void_p()
    cu_p = ctypes.cast(cu, ctypes.c_void_p) if len(cu_seqlens) else None
    sh_p = ctypes.cast(sh, ctypes.c_void_p) if len(shards) else None
    if flags:
        st = _lib.zl_build_tasks_ex(cu_p, n_whole, sh_p, len(shards), total_q, total_kv, n_heads, head_dim,
                                    ctypes.c_uint32(flags), _stream_ptr(stream), ctypes.byref(out))
    else:
        st = _lib.zl_build_tasks(cu_p, n_whole, sh_p, len(shards), total_q, total_kv, n_heads, head_dim,
                                 _stream_ptr(stream), ctypes.byref(out))
    _check(st, "zl_build_tasks")
    return TaskHandle(out.value, n_heads, head_dim, total_q, total_kv, len(shards), n_whole)


def build_tasks_heads(whole: Sequence[Sequence[int]], shards: Sequence[Sequence[int]],
                      shard_heads: Optional[Sequence[Sequence[int]]], total_q: int, total_kv: int,
                      n_heads: int, head_dim: int, stream=None, flags: int = 0) -> TaskHandle:
    """zl_build_tasks_heads: whole = (off, len, head_begin, head_count) per whole sequence, shards =
    (q_off, q_len, kv_off, kv_len, seq_id) per shard, shard_heads = (head_begin, head_count) per shard or
    None for all heads."""
    total_q, total_kv, n_heads, head_dim = _int32s((total_q, total_kv, n_heads, head_dim))
    wd = (WholeDesc * max(1, len(whole)))(*[WholeDesc(*_int32s(w)) for w in whole])
    sh = (ShardDesc * max(1, len(shards)))(*[ShardDesc(*_int32s(s[:5])) for s in shards])
    hr = None
    if shard_heads is not None:
        assert len(shard_heads) == len(shards)
        hr = (HeadRange * max(1, len(shards)))(*[HeadRange(*_int32s((a, b))) for a, b in shard_heads])
    out = ctypes.c_void_p()
    st = _lib.zl_build_tasks_heads(ctypes.cast(wd, ctypes.c_void_p) if len(whole) else None, len(whole),
                                   ctypes.cast(sh, ctypes.c_void_p) if len(shards) else None,
                                   ctypes.cast(hr, ctypes.c_void_p) if hr is not None and len(shards) else None,
                                   len(shards), total_q, total_kv, n_heads, head_dim, ctypes.c_uint32(flags),
                                   _stream_ptr(stream), ctypes.byref(out))
    _check(st, "zl_build_tasks_heads")
    return TaskHandle(out.value, n_heads, head_dim, total_q, total_kv, len(shards), len(whole))


def build_tasks_prefix(cu_q: Sequence[int], cu_kv: Sequence[int], prefix_len: int, total_q: int, total_kv: int,
                       n_heads: int, head_dim: int, stream=None) -> TaskHandle:
    """zl_build_tasks_prefix: sequence i owns query rows [cu_q[i], cu_q[i+1]) and, behind the shared prefix rows
    [0, prefix_len), key rows prefix_len + [cu_kv[i], cu_kv[i+1])."""
    n = max(0, len(cu_q) - 1)
    if max(0, len(cu_kv) - 1) != n:
        raise ZlError(1, f"build_tasks_prefix: {n} query ranges, {max(0, len(cu_kv) - 1)} key ranges")
    prefix_len, total_q, total_kv, n_heads, head_dim = _int32s((prefix_len, total_q, total_kv, n_heads, head_dim))
    a = (ctypes.c_int32 * max(1, len(cu_q)))(*_int32s(cu_q))
    b = (ctypes.c_int32 * max(1, len(cu_kv)))(*_int32s(cu_kv))
    out = ctypes.c_void_p()
    _check(_lib.zl_build_tasks_prefix(ctypes.cast(a, ctypes.c_void_p), ctypes.cast(b, ctypes.c_void_p), n, prefix_len,
                                      total_q, total_kv, n_heads, head_dim, _stream_ptr(stream), ctypes.byref(out)),
           "zl_build_tasks_prefix")
    return TaskHandle(out.value, n_heads, head_dim, total_q, total_kv, n)


def coalesced_attn_fwd(tasks: TaskHandle, q, k, v, scale: float, o, lse, o_partial=None, lse_partial=None,
                       stream=None):
    """zl_coalesced_attn_fwd.  Tensors: torch CUDA tensors or raw device pointers (int)."""
    _check(_lib.zl_coalesced_attn_fwd(tasks.ptr, _ptr(q), _ptr(k), _ptr(v), ctypes.c_float(scale), _ptr(o),
                                      _ptr(lse), _ptr(o_partial), _ptr(lse_partial), _stream_ptr(stream)),
           "zl_coalesced_attn_fwd")


def coalesced_attn_fwd_phase(tasks: TaskHandle, phase: int, q, k, v, scale: float, o, lse, o_partial=None,
                             lse_partial=None, stream=None):
    """zl_coalesced_attn_fwd_phase: the tasks of one launch phase."""
    _check(_lib.zl_coalesced_attn_fwd_phase(tasks.ptr, phase, _ptr(q), _ptr(k), _ptr(v), ctypes.c_float(scale), _ptr(o),
                                            _ptr(lse), _ptr(o_partial), _ptr(lse_partial), _stream_ptr(stream)),
           "zl_coalesced_attn_fwd_phase")


def coalesced_attn_bwd_phase(tasks: TaskHandle, phase: int, q, k, v, o, lse, d_o, scale: float, dq, dk, dv, workspace,
                             workspace_bytes: Optional[int] = None, stream=None):
    """zl_coalesced_attn_bwd_phase: phases 0 .. n-1 in order, same arguments."""
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size()
    _check(_lib.zl_coalesced_attn_bwd_phase(tasks.ptr, phase, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(d_o),
                                            ctypes.c_float(scale), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(workspace),
                                            ctypes.c_size_t(workspace_bytes), _stream_ptr(stream)),
           "zl_coalesced_attn_bwd_phase")


def lse_merge(tasks: TaskHandle, o_partial, lse_partial, o, lse, stream=None):
    """zl_lse_merge."""
    _check(_lib.zl_lse_merge(tasks.ptr, _ptr(o_partial), _ptr(lse_partial), _ptr(o), _ptr(lse),
                             _stream_ptr(stream)), "zl_lse_merge")


def coalesced_attn_bwd(tasks: TaskHandle, q, k, v, o, lse, d_o, scale: float, dq, dk, dv, workspace,
                       workspace_bytes: Optional[int] = None, stream=None):
    """zl_coalesced_attn_bwd."""
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size()
    _check(_lib.zl_coalesced_attn_bwd(tasks.ptr, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(d_o),
                                      ctypes.c_float(scale), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(workspace),
                                      ctypes.c_size_t(workspace_bytes), _stream_ptr(stream)),
           "zl_coalesced_attn_bwd")


def coalesced_attn_fwd_packed(tasks: TaskHandle, qkv, scale: float, o, lse, o_partial=None, lse_partial=None,
                              stream=None):
    """zl_coalesced_attn_fwd_packed: qkv is [T, 3, H, d] bf16 (total_q == total_kv == T)."""
    _check(_lib.zl_coalesced_attn_fwd_packed(tasks.ptr, _ptr(qkv), ctypes.c_float(scale), _ptr(o), _ptr(lse),
                                             _ptr(o_partial), _ptr(lse_partial), _stream_ptr(stream)),
           "zl_coalesced_attn_fwd_packed")


def coalesced_attn_bwd_packed(tasks: TaskHandle, qkv, o, lse, d_o, scale: float, dqkv, workspace,
                              workspace_bytes: Optional[int] = None, stream=None):
    """zl_coalesced_attn_bwd_packed: reads qkv [T, 3, H, d], writes dqkv [T, 3, H, d]."""
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size()
    _check(_lib.zl_coalesced_attn_bwd_packed(tasks.ptr, _ptr(qkv), _ptr(o), _ptr(lse), _ptr(d_o),
                                             ctypes.c_float(scale), _ptr(dqkv), _ptr(workspace),
                                             ctypes.c_size_t(workspace_bytes), _stream_ptr(stream)),
           "zl_coalesced_attn_bwd_packed")


MAX_BUCKETS = 64  # ZL_MAX_BUCKETS


class Score:
    """zl_score: scores beyond ``scale * q.k``.

    cap          0 = none, else scores become ``cap * tanh(scale * q.k / cap)``
    slopes       fp32 [n_heads]: ``- slope * |distance|``, of magnitude at most 1e18
    bucket_bias  fp32 [n_buckets, n_heads]: learned bias, with
    bucket_of    int32 [2 * max_distance + 1]: the bucket of every distance key - query from -max_distance on
                 (see :func:`relative_position_buckets`)
    masked       prefix mask of ``TaskHandle.set_positions``

    The attributes can be changed, and their storage swapped (``module.to``): every call takes what they hold then.  Their
    values are read when a kernel runs, so a captured call keeps the storage of its capture.
    """

    def __init__(self, cap: float = 0.0, slopes=None, bucket_bias=None, bucket_of=None, masked: bool = False):
        self.cap, self.slopes, self.bucket_bias, self.bucket_of, self.masked = cap, slopes, bucket_bias, bucket_of, masked
        self._fields = self._desc = None
        self.desc

    @property
    def desc(self) -> ScoreDesc:
        """The C struct of what the attributes hold now (not to be written to); raises where they do not fit."""
        return self._read(None)

    def check(self, tasks: TaskHandle) -> ScoreDesc:
        """The same for a call on `tasks`: the tensors are of its heads and on the current GPU."""
        return self._read(tasks.n_heads)

    def _read(self, heads: Optional[int]) -> ScoreDesc:
        import torch
        slopes, bias, of = self.slopes, self.bucket_bias, self.bucket_of
        p_slopes = p_bias = p_of = None
        buckets = reach = 0
        if slopes is not None:
            shape = slopes.shape
            if slopes.dtype is not torch.float32 or len(shape) != 1 or not slopes.is_contiguous():
                raise ZlError(1, "Score: slopes must be a contiguous torch.float32 tensor of 1 dimension")
            if heads is not None:
                device = _current_device() if slopes.is_cuda else None
                self._fits("slopes", slopes, shape[0], heads, device)
            p_slopes = slopes.data_ptr()
        if bias is not None or of is not None:
            if bias is None or of is None:
                raise ZlError(1, "Score: bucket_bias and bucket_of come together")
            shape, entries = bias.shape, of.shape
            if bias.dtype is not torch.float32 or len(shape) != 2 or not bias.is_contiguous():
                raise ZlError(1, "Score: bucket_bias must be a contiguous torch.float32 tensor of 2 dimensions")
            if of.dtype is not torch.int32 or len(entries) != 1 or not of.is_contiguous():
                raise ZlError(1, "Score: bucket_of must be a contiguous torch.int32 tensor of 1 dimension")
            if entries[0] % 2 == 0:
                raise ZlError(1, "Score: bucket_of has an entry for every distance from -max_distance to max_distance")
            if heads is not None:
                device = _current_device() if bias.is_cuda else None
                self._fits("bucket_bias", bias, shape[1], heads, device)
                self._fits("bucket_of", of, heads, heads, device)
            p_bias, p_of, buckets, reach = bias.data_ptr(), of.data_ptr(), shape[0], entries[0] // 2
        fields = (self.cap, p_slopes, p_bias, p_of, buckets, reach, 1 if self.masked else 0)
        desc = self._desc
        if fields != self._fields:
            # a struct of its own per state: a call of another thread may be reading the one before
            self._desc = desc = ScoreDesc(*fields)
            self._fields = fields
        return desc

    @staticmethod
    def _fits(name: str, t, n: int, heads: int, device: Optional[int]):
        if n != heads:
            raise ZlError(1, f"Score: {name} has {n} heads, the handle {heads}")
        if not t.is_cuda or t.get_device() != device:
            raise ZlError(1, f"Score: {name} is not on the current GPU")


def relative_position_buckets(n_buckets: int, max_distance: int, bidirectional: bool = True) -> List[int]:
    """Bucket of every distance key - query from -max_distance to max_distance, for ``Score(bucket_of=...)``.

    Half of a side's buckets hold one distance each, the rest grow by a constant factor until max_distance, from which on
    the last bucket holds everything: with m buckets of a side, e = m // 2 exact ones and a = |distance| >= e,
    bucket = e + floor((m - e) * ln(a / e) / ln(max_distance / e)), at most m - 1.  Bidirectional: keys after the
    query use the second half of the buckets; otherwise they share bucket 0 with distance 0 (a mask hides them).
    The borders are compared as whole numbers, so a distance that lies on one is never rounded to the wrong side."""
    side = n_buckets // 2 if bidirectional else n_buckets
    exact = side // 2
    if exact < 1 or max_distance <= exact:
        raise ZlError(1, "relative_position_buckets: needs max_distance beyond the exact buckets, at least "
                         f"{4 if bidirectional else 2} buckets")

    def of(a: int) -> int:
        if a < exact:
            return a
        steps = side - exact
        k = 0  # largest k with exact * (max_distance / exact)^(k / steps) <= a
        while k < steps - 1 and max_distance ** (k + 1) * exact ** (steps - k - 1) <= a ** steps:
            k += 1
        return exact + k

    out = []
    for d in range(-max_distance, max_distance + 1):
        if bidirectional:
            out.append(of(abs(d)) + (side if d > 0 else 0))
        else:
            out.append(of(max(0, -d)))
    return out


def scored_attn_fwd(tasks: TaskHandle, score: Score, q, k, v, scale: float, o, lse, o_partial=None, lse_partial=None,
                    stream=None):
    """zl_scored_attn_fwd: coalesced_attn_fwd with capped, biased or masked scores."""
    desc = score.check(tasks)
    _check(_lib.zl_scored_attn_fwd(tasks.ptr, ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), scale,
                                   _ptr(o), _ptr(lse), _ptr(o_partial), _ptr(lse_partial), _stream_ptr(stream)),
           "zl_scored_attn_fwd")


def scored_attn_fwd_packed(tasks: TaskHandle, score: Score, qkv, scale: float, o, lse, o_partial=None, lse_partial=None,
                           stream=None):
    """zl_scored_attn_fwd_packed: qkv is [T, 3, H, d] bf16."""
    desc = score.check(tasks)
    _check(_lib.zl_scored_attn_fwd_packed(tasks.ptr, ctypes.byref(desc), _ptr(qkv), scale, _ptr(o),
                                          _ptr(lse), _ptr(o_partial), _ptr(lse_partial), _stream_ptr(stream)),
           "zl_scored_attn_fwd_packed")


def _check_table(score: Score, d_bucket_bias):
    t = score.bucket_bias
    if d_bucket_bias is not None and t is not None and not isinstance(d_bucket_bias, int):
        if d_bucket_bias.shape != t.shape or d_bucket_bias.dtype != t.dtype or not d_bucket_bias.is_contiguous():
            raise ZlError(1, "d_bucket_bias must be contiguous and of bucket_bias' shape and type")
        if not d_bucket_bias.is_cuda or d_bucket_bias.get_device() != _current_device():
            raise ZlError(1, "d_bucket_bias is not on the current GPU")


def scored_attn_bwd(tasks: TaskHandle, score: Score, q, k, v, o, lse, d_o, scale: float, dq, dk, dv, d_bucket_bias,
                    workspace, workspace_bytes: Optional[int] = None, stream=None):
    """zl_scored_attn_bwd.  d_bucket_bias: fp32 [n_buckets, n_heads] or None."""
    desc = score.check(tasks)
    _check_table(score, d_bucket_bias)
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size()
    _check(_lib.zl_scored_attn_bwd(tasks.ptr, ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse),
                                   _ptr(d_o), scale, _ptr(dq), _ptr(dk), _ptr(dv), _ptr(d_bucket_bias),
                                   _ptr(workspace), ctypes.c_size_t(workspace_bytes), _stream_ptr(stream)),
           "zl_scored_attn_bwd")


def scored_attn_bwd_packed(tasks: TaskHandle, score: Score, qkv, o, lse, d_o, scale: float, dqkv, d_bucket_bias,
                           workspace, workspace_bytes: Optional[int] = None, stream=None):
    """zl_scored_attn_bwd_packed: reads qkv [T, 3, H, d], writes dqkv [T, 3, H, d]."""
    desc = score.check(tasks)
    _check_table(score, d_bucket_bias)
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size()
    _check(_lib.zl_scored_attn_bwd_packed(tasks.ptr, ctypes.byref(desc), _ptr(qkv), _ptr(o), _ptr(lse), _ptr(d_o),
                                          scale, _ptr(dqkv), _ptr(d_bucket_bias), _ptr(workspace),
                                          ctypes.c_size_t(workspace_bytes), _stream_ptr(stream)),
           "zl_scored_attn_bwd_packed")


def _on_gpu(what: str, t, device: int):
    """The tensor is on the current GPU (`device`), where the call's kernels run."""
    if t.get_device() != device:  # (-1 of a tensor that is on none)
        raise ZlError(1, f"{what} is not on the current GPU")


def _call_stream(stream, device: int) -> int:
    """_stream_ptr of a call whose tensors are on the current GPU (`device`): CUDA is up, which need not be asked."""
    if stream is None:
        import torch
        return torch._C._cuda_getCurrentRawStream(device)
    return _stream_ptr(stream)


def _ints(what: str, t, shape=None):
    import torch
    if t.dtype is not torch.int32 or not t.is_contiguous() or (shape is not None and t.shape != shape):
        raise ZlError(1, f"{what} must be a contiguous torch.int32 tensor" + (f" of shape {shape}" if shape is not None else ""))


class KvCache:
    """zl_kv_cache: the keys and values of one layer in pages.

    k, v              [n_pages, page_size, n_kv_heads, head_dim] of torch.bfloat16, torch.int8 or torch.float8_e4m3fn; any
                      strides (the same for both) with contiguous rows, e.g. ``pool[:, 0]``, ``pool[:, 1]`` or a transposed
                      [n_pages, n_kv_heads, page_size, head_dim]
    k_scale, v_scale  fp32 [n_pages, page_size, n_kv_heads] of an 8-bit cache, written by cache_write; else None.  Any strides
                      (the same for both); a transposed [n_pages, n_kv_heads, page_size] is read faster

    The attributes can be changed, and their storage swapped: every call takes what they hold then.
    """

    def __init__(self, k, v, k_scale=None, v_scale=None):
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self._seen = (None,) * 3
        self.desc

    @property
    def desc(self) -> KvCacheDesc:
        """The C struct of what the attributes hold now (not to be written to); raises where they do not fit."""
        return self._look()[2]

    def check(self) -> Tuple[KvCacheDesc, int]:
        """The same for a call: the tensors are on the current GPU, whose number comes with it."""
        key, on_gpu, desc = self._look()
        device = key[0]
        if not on_gpu or device != _current_device():
            raise ZlError(1, "KvCache: the tensors are not on the current GPU")
        return desc, device

    def _look(self):
        # All that _read looks at (written out: calls of a function per tensor would cost as much again): as long as that is the same, so
        # is what it makes of it.  A state of its own per change: a call of another thread may be reading the one before
        k, v, ks, vs = self.k, self.v, self.k_scale, self.v_scale
        key = (k.get_device(), k.data_ptr(), k.dtype, k.shape, k.stride(), v.data_ptr(), v.dtype, v.shape, v.stride())
        if ks is not None:
            key += (ks.data_ptr(), ks.dtype, ks.shape, ks.stride())
        if vs is not None:
            key += (vs.data_ptr(), vs.dtype, vs.shape, vs.stride())
        seen = self._seen
        if seen[0] != key:
            self._seen = seen = (key, k.is_cuda, self._read(k, v, ks, vs))
        return seen

    def _read(self, k, v, ks, vs) -> KvCacheDesc:
        import torch
        fmt = {torch.bfloat16: 0, torch.int8: 1, torch.float8_e4m3fn: 2}.get(k.dtype)
        if fmt is None or v.dtype is not k.dtype:
            raise ZlError(1, "KvCache: k and v must both be torch.bfloat16, torch.int8 or torch.float8_e4m3fn")
        shape, strides = k.shape, k.stride()
        if len(shape) != 4 or v.shape != shape or v.stride() != strides or strides[3] != 1:
            raise ZlError(1, "KvCache: k and v must be [n_pages, page_size, n_kv_heads, head_dim] with the same strides and contiguous rows")
        if (ks is None) != (fmt == 0) or (vs is None) != (fmt == 0):
            raise ZlError(1, "KvCache: an 8-bit cache has k_scale and v_scale, one in bf16 neither")
        for name, t in (("k_scale", ks), ("v_scale", vs)):
            if t is not None and (t.dtype is not torch.float32 or t.shape != shape[:3] or t.stride() != ks.stride()):
                raise ZlError(1, f"KvCache: {name} must be torch.float32 [n_pages, page_size, n_kv_heads], the strides of k_scale and v_scale the same")
        for t in (v, ks, vs):
            if t is not None and t.get_device() != k.get_device():
                raise ZlError(1, "KvCache: the tensors are on different devices")
        # (a stride of a dimension of one entry may be any number)
        page, token, head = (strides[i] if shape[i] > 1 else shape[3] for i in range(3))
        by = (0, 0, 0) if ks is None else tuple(ks.stride()[i] if shape[i] > 1 else 1 for i in range(3))
        return KvCacheDesc(k.data_ptr(), v.data_ptr(), _ptr(ks), _ptr(vs), page, token, head, *by, *_int32s(shape), fmt)


class CacheBatch:
    """zl_cache_batch: sequences over a cache.  int32 tensors on the GPU, read when a kernel runs:

    cu_q    [n_seqs + 1]: rows [cu_q[s], cu_q[s+1]) are the new tokens of sequence s
    kv_len  [n_seqs]: tokens of the sequence, the new ones included
    pages   [n_seqs, max_pages]: the sequence's pages; a number outside the cache is a page without keys
    prefix  [n_seqs]: keys that every new token sees, or None for causal order
    max_q   the largest number of new tokens of a sequence, where it is known (it only chooses kernels)

    The attributes can be changed: every call takes what they hold then.
    """

    def __init__(self, cu_q, kv_len, pages, prefix=None, max_q: int = 0):
        self.cu_q, self.kv_len, self.pages, self.prefix, self.max_q = cu_q, kv_len, pages, prefix, max_q
        self._seen = (None,) * 3
        self._look(0)

    def check(self, total_q: Optional[int], device: int) -> CacheBatchDesc:
        """The C struct of what the attributes hold now, for a call with token tensors of total_q rows; raises where they do
        not fit or are not on the current GPU (`device`)."""
        key, on_gpu, desc = self._look(total_q)
        if not on_gpu or key[0] != device:
            raise ZlError(1, "CacheBatch: the tensors are not on the current GPU")
        return desc

    def _look(self, total_q: Optional[int]):
        # as KvCache._look; None: the call has no token tensors, whatever was there last will do
        cu, lens, pages, prefix, max_q = self.cu_q, self.kv_len, self.pages, self.prefix, self.max_q
        seen = self._seen
        if total_q is None:
            total_q = seen[2].total_q
        key = (cu.get_device(), total_q, max_q, cu.data_ptr(), cu.dtype, cu.shape, cu.is_contiguous(), lens.data_ptr(), lens.dtype, lens.shape,
               lens.is_contiguous(), pages.data_ptr(), pages.dtype, pages.shape, pages.is_contiguous())
        if prefix is not None:
            key += (prefix.data_ptr(), prefix.dtype, prefix.shape, prefix.is_contiguous())
        if seen[0] != key:
            self._seen = seen = (key, cu.is_cuda, self._read(cu, lens, pages, prefix, max_q, total_q))
        return seen

    def _read(self, cu, lens, pages, prefix, max_q, total_q: int) -> CacheBatchDesc:
        n = lens.shape[0] if lens.dim() == 1 else -1
        _ints("CacheBatch: kv_len", lens, (max(0, n),))
        _ints("CacheBatch: cu_q", cu, (n + 1,))
        if pages.dim() != 2 or pages.shape[0] != n:
            raise ZlError(1, f"CacheBatch: pages must be [{n}, max_pages]")
        _ints("CacheBatch: pages", pages)
        if prefix is not None:
            _ints("CacheBatch: prefix", prefix, (n,))
        for t in (lens, pages, prefix):
            if t is not None and t.get_device() != cu.get_device():
                raise ZlError(1, "CacheBatch: the tensors are on different devices")
        n, width, total_q, max_q = _int32s((n, pages.shape[1], total_q, max_q))
        return CacheBatchDesc(cu.data_ptr(), lens.data_ptr(), pages.data_ptr(), _ptr(prefix), n, width, total_q, max_q)


def _token_rows(what: str, t, heads: int, dim: int, device: int) -> Tuple[int, int, tuple, tuple]:
    """Rows of a bf16 tensor [tokens, heads, dim] whose rows are contiguous, and their stride; the tensor's shape and strides."""
    import torch
    shape, strides = t.shape, t.stride()
    if t.dtype is not torch.bfloat16 or len(shape) != 3 or shape[1] != heads or shape[2] != dim:
        raise ZlError(1, f"{what} must be a torch.bfloat16 tensor [tokens, {heads}, {dim}]")
    if strides[2] != 1 or (heads > 1 and strides[1] != dim):
        raise ZlError(1, f"{what}: heads and elements of a token must be contiguous")
    _on_gpu(what, t, device)
    n = shape[0]
    return n, strides[0] if n > 1 else heads * dim, shape, strides


def _like(t, other, shape: tuple, device: int, strides: Optional[tuple] = None) -> bool:
    """Of the other's type, of its shape, on its device; of these strides, or contiguous."""
    return (t.shape == shape and t.dtype is other.dtype and t.get_device() == device and
            (t.is_contiguous() if strides is None else t.stride() == strides))


def cache_write(cache: KvCache, batch: CacheBatch, k, v, stream=None):
    """zl_cache_write: the new tokens' k, v [total_q, n_kv_heads, head_dim] bf16 (slices of a packed tensor will do) go into
    their places of the cache, quantised where it holds 8 bits."""
    c, dev = cache.check()
    n, stride, shape, strides = _token_rows("k", k, c.n_kv_heads, c.head_dim, dev)
    if not _like(v, k, shape, dev, strides):
        raise ZlError(1, "k and v must be of the same shape, strides, type and device")
    b = batch.check(n, dev)
    _check(_lib.zl_cache_write(ctypes.byref(c), ctypes.byref(b), k.data_ptr(), v.data_ptr(), stride, _call_stream(stream, dev)), "zl_cache_write")


def cache_read(cache: KvCache, batch: CacheBatch, cu_kv, k, v, first=None, stream=None):
    """zl_cache_read: the tokens of sequence s from position first[s] on (None: 0) into rows [cu_kv[s], cu_kv[s+1]) of the
    packed bf16 tensors k, v [total_kv, n_kv_heads, head_dim]; rows without a key become 0."""
    c, dev = cache.check()
    n, _, shape, _ = _token_rows("k", k, c.n_kv_heads, c.head_dim, dev)
    if not k.is_contiguous():
        raise ZlError(1, "k must be contiguous")
    if not _like(v, k, shape, dev):
        raise ZlError(1, "v must be contiguous, of k's shape and type, on its device")
    b = batch.check(None, dev)
    _ints("cu_kv", cu_kv, (b.n_seqs + 1,))
    _on_gpu("cu_kv", cu_kv, dev)
    if first is not None:
        _ints("first", first, (b.n_seqs,))
        _on_gpu("first", first, dev)
    _check(_lib.zl_cache_read(ctypes.byref(c), ctypes.byref(b), _ptr(first), cu_kv.data_ptr(), n, k.data_ptr(), v.data_ptr(),
                              _call_stream(stream, dev)), "zl_cache_read")


class CachedAttnHandle:
    """Owns a ``zl_cached_attn*``: attention over caches of a number of heads, for every layer and batch."""

    def __init__(self, ptr: int, n_heads: int, n_kv_heads: int, head_dim: int):
        self._ptr = ctypes.c_void_p(ptr)
        self.n_heads, self.n_kv_heads, self.head_dim = n_heads, n_kv_heads, head_dim

    @property
    def ptr(self):
        return self._ptr

    @property
    def workspace_bytes(self) -> int:
        """zl_cached_attn_workspace_bytes: workspace of cached_attn_fwd, whatever the batch."""
        n = ctypes.c_size_t()
        _check(_lib.zl_cached_attn_workspace_bytes(self._ptr, ctypes.byref(n)), "zl_cached_attn_workspace_bytes")
        return int(n.value)

    def last_device_status(self) -> Tuple[int, int]:
        c, w = ctypes.c_int32(), ctypes.c_int32()
        _check(_lib.zl_cached_attn_device_status(self._ptr, ctypes.byref(c), ctypes.byref(w)), "zl_cached_attn_device_status")
        return c.value, w.value

    def close(self):
        if self._ptr:
            _lib.zl_free_cached_attn(self._ptr)
            self._ptr = ctypes.c_void_p(0)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def build_cached_attn(n_heads: int, n_kv_heads: int, head_dim: int, stream=None) -> CachedAttnHandle:
    """zl_build_cached_attn: n_heads query heads, a multiple of n_kv_heads."""
    n_heads, n_kv_heads, head_dim = _int32s((n_heads, n_kv_heads, head_dim))
    out = ctypes.c_void_p()
    _check(_lib.zl_build_cached_attn(n_heads, n_kv_heads, head_dim, _stream_ptr(stream), ctypes.byref(out)), "zl_build_cached_attn")
    return CachedAttnHandle(out.value, n_heads, n_kv_heads, head_dim)


def cached_attn_fwd(attn: CachedAttnHandle, cache: KvCache, batch: CacheBatch, q, scale: float, o, lse, workspace, stream=None):
    """zl_cached_attn_fwd: attention of the new tokens q [total_q, n_heads, head_dim] over the cache, which holds their own keys
    already; o like q (contiguous), lse fp32 [n_heads, total_q] or None, workspace of attn.workspace_bytes."""
    import torch
    c, dev = cache.check()
    n, stride, shape, _ = _token_rows("q", q, attn.n_heads, attn.head_dim, dev)
    if not _like(o, q, shape, dev):
        raise ZlError(1, "o must be contiguous, of q's shape and type, on its device")
    if lse is not None:
        if lse.dtype is not torch.float32 or lse.shape != (attn.n_heads, n) or not lse.is_contiguous():
            raise ZlError(1, f"lse must be a contiguous torch.float32 tensor [{attn.n_heads}, {n}]")
        _on_gpu("lse", lse, dev)
    _on_gpu("workspace", workspace, dev)
    if not workspace.is_contiguous():
        raise ZlError(1, "workspace must be contiguous")
    b = batch.check(n, dev)
    _check(_lib.zl_cached_attn_fwd(attn.ptr, ctypes.byref(c), ctypes.byref(b), q.data_ptr(), stride, scale, o.data_ptr(), _ptr(lse),
                                   workspace.data_ptr(), workspace.nbytes, _call_stream(stream, dev)),
           "zl_cached_attn_fwd")


NOALLOC_SCRATCH_BYTES = 64 * 1024 * 1024


def coalesced_attn_bwd_noalloc(tasks: TaskHandle, q, k, v, o, lse, d_o, scale: float, dq, dk, dv, stream=None):
    """zl_coalesced_attn_bwd_noalloc: the backward for callers that cannot allocate device memory
    (no workspace argument; the scratch is a fixed 64 MiB array inside the library).  Raises
    ZL_ERR_WORKSPACE for placements that need more scratch than that.  Calls must not overlap on
    the GPU, and the first call on a device should be made outside stream capture."""
    _check(_lib.zl_coalesced_attn_bwd_noalloc(tasks.ptr, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(d_o),
                                              scale, _ptr(dq), _ptr(dk), _ptr(dv),
                                              _stream_ptr(stream)), "zl_coalesced_attn_bwd_noalloc")


def launch_count() -> int:
    return int(_lib.zl_launch_count())
