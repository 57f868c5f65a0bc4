"""ctypes binding of ``libkvp.so`` - argument marshalling only; every step of the path runs in the
library's CUDA kernels.  Function names mirror ``include/kvp.h``.  The paged cache's calls on tensors are marshalled by a
module in C++ (``csrc/kvp_calls.cpp``); what it does not take is looked at here, and refused with the reason; where the module is not there, all calls are.

PyTorch is used here for device memory and streams only (``Context`` accepts torch tensors and
passes their ``data_ptr()``).  There is no CPU fallback: if the shared library is missing or cannot
be loaded, importing a symbol raises.
"""
from __future__ import annotations

import ctypes
import importlib.util
import os
import struct
import subprocess
import warnings
from typing import List, Optional, Sequence, Tuple

from . import build as _build

KVP_OK = 0
STATUS_NAMES = {0: "KVP_OK", 1: "KVP_ERR_INVALID", 2: "KVP_ERR_CAPACITY", 3: "KVP_ERR_NOT_FOUND",
                4: "KVP_ERR_STATE", 5: "KVP_ERR_UNSUPPORTED", 6: "KVP_ERR_CUDA", 7: "KVP_ERR_TIMEOUT"}
DTYPE_F32, DTYPE_BF16 = 0, 1
REBASE, MATERIALIZE = 1, 2
ROPE_QUERY, FORCE_SIMPLE, CONTINUE, PRECISE_QK, PARTIAL, SKIP_QUERY_BLOCK = 1, 2, 4, 8, 16, 32
TUNE_SPLIT_TARGET_CTAS, TUNE_FORCE_SPLITS, TUNE_TIME_KERNELS, TUNE_FUSED_APPEND, TUNE_CTA_PAIRS = 1, 2, 3, 5, 6


class KvpError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"{STATUS_NAMES.get(code, code)}: {text}")
        self.code = code


class kvp_config(ctypes.Structure):
    _fields_ = [
        ("struct_bytes", ctypes.c_int32), ("device", ctypes.c_int32), ("n_layers", ctypes.c_int32),
        ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("rope_pairing", ctypes.c_int32), ("rope_theta", ctypes.c_double),
        ("inv_freq", ctypes.POINTER(ctypes.c_double)), ("softmax_scale", ctypes.c_double),
        ("pool", ctypes.c_void_p), ("pool_bytes", ctypes.c_uint64), ("workspace", ctypes.c_void_p),
        ("workspace_bytes", ctypes.c_uint64), ("max_packets", ctypes.c_int32), ("max_adapters", ctypes.c_int32),
        ("max_batch", ctypes.c_int32), ("max_slots", ctypes.c_int32), ("max_prefix_tokens", ctypes.c_int32),
        ("max_query_tokens", ctypes.c_int32), ("max_ws_rows", ctypes.c_int32), ("max_assemblies", ctypes.c_int32),
        ("max_compressed", ctypes.c_int32),
    ]


class kvp_rope(ctypes.Structure):
    _fields_ = [
        ("struct_bytes", ctypes.c_int32), ("pairing", ctypes.c_int32), ("rotary_dim", ctypes.c_int32),
        ("reserved", ctypes.c_int32), ("theta", ctypes.c_double), ("inv_freq", ctypes.POINTER(ctypes.c_double)),
        ("scale", ctypes.c_double), ("original_positions", ctypes.c_double), ("low_rotations", ctypes.c_double),
        ("high_rotations", ctypes.c_double), ("magnitude", ctypes.c_double),
    ]


class kvp_tokens(ctypes.Structure):
    _fields_ = [
        ("struct_bytes", ctypes.c_int32), ("n_tokens", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32), ("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
        ("q_out", ctypes.c_void_p), ("k_out", ctypes.c_void_p), ("q_stride", ctypes.c_int64 * 2),
        ("k_stride", ctypes.c_int64 * 2), ("v_stride", ctypes.c_int64 * 2), ("q_out_stride", ctypes.c_int64 * 2),
        ("k_out_stride", ctypes.c_int64 * 2), ("positions", ctypes.c_void_p), ("slots", ctypes.c_void_p),
        ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("eps", ctypes.c_double),
    ]


class kvp_cache_config(ctypes.Structure):
    _fields_ = [
        ("struct_bytes", ctypes.c_int32), ("device", ctypes.c_int32), ("n_layers", ctypes.c_int32),
        ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("page_size", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("max_batch", ctypes.c_int32),
        ("layer_stride", ctypes.c_int64), ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
        ("row_stride", ctypes.c_int64), ("softmax_scale", ctypes.c_double), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_uint64),
    ]


_lib = None


def lib() -> ctypes.CDLL:
    """Load (building first if the sources are newer) ``libkvp.so``; raises if that fails."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.LIB_PATH
    if not os.path.exists(path) or os.environ.get("KVP_REBUILD"):
        path = _build.build()
    L = ctypes.CDLL(path)
    vp, i32, u32, u64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint32, ctypes.c_uint64
    i64 = ctypes.c_int64
    pi32 = ctypes.POINTER(ctypes.c_int32)
    pcfg = ctypes.POINTER(kvp_config)
    sig = {
        "kvp_version": (i32, []),
        "kvp_token_bytes": (u64, [pcfg]),
        "kvp_workspace_bytes": (u64, [pcfg]),
        "kvp_create": (i32, [pcfg, ctypes.POINTER(vp)]),
        "kvp_destroy": (i32, [vp]),
        "kvp_register_packet": (i32, [vp, vp, vp, i32, i32, vp, pi32]),
        "kvp_register_packet_compressed": (i32, [vp, vp, vp, i32, i32, pi32, vp, pi32]),
        "kvp_register_packet_host": (i32, [vp, vp, vp, i32, i32, pi32]),
        "kvp_evict_packet": (i32, [vp, i32]),
        "kvp_register_adapter": (i32, [vp, vp, vp, i32, i32, vp, vp, i32, i32, vp, pi32]),
        # host index arrays go as addresses: assemble and the ragged call are on the path of every request
        "kvp_assemble": (i32, [vp, i32, vp, vp, vp, u32, vp, pi32, pi32]),
        "kvp_assemble_at": (i32, [vp, i32, vp, vp, vp, vp, u32, vp, pi32, pi32]),
        "kvp_partial_bytes": (u64, [vp, i32, i32]),
        "kvp_merge_partials": (i32, [vp, vp, i32, i32, i32, vp, vp, vp]),
        "kvp_query_prefill": (i32, [vp, i32, i32, vp, vp, vp, i32, u32, vp, vp, vp]),
        "kvp_query_prefill_ragged": (i32, [vp, i32, i32, vp, vp, vp, i32, vp, vp, vp, vp]),
        "kvp_export_plan": (i32, [vp, i32, i32, pi32, pi32, pi32, pi32]),
        "kvp_export_cache": (i32, [vp, i32, i32, i32, i32, vp, vp, i32, vp]),
        "kvp_export_schedule": (i32, [vp, i32, i32, pi32, i32, pi32, i32, pi32, i32, pi32]),
        "kvp_segment_mass": (i32, [vp, i32, i32, vp, vp, i32, u32, vp, i32, vp]),
        "kvp_status_word": (i32, [vp, pi32]),
        "kvp_last_launch": (i32, [vp, pi32, pi32, pi32, pi32]),
        "kvp_tune": (i32, [vp, i32, i32]),
        "kvp_kernel_times": (i32, [vp, i32, ctypes.POINTER(ctypes.c_float), i32, pi32]),
        "kvp_last_error": (ctypes.c_char_p, [vp]),
        "kvp_compose_noalloc": (i32, [vp, vp, ctypes.c_int64, i32, i32, i32, i32, ctypes.c_double, i32, pi32, pi32, pi32,
                                      vp, vp, ctypes.c_int64, vp, ctypes.c_char_p, i32]),
        "kvp_rope_frequencies": (i32, [ctypes.POINTER(kvp_rope), ctypes.POINTER(ctypes.c_double)]),
        "kvp_norm_rope": (i32, [i32, i32, i32, vp, vp, vp]),
        "kvp_cache_workspace_bytes": (u64, [ctypes.POINTER(kvp_cache_config)]),
        "kvp_cache_create": (i32, [ctypes.POINTER(kvp_cache_config), ctypes.POINTER(vp)]),
        "kvp_cache_destroy": (i32, [vp]),
        "kvp_cache_append": (i32, [vp, i32, vp, vp, vp]),
        "kvp_cache_attend": (i32, [vp, i32, i32, vp, vp, vp, i64, i32, vp, vp, vp, vp, vp, vp]),
        "kvp_cache_copy": (i32, [vp, i32, vp, vp, vp, vp]),
        "kvp_cache_compact": (i32, [vp, i32, vp, i64, i32, vp, vp, i64, i32, vp, vp, i32, vp, vp]),
        "kvp_cache_take": (i32, [vp, i32, vp]),
        "kvp_cache_share": (i32, [vp, i32, vp]),
        "kvp_cache_release": (i32, [vp, i32, vp]),
        "kvp_cache_fork": (i32, [vp, i32, vp, i32, vp, vp]),
        "kvp_cache_free_pages": (i32, [vp, pi32]),
        "kvp_cache_last_error": (ctypes.c_char_p, [vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)          # AttributeError if the library lacks a declared symbol
        fn.restype = res
        fn.argtypes = args
    _lib = L
    return L


EXPORTED = ["kvp_version", "kvp_token_bytes", "kvp_workspace_bytes", "kvp_create", "kvp_destroy",
            "kvp_register_packet", "kvp_register_packet_compressed", "kvp_register_packet_host", "kvp_evict_packet",
            "kvp_register_adapter", "kvp_assemble", "kvp_assemble_at", "kvp_partial_bytes", "kvp_merge_partials", "kvp_query_prefill", "kvp_query_prefill_ragged",
            "kvp_export_plan", "kvp_export_cache", "kvp_export_schedule", "kvp_segment_mass", "kvp_status_word", "kvp_last_launch", "kvp_tune",
            "kvp_kernel_times", "kvp_last_error", "kvp_compose_noalloc", "kvp_rope_frequencies", "kvp_norm_rope",
            "kvp_cache_workspace_bytes", "kvp_cache_create", "kvp_cache_destroy", "kvp_cache_append", "kvp_cache_attend",
            "kvp_cache_copy", "kvp_cache_compact", "kvp_cache_take", "kvp_cache_share", "kvp_cache_release", "kvp_cache_fork",
            "kvp_cache_free_pages", "kvp_cache_last_error"]


_calls = None


class _NoModule:
    """Takes no call, so that Python marshals all of them."""

    @staticmethod
    def append(*args):
        return -1

    attend = compact = norm_rope = append


def calls():
    """The module that marshals the paged cache's calls on tensors (needs PyTorch, of the version that it was built for); built
    like the library.  Where it can be neither built nor loaded, Python marshals them: 4 us more for each call, the same kernels."""
    global _calls
    if _calls is None:
        L = lib()
        try:
            path = _build.calls_path()
            if not os.path.exists(path) or os.environ.get("KVP_REBUILD"):
                path = _build.build_calls()
            spec = importlib.util.spec_from_file_location("_kvp_calls", path)
            module = importlib.util.module_from_spec(spec)
            spec.loader.exec_module(module)
        except (ImportError, OSError, subprocess.SubprocessError) as e:
            warnings.warn(f"the paged cache's calls are marshalled in Python: {e}", RuntimeWarning)
            module = _NoModule
        else:
            module.bind(*(ctypes.cast(f, ctypes.c_void_p).value for f in (L.kvp_cache_append, L.kvp_cache_attend, L.kvp_cache_compact, L.kvp_norm_rope)))
        _calls = module
    return _calls


def _i32_array(xs: Sequence[int]):
    return (ctypes.c_int32 * max(1, len(xs)))(*[int(x) for x in xs])


def _i32_packed(xs: List[int]):
    # a ctypes array costs six times as much to fill; it takes what is not an int, or not one of 32 bits
    try:
        return struct.pack(f"{len(xs)}i", *xs)
    except struct.error:
        return _i32_array(xs)


def _i32(x: int, name: str) -> int:
    """``x``, which ctypes would cut to 32 bits without a word."""
    if not -2 ** 31 <= x < 2 ** 31:
        raise KvpError(1, f"{name}: {x} is not a number of 32 bits")
    return x


def _i32_list(xs: Sequence[int], name: str):
    try:
        return struct.pack(f"{len(xs)}i", *xs)
    except struct.error:
        return _i32_array([_i32(x, name) for x in xs])


def _ptr(t) -> Optional[int]:
    """Device (or host) address of a torch tensor / int / None."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return int(t.data_ptr())


class Context:
    """Thin object wrapper over the C calls.  ``device=-1`` makes a host-only planning context
    (no GPU needed; nothing can be launched)."""

    def __init__(self, n_layers: int, n_q_heads: int, n_kv_heads: int, head_dim: int, dtype: str,
                 rope_theta: float = 10000.0, rope_pairing: int = 0, softmax_scale: float = 0.0,
                 inv_freq: Optional[Sequence[float]] = None, pool_tokens: int = 0, max_packets: int = 64,
                 max_adapters: int = 4, max_batch: int = 1, max_slots: int = 64, max_prefix_tokens: int = 4096,
                 max_query_tokens: int = 128, max_ws_rows: int = 0, max_assemblies: int = 1, device: int = 0,
                 max_compressed: int = 0):
        self._L = lib()
        self._h = ctypes.c_void_p()
        cfg = kvp_config()
        cfg.struct_bytes = ctypes.sizeof(kvp_config)
        cfg.device = device
        cfg.n_layers, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim = n_layers, n_q_heads, n_kv_heads, head_dim
        cfg.dtype = DTYPE_BF16 if dtype == "bf16" else DTYPE_F32
        cfg.rope_pairing = rope_pairing
        cfg.rope_theta = rope_theta
        self._inv_freq = None
        if inv_freq is not None:
            self._inv_freq = (ctypes.c_double * (head_dim // 2))(*inv_freq)
            cfg.inv_freq = ctypes.cast(self._inv_freq, ctypes.POINTER(ctypes.c_double))
        cfg.softmax_scale = softmax_scale
        cfg.max_packets, cfg.max_adapters, cfg.max_batch, cfg.max_slots = max_packets, max_adapters, max_batch, max_slots
        cfg.max_prefix_tokens, cfg.max_query_tokens = max_prefix_tokens, max_query_tokens
        if max_ws_rows <= 0:
            max_ws_rows = max_batch * max_query_tokens + 64 * max_slots
        cfg.max_ws_rows, cfg.max_assemblies = max_ws_rows, max_assemblies
        cfg.max_compressed = max_compressed
        self.dtype, self.device = dtype, device
        self.n_layers, self.n_q_heads, self.n_kv_heads, self.head_dim = n_layers, n_q_heads, n_kv_heads, head_dim
        self.token_bytes = int(self._L.kvp_token_bytes(ctypes.byref(cfg)))
        if self.token_bytes == 0:
            raise KvpError(1, "invalid configuration")
        self.pool = self.workspace = None
        if device >= 0:
            import torch
            self._torch = torch
            self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
                lambda index: torch.cuda.current_stream(index).cuda_stream)
            dev = torch.device(f"cuda:{device}")
            ws_bytes = int(self._L.kvp_workspace_bytes(ctypes.byref(cfg)))
            self.pool = torch.empty(max(1, pool_tokens) * self.token_bytes + 1024, dtype=torch.uint8, device=dev)
            self.workspace = torch.empty(ws_bytes + 1024, dtype=torch.uint8, device=dev)
            pa = (self.pool.data_ptr() + 1023) // 1024 * 1024
            wa = (self.workspace.data_ptr() + 1023) // 1024 * 1024
            cfg.pool, cfg.pool_bytes = pa, max(1, pool_tokens) * self.token_bytes
            cfg.workspace, cfg.workspace_bytes = wa, ws_bytes
            self.workspace_bytes = ws_bytes
        self.cfg = cfg
        rc = self._L.kvp_create(ctypes.byref(cfg), ctypes.byref(self._h))
        if rc != KVP_OK:
            raise KvpError(rc, (self._L.kvp_last_error(None) or b"").decode())

    # -- plumbing ------------------------------------------------------------------------------
    def _check(self, rc: int):
        if rc != KVP_OK:
            raise KvpError(rc, (self._L.kvp_last_error(self._h) or b"").decode())

    def _stream(self, stream=None):
        if stream is not None:
            return stream.cuda_stream if self.device >= 0 else None
        return self._raw_stream(self.device) if self.device >= 0 else None

    def close(self):
        if self._h:
            self._L.kvp_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- the six calls ---------------------------------------------------------------------------
    def register_packet(self, k, v, n_tokens: int, cache_pos0: int = 0, stream=None) -> int:
        out = ctypes.c_int32(-1)
        self._check(self._L.kvp_register_packet(self._h, _ptr(k), _ptr(v), n_tokens, cache_pos0,
                                                self._stream(stream), ctypes.byref(out)))
        return out.value

    def register_packet_compressed(self, k, v, n_tokens: int, cache_pos0: int, kept: Sequence[int], stream=None) -> int:
        """kept: n_layers * n_kv_heads row counts; k, v: the kept rows of every (layer, kv head), runs back to back."""
        out = ctypes.c_int32(-1)
        self._check(self._L.kvp_register_packet_compressed(self._h, _ptr(k), _ptr(v), n_tokens, cache_pos0,
                                                           _i32_array(list(kept)), self._stream(stream), ctypes.byref(out)))
        return out.value

    def register_packet_host(self, k_host, v_host, n_tokens: int, cache_pos0: int = 0) -> int:
        """k_host, v_host: host tensors [n_layers][n_kv_heads][n_tokens][head_dim] (pinned for overlap), kept alive
        by the caller; they are copied into the pool by the first assemble that names the packet."""
        out = ctypes.c_int32(-1)
        self._check(self._L.kvp_register_packet_host(self._h, _ptr(k_host), _ptr(v_host), n_tokens, cache_pos0,
                                                     ctypes.byref(out)))
        return out.value

    def evict_packet(self, packet_id: int) -> None:
        self._check(self._L.kvp_evict_packet(self._h, packet_id))

    def register_adapter(self, hk, hv, n_header: int, header_pos0: int, tk, tv, n_trailer: int,
                         trailer_pos0: int, stream=None) -> int:
        out = ctypes.c_int32(-1)
        self._check(self._L.kvp_register_adapter(self._h, _ptr(hk), _ptr(hv), n_header, header_pos0, _ptr(tk),
                                                 _ptr(tv), n_trailer, trailer_pos0, self._stream(stream),
                                                 ctypes.byref(out)))
        return out.value

    def assemble(self, items: Sequence[Sequence[Tuple[int, int]]], flags: int = REBASE, stream=None, pos_base=None):
        """items[b] = [(packet_id, adapter_id), ...].  Returns (assembly_id, prefix_len list).
        pos_base (one position per request) -> ``kvp_assemble_at``: this rank's part of a sharded request."""
        B = len(items)
        offs, pids, aids = [0], [], []
        for it in items:
            for pid, aid in it:
                pids.append(pid)
                aids.append(aid)
            offs.append(len(pids))
        offs, pids, aids = _i32_packed(offs), _i32_packed(pids), _i32_packed(aids)
        plen = (ctypes.c_int32 * max(1, B))()
        aid = ctypes.c_int32(-1)
        if pos_base is not None:
            self._check(self._L.kvp_assemble_at(self._h, B, offs, pids, aids, _i32_array(list(pos_base)), flags,
                                                self._stream(stream), plen, ctypes.byref(aid)))
        else:
            self._check(self._L.kvp_assemble(self._h, B, offs, pids, aids, flags, self._stream(stream), plen,
                                             ctypes.byref(aid)))
        return aid.value, plen[:B]

    def partial_bytes(self, batch: int, q_len: int) -> int:
        return int(self._L.kvp_partial_bytes(self._h, batch, q_len))

    def merge_partials(self, parts, n_parts: int, batch: int, q_len: int, out, lse=None, stream=None):
        self._check(self._L.kvp_merge_partials(self._h, _ptr(parts), n_parts, batch, q_len, _ptr(out), _ptr(lse),
                                               self._stream(stream)))

    def query_prefill(self, assembly_id: int, layer: int, q, k_new, v_new, q_len: int, out, lse=None,
                      flags: int = 0, stream=None):
        self._check(self._L.kvp_query_prefill(self._h, assembly_id, layer, _ptr(q), _ptr(k_new), _ptr(v_new), q_len,
                                              flags, _ptr(out), _ptr(lse), self._stream(stream)))

    def query_prefill_ragged(self, assembly_id: int, layer: int, q, k_new, v_new, q_len_max: int, q_lens: Sequence[int],
                             out, lse=None, stream=None):
        """Per-request query lengths; the tensors are padded to q_len_max tokens per request."""
        self._check(self._L.kvp_query_prefill_ragged(self._h, assembly_id, layer, _ptr(q), _ptr(k_new), _ptr(v_new),
                                                     q_len_max, _i32_array(list(q_lens)), _ptr(out), _ptr(lse),
                                                     self._stream(stream)))

    # -- helpers ---------------------------------------------------------------------------------
    def export_plan(self, assembly_id: int, b: int):
        """(src_row [P], delta [P], seg_table [n_seg][4]) of request b as numpy int32 arrays."""
        import numpy as np
        nseg = ctypes.c_int32(0)
        pi = ctypes.POINTER(ctypes.c_int32)
        self._check(self._L.kvp_export_plan(self._h, assembly_id, b, None, None, None, ctypes.byref(nseg)))
        segs = np.zeros((max(1, nseg.value), 4), dtype=np.int32)
        self._check(self._L.kvp_export_plan(self._h, assembly_id, b, None, None, segs.ctypes.data_as(pi),
                                            ctypes.byref(nseg)))
        segs = segs[:nseg.value]
        prefix_len = int((segs[:, 1] + segs[:, 2]).max()) if nseg.value else 0
        src = np.zeros(max(1, prefix_len), dtype=np.int32)
        dl = np.zeros(max(1, prefix_len), dtype=np.int32)
        self._check(self._L.kvp_export_plan(self._h, assembly_id, b, src.ctypes.data_as(pi), dl.ctypes.data_as(pi),
                                            None, ctypes.byref(nseg)))
        return src[:prefix_len], dl[:prefix_len], segs

    def export_cache(self, assembly_id: int, layer: int, b: int, prefix_len: int, n_query_rows: int,
                     k_as_f32: bool = False, stream=None):
        torch = self._torch
        dt = torch.bfloat16 if self.dtype == "bf16" else torch.float32
        n = prefix_len + n_query_rows
        dev = torch.device(f"cuda:{self.device}")
        k = torch.empty((n, self.n_kv_heads, self.head_dim), dtype=torch.float32 if k_as_f32 else dt, device=dev)
        v = torch.empty((n, self.n_kv_heads, self.head_dim), dtype=dt, device=dev)
        self._check(self._L.kvp_export_cache(self._h, assembly_id, layer, b, n_query_rows, _ptr(k), _ptr(v),
                                             1 if k_as_f32 else 0, self._stream(stream)))
        return k, v

    def export_schedule(self, assembly_id: int, q_len: int):
        """(cta_begin [n_ctas+1], works [n][8], merges [m][8], n_slots) as numpy int32 arrays."""
        import numpy as np
        pi = ctypes.POINTER(ctypes.c_int32)
        counts = (ctypes.c_int32 * 4)()
        self._check(self._L.kvp_export_schedule(self._h, assembly_id, q_len, None, 0, None, 0, None, 0, counts))
        cb = np.zeros(counts[0] + 1, dtype=np.int32)
        works = np.zeros((max(1, counts[1]), 8), dtype=np.int32)
        merges = np.zeros((max(1, counts[2]), 8), dtype=np.int32)
        self._check(self._L.kvp_export_schedule(self._h, assembly_id, q_len, cb.ctypes.data_as(pi), cb.size,
                                                works.ctypes.data_as(pi), works.shape[0],
                                                merges.ctypes.data_as(pi), merges.shape[0], counts))
        return cb, works[:counts[1]], merges[:counts[2]], int(counts[3])

    def segment_mass(self, assembly_id: int, layer: int, q, lse, q_len: int, n_cols: int, flags: int = 0, stream=None):
        """float32 [batch][q_len][n_q_heads][n_cols] attention mass per segment (+ query block) of the last prefill."""
        torch = self._torch
        mass = torch.empty((q.shape[0], q_len, self.n_q_heads, n_cols), dtype=torch.float32, device=q.device)
        self._check(self._L.kvp_segment_mass(self._h, assembly_id, layer, _ptr(q), _ptr(lse), q_len, flags, _ptr(mass),
                                             n_cols, self._stream(stream)))
        return mass

    def status_word(self) -> int:
        w = ctypes.c_int32(0)
        rc = self._L.kvp_status_word(self._h, ctypes.byref(w))
        if rc not in (KVP_OK, 7):
            self._check(rc)
        return w.value

    def last_launch(self):
        a, b, c, d = (ctypes.c_int32() for _ in range(4))
        self._check(self._L.kvp_last_launch(self._h, ctypes.byref(a), ctypes.byref(b), ctypes.byref(c), ctypes.byref(d)))
        return {"kind": a.value, "ctas": b.value, "splits": c.value, "launches": d.value}

    def tune(self, key: int, value: int):
        self._check(self._L.kvp_tune(self._h, key, value))

    def kernel_times(self, which: int = 0, cap: int = 4096) -> List[float]:
        """Device durations (ms) of the attention (0) / gather (1) kernels since the last call."""
        buf = (ctypes.c_float * cap)()
        n = ctypes.c_int32(0)
        self._check(self._L.kvp_kernel_times(self._h, which, buf, cap, ctypes.byref(n)))
        return [float(buf[i]) for i in range(n.value)]


def compose_noalloc(pool_k: int, pool_v: int, pool_rows: int, n_planes: int, head_dim: int, dtype: str,
                    rope_pairing: int, rope_theta: float, segments, cache_k, cache_v, cache_rows: int, stream=None):
    """``kvp_compose_noalloc``: gather + re-base ``segments`` = [(src_row0, length, delta), ...] from the
    caller's pool planes into the caller's cache planes without any allocation in the library.
    ``pool_k``/``pool_v`` are device addresses, ``cache_k``/``cache_v`` torch tensors (or addresses)."""
    L = lib()
    n = len(segments)
    err = ctypes.create_string_buffer(256)
    st = ctypes.c_void_p(stream.cuda_stream) if stream is not None else None
    rc = L.kvp_compose_noalloc(pool_k, pool_v, pool_rows, n_planes, head_dim, DTYPE_BF16 if dtype == "bf16" else DTYPE_F32,
                               rope_pairing, rope_theta, n, _i32_array([s[0] for s in segments]),
                               _i32_array([s[1] for s in segments]), _i32_array([s[2] for s in segments]),
                               _ptr(cache_k), _ptr(cache_v), cache_rows, st, err, 256)
    if rc != KVP_OK:
        raise KvpError(rc, err.value.decode())


# ---- norms and rotation of new tokens; a cache in pages ------------------------------------------------------

class Rope:
    """``kvp_rope``: rotary positions of the first ``rotary_dim`` elements of a head, scaled for long contexts or not."""

    def __init__(self, head_dim: int, rotary_dim: Optional[int] = None, theta: float = 10000.0, pairing: int = 0,
                 inv_freq: Optional[Sequence[float]] = None, scale: float = 1.0, original_positions: float = 0.0,
                 low_rotations: float = 1.0, high_rotations: float = 4.0, magnitude: float = 1.0):
        r = kvp_rope()
        r.struct_bytes = ctypes.sizeof(kvp_rope)
        r.pairing, r.rotary_dim = _i32(pairing, "pairing"), _i32(head_dim if rotary_dim is None else rotary_dim, "rotary_dim")
        r.theta, r.scale, r.original_positions = theta, scale, original_positions
        r.low_rotations, r.high_rotations, r.magnitude = low_rotations, high_rotations, magnitude
        self._inv_freq = None
        if inv_freq is not None:
            if len(inv_freq) != r.rotary_dim // 2:
                raise KvpError(1, f"rope: {len(inv_freq)} frequencies for rotary_dim {r.rotary_dim}")
            self._inv_freq = (ctypes.c_double * max(1, len(inv_freq)))(*inv_freq)
            r.inv_freq = ctypes.cast(self._inv_freq, ctypes.POINTER(ctypes.c_double))
        # the frequencies after scaling are formed once, not by every call that rotates (64 powers: 4 us)
        self._scaled = (ctypes.c_double * max(1, r.rotary_dim // 2))()
        _checked(lib().kvp_rope_frequencies(ctypes.byref(r), self._scaled))
        r.inv_freq = ctypes.cast(self._scaled, ctypes.POINTER(ctypes.c_double))
        r.scale, r.original_positions = 1.0, 0.0
        self.struct, self.address = r, ctypes.addressof(r)

    def frequencies(self) -> List[float]:
        """The frequencies after scaling, as ``Context(inv_freq=...)`` takes them."""
        return list(self._scaled)[:self.struct.rotary_dim // 2]


def _checked(rc: int, cache=None):
    if rc != KVP_OK:
        raise KvpError(rc, (lib().kvp_cache_last_error(cache) or b"").decode())


def _raw_stream(index: int) -> int:
    """The current stream of device ``index``."""
    import torch
    get = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return get(index) if get else torch.cuda.current_stream(index).cuda_stream


def _dtype_of(t) -> int:
    import torch
    if t.dtype not in (torch.float32, torch.bfloat16):
        raise KvpError(1, f"{t.dtype} is neither float32 nor bfloat16")
    return DTYPE_F32 if t.dtype == torch.float32 else DTYPE_BF16


def _rows(t, dtype, device: int, d: int, n: int, name: str):
    """(address, heads, token stride, head stride) of [n][head][d]."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 3 or shape[0] != n or shape[2] != d or t.dtype is not dtype or t.get_device() != device or stride[2] != 1:
        raise KvpError(1, f"{name}: {tuple(shape)} with strides {stride}, {t.dtype} on {t.device}, not [{n}][heads][{d}] of {dtype}")
    return t.data_ptr(), shape[1], stride[0], stride[1]


def _ints(t, device: int, shape, name: str) -> int:
    if t.dtype is not _int32() or t.get_device() != device or t.shape != shape or not t.is_contiguous():
        raise KvpError(1, f"{name}: {tuple(t.shape)} with strides {t.stride()}, {t.dtype} on {t.device}, not {shape} of int32")
    return t.data_ptr()


def _table(t, device: int, n: int, name: str):
    """(address, row stride, columns) of [n][columns]."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or shape[0] != n or t.dtype is not _int32() or t.get_device() != device or (stride[1] != 1 and shape[1] > 1):
        raise KvpError(1, f"{name}: {tuple(shape)} with strides {stride}, {t.dtype} on {t.device}, not [{n}][pages] of int32")
    return t.data_ptr(), stride[0], _i32(shape[1], name)


_int32_dtype = None


def _int32():
    global _int32_dtype
    if _int32_dtype is None:
        import torch
        _int32_dtype = torch.int32
    return _int32_dtype


_PAIR = struct.Struct("2q").pack
_TOKENS = struct.Struct("4i5Q10q4Qd")                      # kvp_tokens
assert _TOKENS.size == ctypes.sizeof(kvp_tokens)


def _tokens(dtype, device: int, d: int, q, k, v, q_out, k_out, positions, slots, q_weight, k_weight, eps) -> bytes:
    first = q if q is not None else k
    if first is None:
        raise KvpError(1, "neither q nor k")
    n = _i32(first.shape[0], "tokens")
    none = (0, 0, 0, 0)
    qp, hq, q0, q1 = none if q is None else _rows(q, dtype, device, d, n, "q")
    kp, hk, k0, k1 = none if k is None else _rows(k, dtype, device, d, n, "k")
    vp, hv, v0, v1 = none if v is None else _rows(v, dtype, device, d, n, "v")
    qo, hqo, qo0, qo1 = none if q_out is None else _rows(q_out, dtype, device, d, n, "q_out")
    ko, hko, ko0, ko1 = none if k_out is None else _rows(k_out, dtype, device, d, n, "k_out")
    if (v is not None and hv != hk) or (q_out is not None and hqo != hq) or (k_out is not None and hko != hk):
        raise KvpError(1, f"heads: q {hq}, q_out {hqo}, k {hk}, k_out {hko}, v {hv}")
    pos = 0 if positions is None else _ints(positions, device, (n,), "positions")
    slot = 0 if slots is None else _ints(slots, device, (n,), "slots")
    weights = []
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        if w is not None and (w.dtype is not dtype or w.get_device() != device or w.shape != (d,) or not w.is_contiguous()):
            raise KvpError(1, f"{name}: {tuple(w.shape)} {w.dtype} on {w.device}")
        weights.append(0 if w is None else w.data_ptr())
    return _TOKENS.pack(_TOKENS.size, n, hq, hk, qp, kp, vp, qo, ko, q0, q1, k0, k1, v0, v1, qo0, qo1, ko0, ko1, pos, slot, *weights, eps)


def norm_rope(q, k, positions, rope: Optional[Rope], q_out=None, k_out=None, q_weight=None, k_weight=None, eps: float = 1e-6,
              stream=None):
    """``kvp_norm_rope``: q, k = [token][head][d] (either may be None) normed per head where there is a weight, then rotated to
    ``positions`` [token]; what ``query_prefill`` takes."""
    first = q if q is not None else k
    if first is None or first.device.type != "cuda":
        raise KvpError(1, "norm_rope: q or k on a CUDA device")
    device = first.get_device()
    rc = calls().norm_rope(device, q, k, positions, None if rope is None else rope.address, q_out, k_out, q_weight, k_weight, eps,
                           _raw_stream(device) if stream is None else stream.cuda_stream)
    if rc >= 0:
        return _checked(rc)
    a = _tokens(first.dtype, device, first.shape[-1], q, k, None, q_out, k_out, positions, None, q_weight, k_weight, eps)
    _checked(lib().kvp_norm_rope(device, _dtype_of(first), first.shape[-1], a, None if rope is None else rope.address,
                                 _raw_stream(device) if stream is None else stream.cuda_stream))


def _closed(*args):
    raise KvpError(4, "the cache is closed")


# Workspaces of caches that were closed without a wait for the device, by their ids: calls on other streams may still use them, and
# PyTorch's allocator knows only of the stream that they were made on.
_unwaited = {}


def _wait_for(device: int):
    """Waits for all work on the device.  Workspaces that had no wait until then may go."""
    import torch
    before = [i for i, w in list(_unwaited.items()) if w[0] == device]
    torch.cuda.synchronize(device)
    for i in before:
        _unwaited.pop(i, None)


class PagedCache:
    """``kvp_cache`` over the caller's page tensors: ``k``, ``v`` = [layer][page][kv head][row][d] (order "heads") or
    [layer][page][row][kv head][d] ("tokens"), with any strides.  CPU tensors make a host-only cache: pages are counted,
    nothing runs.  attend calls of one cache share its workspace: they have to be ordered among each other, recorded ones too,
    and the cache has to outlive the graphs that hold them."""

    def __init__(self, k, v, n_q_heads: int, order: str = "heads", max_batch: int = 64, softmax_scale: float = 0.0):
        import torch
        self._L, self._h = lib(), ctypes.c_void_p()
        if order not in ("heads", "tokens"):
            raise KvpError(1, f"order {order!r} is neither 'heads' nor 'tokens'")
        if k.dim() != 5 or k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype or k.device != v.device:
            raise KvpError(1, "k and v have to be alike, [layer][page][kv head][row][d] or [layer][page][row][kv head][d]")
        if k.shape[4] > 1 and k.stride(4) != 1:
            raise KvpError(1, "the elements of a row do not lie side by side")
        head, row = (2, 3) if order == "heads" else (3, 2)
        self.k, self.v, self.dtype = k, v, k.dtype
        self._float32 = torch.float32
        self._current = getattr(torch._C, "_cuda_getCurrentRawStream", None) or _raw_stream
        self.device = k.device.index if k.device.type == "cuda" else -1
        self.n_layers, self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = k.shape[0], k.shape[1], k.shape[head], k.shape[row], k.shape[4]
        for n, name in ((n_q_heads, "n_q_heads"), (max_batch, "max_batch"), *((n, "size") for n in k.shape)):
            _i32(n, name)
        self.n_q_heads, self.max_batch = n_q_heads, max_batch
        c = kvp_cache_config()
        c.struct_bytes, c.device, c.n_layers, c.n_q_heads, c.n_kv_heads = ctypes.sizeof(c), self.device, self.n_layers, n_q_heads, self.n_kv_heads
        c.head_dim, c.dtype, c.page_size, c.n_pages, c.max_batch = self.head_dim, _dtype_of(k), self.page_size, self.n_pages, max_batch
        c.layer_stride, c.page_stride, c.head_stride, c.row_stride = k.stride(0), k.stride(1), k.stride(head), k.stride(row)
        c.softmax_scale = softmax_scale
        self.workspace = None
        if self.device >= 0:
            n = int(self._L.kvp_cache_workspace_bytes(ctypes.byref(c)))
            self.workspace = torch.empty(n + 256, dtype=torch.uint8, device=k.device)
            c.k, c.v = k.data_ptr(), v.data_ptr()
            c.workspace, c.workspace_bytes = (self.workspace.data_ptr() + 255) // 256 * 256, n
        self.cfg = c
        _checked(self._L.kvp_cache_create(ctypes.byref(c), ctypes.byref(self._h)))
        module = calls()
        self._append, self._attend, self._compact, self._code = module.append, module.attend, module.compact, c.dtype

    def close(self):
        if self._h:
            self._append = self._attend = self._compact = _closed
            h, self._h = self._h, ctypes.c_void_p()
            self._L.kvp_cache_destroy(h)
            if self.workspace is not None:
                # calls on other streams may still use it; while something is recorded nothing may be waited for
                import torch
                _unwaited[id(self.workspace)] = self.device, self.workspace
                if not torch.cuda.is_current_stream_capturing():
                    _wait_for(self.device)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc: int):
        if rc != KVP_OK:
            _checked(rc, self._h)

    def _stream(self, stream):
        if self.device < 0:
            return None
        return self._current(self.device) if stream is None else stream.cuda_stream

    # -- rows ------------------------------------------------------------------------------------
    def append(self, layer: int, k, v, positions, slots, rope: Optional[Rope] = None, q=None, q_out=None, k_out=None,
               q_weight=None, k_weight=None, eps: float = 1e-6, stream=None):
        """q, k, v = [token][head][d] as a layer's projections give them.  Keys (normed, rotated) and values go to ``slots``
        [token] = page * page_size + row (a slot outside the store: nowhere), queries to ``q_out``."""
        rc = self._append(self._h.value, layer, self._code, self.device, self.head_dim, k, v, positions, slots,
                          None if rope is None else rope.address, q, q_out, k_out, q_weight, k_weight, eps, self._stream(stream))
        if rc == 0:
            return
        if rc > 0:
            self._check(rc)
        # the tensors do not fit one another or the cache: what is wrong is found, and said, here
        _i32(layer, "layer")
        if k is None or v is None or slots is None:
            raise KvpError(1, "append: k, v and slots are needed")
        a = _tokens(self.dtype, self.device, self.head_dim, q, k, v, q_out, k_out, positions, slots, q_weight, k_weight, eps)
        self._check(self._L.kvp_cache_append(self._h, layer, a, None if rope is None else rope.address, self._stream(stream)))

    def attend(self, layer: int, q, table, lens, out, lse=None, first=None, stream=None):
        """q, out = [request][q head][d]; table = [request][pages], lens, first = [request], int32; lse = float32
        [request][q head].  Request b attends to its rows first[b] <= j < lens[b]."""
        rc = self._attend(self._h.value, layer, self._code, self.device, self.head_dim, self.n_q_heads, q, out, table, lens, first, lse,
                          self._stream(stream))
        if rc == 0:
            return
        if rc > 0:
            self._check(rc)
        _i32(layer, "layer")
        n, dev, dtype, d = _i32(q.shape[0], "requests"), self.device, self.dtype, self.head_dim
        qp, hq, q0, q1 = _rows(q, dtype, dev, d, n, "q")
        op, ho, o0, o1 = _rows(out, dtype, dev, d, n, "out")
        if hq != self.n_q_heads or ho != hq:
            raise KvpError(1, f"heads: q {hq}, out {ho}, the cache {self.n_q_heads}")
        if lse is not None and (lse.dtype is not self._float32 or lse.get_device() != dev or lse.shape != (n, hq) or not lse.is_contiguous()):
            raise KvpError(1, f"lse: {tuple(lse.shape)} {lse.dtype} on {lse.device}")
        tp, t0, cols = _table(table, dev, n, "table")
        self._check(self._L.kvp_cache_attend(self._h, layer, n, qp, _PAIR(q0, q1), tp, t0, cols, _ints(lens, dev, (n,), "lens"),
                                             None if first is None else _ints(first, dev, (n,), "first"), op, _PAIR(o0, o1),
                                             None if lse is None else lse.data_ptr(), self._stream(stream)))

    def copy(self, src: Sequence[int], dst: Sequence[int], rows: Optional[Sequence[int]] = None, stream=None):
        """The first rows[i] rows (None: all) of page src[i] to page dst[i], in all layers."""
        if len(src) != len(dst) or (rows is not None and len(rows) != len(src)):
            raise KvpError(1, "copy: lists of different lengths")
        self._check(self._L.kvp_cache_copy(self._h, len(src), _i32_list(src, "page"), _i32_list(dst, "page"),
                                           None if rows is None else _i32_list(rows, "rows"), self._stream(stream)))

    def compact(self, table, lens, new_table, kept, n_kept, stream=None):
        """Row i < n_kept[b] of new_table[b]'s pages becomes row kept[b][l][h][i] of table[b]'s; kept = [request][layer or
        1][kv head or 1][entries], int32.  The new pages must not be among those that are read."""
        rc = self._compact(self._h.value, self.device, self.n_layers, self.n_kv_heads, table, lens, new_table, kept, n_kept, self._stream(stream))
        if rc == 0:
            return
        if rc > 0:
            self._check(rc)
        n, dev = _i32(n_kept.shape[0], "requests"), self.device
        shape, stride = kept.shape, kept.stride()
        if len(shape) != 4 or shape[0] != n or kept.dtype is not _int32() or kept.get_device() != dev or (stride[3] != 1 and shape[3] > 1):
            raise KvpError(1, f"kept: {tuple(shape)} with strides {stride}, {kept.dtype} on {kept.device}")
        if shape[1] not in (1, self.n_layers) or shape[2] not in (1, self.n_kv_heads):
            raise KvpError(1, f"kept: lists for {shape[1]} layers and {shape[2]} heads")
        strides = struct.pack("3q", stride[0], stride[1] if shape[1] > 1 else 0, stride[2] if shape[2] > 1 else 0)
        tp, t0, cols = _table(table, dev, n, "table")
        np, n0, new_cols = _table(new_table, dev, n, "new_table")
        self._check(self._L.kvp_cache_compact(self._h, n, tp, t0, cols, _ints(lens, dev, (n,), "lens"), np, n0, new_cols, kept.data_ptr(),
                                              strides, _i32(shape[3], "kept"), _ints(n_kept, dev, (n,), "n_kept"), self._stream(stream)))

    # -- pages -----------------------------------------------------------------------------------
    def take(self, n: int) -> List[int]:
        out = (ctypes.c_int32 * max(1, min(_i32(n, "pages"), self.n_pages)))()     # (no more can be taken)
        self._check(self._L.kvp_cache_take(self._h, n, out))
        return list(out)[:n]

    def share(self, pages: Sequence[int]):
        self._check(self._L.kvp_cache_share(self._h, len(pages), _i32_list(pages, "page")))

    def release(self, pages: Sequence[int]):
        self._check(self._L.kvp_cache_release(self._h, len(pages), _i32_list(pages, "page")))

    def fork(self, pages: Sequence[int], n_tokens: int, n_forks: int = 1, stream=None) -> List[List[int]]:
        """``n_forks`` page lists for the first ``n_tokens`` rows of ``pages``: whole pages are shared, a last one that is not
        full is copied to a new page for each."""
        cols = -(-_i32(n_tokens, "tokens") // self.page_size)
        if cols > len(pages):
            raise KvpError(1, f"fork: {n_tokens} tokens in {len(pages)} pages of {self.page_size}")
        out = (ctypes.c_int32 * max(1, _i32(n_forks, "forks") * cols))()
        self._check(self._L.kvp_cache_fork(self._h, n_tokens, _i32_list(pages, "page"), n_forks, out, self._stream(stream)))
        return [list(out[f * cols:(f + 1) * cols]) for f in range(n_forks)]

    @property
    def free_pages(self) -> int:
        n = ctypes.c_int32(0)
        self._check(self._L.kvp_cache_free_pages(self._h, ctypes.byref(n)))
        return n.value
