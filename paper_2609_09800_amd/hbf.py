"""Thin ctypes binding of ``libhbf.so`` (the C ABI in ``include/hbf.h``).

Argument marshalling only: every step of the hot path runs in the HIP
kernels of the library.  PyTorch supplies device memory and streams.  If the
library has not been built this module raises on use -- there is no CPU
fallback.
"""
import ctypes
import os
import struct

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libhbf.so")

HBF_OK = 0
HBF_EINVAL = -1
HBF_EALIGN = -2
HBF_EOVERLAP = -3
HBF_ENOWORKSPACE = -4
HBF_EUNSORTED = -5
HBF_ERANGE_TIME = -6
HBF_EHIP = -7
HBF_ENOMEM = -8
HBF_EINTERNAL = -9
HBF_TIME_ERROR = -(1 << 63)
HBF_FLAG_PLANE_PARALLEL = 1
HBF_FLAG_REGISTER_BLOCKING = 2
HBF_FLAG_VMEM_CURVE = 4

EXPORTED = [
    "hbf_model_create", "hbf_model_destroy", "hbf_xfer_ns", "hbf_n_die_queues", "hbf_model_reset",
    "hbf_register_range", "hbf_workspace_bytes", "hbf_set_workspace", "hbf_classify_map",
    "hbf_time_requests", "hbf_time_layers", "hbf_gemv_instrumented", "hbf_wall_clock_tick_ps", "hbf_get_status",
    "hbf_get_state", "hbf_set_state", "hbf_profile", "hbf_kernel_times", "hbf_strerror",
    "hbf_refresh_plan", "hbf_refresh_configure", "hbf_refresh_submit", "hbf_refresh_drain", "hbf_refresh_pending",
    "hbf_cache_create", "hbf_cache_destroy", "hbf_cache_reset", "hbf_cache_access", "hbf_cache_sweep",
    "hbf_cache_set_chunk", "hbf_cache_get_chunk",
    "hbf_time_requests_noalloc", "hbf_vmem_configure",
    "hbf_kv_workspace_bytes", "hbf_kv_extend", "hbf_kv_fork", "hbf_kv_free", "hbf_kv_copy", "hbf_kv_compact",
    "hbf_kv_write", "hbf_kv_get_status", "hbf_kv_attention_workspace_bytes", "hbf_kv_attention",
    "hbf_moe_workspace_bytes", "hbf_moe_layer",
    "hbf_kv_write_rotated", "hbf_kv_chunk_workspace_bytes", "hbf_kv_chunk_attention", "hbf_kv_evict",
]
HBF_NOALLOC_SCRATCH_BYTES = 64 << 20
REFRESH_PENDING = -1
HBF_BF16 = 0
HBF_FP16 = 1
HBF_MOE_RENORM = 1
HBF_ROT_PAIRS = 1
HBF_CHUNK_CTL_WORDS = 2048


class hbf_params(ctypes.Structure):
    _fields_ = [("channels", ctypes.c_uint32), ("dies_per_channel", ctypes.c_uint32),
                ("planes_per_die", ctypes.c_uint32), ("page_bytes", ctypes.c_uint32),
                ("t_read_ns", ctypes.c_int64), ("channel_bytes_per_s", ctypes.c_uint64),
                ("flags", ctypes.c_uint32)]


class hbf_refresh_block(ctypes.Structure):
    _fields_ = [("epoch", ctypes.c_uint32), ("zone", ctypes.c_uint32), ("channel", ctypes.c_uint32),
                ("die", ctypes.c_uint32), ("plane", ctypes.c_uint32), ("block", ctypes.c_uint32)]


class hbf_kv(ctypes.Structure):
    _fields_ = [("dev_pool", ctypes.c_void_p), ("plane_stride", ctypes.c_uint64), ("page_stride", ctypes.c_uint64),
                ("token_bytes", ctypes.c_uint64), ("planes", ctypes.c_int32), ("pages", ctypes.c_int32),
                ("page_tokens", ctypes.c_int32), ("slots", ctypes.c_int32), ("table_cols", ctypes.c_int32),
                ("table_stride", ctypes.c_int64), ("dev_refs", ctypes.c_void_p), ("dev_tables", ctypes.c_void_p),
                ("dev_lens", ctypes.c_void_p), ("dev_ws", ctypes.c_void_p)]


class hbf_kv_layer(ctypes.Structure):
    _fields_ = [("dev_k", ctypes.c_void_p), ("dev_v", ctypes.c_void_p), ("page_stride", ctypes.c_int64),
                ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("pages", ctypes.c_int32),
                ("page_tokens", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_uint32)]


class hbf_attention(ctypes.Structure):
    _fields_ = [("dev_q", ctypes.c_void_p), ("q_row_stride", ctypes.c_int64), ("q_head_stride", ctypes.c_int64),
                ("rows", ctypes.c_int32), ("heads", ctypes.c_int32), ("scale", ctypes.c_float),
                ("dev_prefix_pages", ctypes.c_void_p), ("prefix_len", ctypes.c_int64),
                ("dev_tables", ctypes.c_void_p), ("table_stride", ctypes.c_int64),
                ("dev_own_len", ctypes.c_void_p), ("max_own", ctypes.c_int32), ("dev_out", ctypes.c_void_p),
                ("out_row_stride", ctypes.c_int64), ("out_head_stride", ctypes.c_int64),
                ("dev_lse", ctypes.c_void_p), ("dev_ctl", ctypes.c_void_p)]


_pack_attention = struct.Struct("@PqqiifPqPqPiPqqPP").pack_into   # its fields, in order


class hbf_new_tokens(ctypes.Structure):
    _fields_ = [("dev_q", ctypes.c_void_p), ("dev_k", ctypes.c_void_p), ("dev_v", ctypes.c_void_p),
                ("q_row_stride", ctypes.c_int64), ("q_head_stride", ctypes.c_int64), ("k_row_stride", ctypes.c_int64),
                ("k_head_stride", ctypes.c_int64), ("v_row_stride", ctypes.c_int64), ("v_head_stride", ctypes.c_int64),
                ("dev_q_out", ctypes.c_void_p), ("out_row_stride", ctypes.c_int64), ("out_head_stride", ctypes.c_int64),
                ("n", ctypes.c_int32), ("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_uint32), ("flags", ctypes.c_uint32),
                ("dev_q_weight", ctypes.c_void_p), ("dev_k_weight", ctypes.c_void_p), ("eps", ctypes.c_float),
                ("pairs", ctypes.c_int32), ("dev_freqs", ctypes.c_void_p), ("dev_slots", ctypes.c_void_p),
                ("dev_pos", ctypes.c_void_p), ("dev_positions", ctypes.c_void_p)]


_pack_new_tokens = struct.Struct("@PPPqqqqqqPqqiiiiIIPPfiPPPP").pack_into


class hbf_chunk(ctypes.Structure):
    _fields_ = [("dev_q", ctypes.c_void_p), ("q_row_stride", ctypes.c_int64), ("q_head_stride", ctypes.c_int64),
                ("tokens", ctypes.c_int32), ("rows", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("scale", ctypes.c_float), ("dev_slots", ctypes.c_void_p), ("dev_starts", ctypes.c_void_p),
                ("window", ctypes.c_int32), ("sinks", ctypes.c_int32), ("dev_out", ctypes.c_void_p),
                ("out_row_stride", ctypes.c_int64), ("out_head_stride", ctypes.c_int64), ("dev_lse", ctypes.c_void_p),
                ("dev_weights", ctypes.c_void_p), ("weights_slot_stride", ctypes.c_int64),
                ("weights_head_stride", ctypes.c_int64), ("weights_tokens", ctypes.c_int32), ("dev_ctl", ctypes.c_void_p)]


_pack_chunk = struct.Struct("@PqqiiifPPiiPqqPPqqiP").pack_into


class hbf_eviction(ctypes.Structure):
    _fields_ = [("dev_slots", ctypes.c_void_p), ("dev_keep", ctypes.c_void_p), ("n", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("sinks", ctypes.c_int32), ("recent", ctypes.c_int32),
                ("dev_weights", ctypes.c_void_p), ("layer_stride", ctypes.c_int64), ("slot_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64), ("weights_tokens", ctypes.c_int32),
                ("dev_weights_out", ctypes.c_void_p), ("dev_kept", ctypes.c_void_p), ("max_keep", ctypes.c_int32)]


class hbf_moe(ctypes.Structure):
    _fields_ = [("experts", ctypes.c_int32), ("topk", ctypes.c_int32), ("hidden", ctypes.c_int32),
                ("ffn", ctypes.c_int32), ("dtype", ctypes.c_uint32), ("flags", ctypes.c_uint32),
                ("dev_router", ctypes.c_void_p), ("dev_gate_up", ctypes.c_void_p), ("dev_down", ctypes.c_void_p),
                ("gate_up_stride", ctypes.c_int64), ("down_stride", ctypes.c_int64)]


_lib = None


def load_library(path=LIB_PATH):
    """Load libhbf.so and declare every exported signature."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"libhbf.so not built at {path}; run `python -m paper_2609_09800_amd.build`")
    lib = ctypes.CDLL(path)
    vp, i64, u64, i32, u32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_uint64, ctypes.c_int, ctypes.c_uint32
    sig = {
        "hbf_model_create": ([ctypes.POINTER(hbf_params), ctypes.POINTER(vp)], i32),
        "hbf_model_destroy": ([vp], None),
        "hbf_xfer_ns": ([vp, ctypes.POINTER(i64)], i32),
        "hbf_n_die_queues": ([vp, ctypes.POINTER(u32)], i32),
        "hbf_model_reset": ([vp, vp], i32),
        "hbf_register_range": ([vp, u64, u64, ctypes.POINTER(ctypes.c_int32)], i32),
        "hbf_workspace_bytes": ([vp, i64, ctypes.POINTER(ctypes.c_size_t)], i32),
        "hbf_set_workspace": ([vp, vp, ctypes.c_size_t], i32),
        "hbf_classify_map": ([vp, vp, i64, vp, vp], i32),
        "hbf_time_requests": ([vp, vp, vp, i64, vp, vp], i32),
        "hbf_time_requests_noalloc": ([vp, vp, vp, i64, vp, vp], i32),
        "hbf_vmem_configure": ([vp, vp], i32),
        "hbf_gemv_instrumented": ([vp, vp, i32, i32, i32, vp, i32, vp, vp, vp, vp, vp], i32),
        "hbf_wall_clock_tick_ps": ([vp, ctypes.POINTER(i64)], i32),
        "hbf_get_status": ([vp, vp], i32),
        "hbf_get_state": ([vp, vp, vp, vp], i32),
        "hbf_set_state": ([vp, vp, vp, vp], i32),
        "hbf_profile": ([vp, i32], i32),
        "hbf_kernel_times": ([vp, vp, vp, i32, ctypes.POINTER(i32)], i32),
        "hbf_time_layers": ([vp, vp, i64, vp, i32, i64, i64, vp, vp, vp, vp], i32),
        "hbf_strerror": ([i32], ctypes.c_char_p),
        "hbf_refresh_plan": ([ctypes.POINTER(hbf_params), vp, i64, u32, vp, i64], i32),
        "hbf_refresh_configure": ([vp, i64], i32),
        "hbf_refresh_submit": ([vp, vp, i64, vp, vp], i32),
        "hbf_refresh_drain": ([vp, i64, i64, vp], i32),
        "hbf_refresh_pending": ([vp, vp, vp], i32),
        "hbf_cache_create": ([u32, u32, u64, ctypes.POINTER(vp)], i32),
        "hbf_cache_destroy": ([vp], None),
        "hbf_cache_reset": ([vp, vp], i32),
        "hbf_cache_access": ([vp, vp, i64, vp, vp, vp, i64, vp, vp], i32),
        "hbf_cache_sweep": ([vp, vp, i32, u64, vp, i64, vp, vp], i32),
        "hbf_cache_set_chunk": ([vp, u32], i32),
        "hbf_cache_get_chunk": ([vp, ctypes.POINTER(u32)], i32),
        "hbf_kv_workspace_bytes": ([ctypes.POINTER(hbf_kv), i32, ctypes.POINTER(ctypes.c_size_t)], i32),
        "hbf_kv_extend": ([ctypes.POINTER(hbf_kv), vp, vp, i32, i32, vp], i32),
        "hbf_kv_fork": ([ctypes.POINTER(hbf_kv), vp, vp, i32, i32, vp], i32),
        "hbf_kv_free": ([ctypes.POINTER(hbf_kv), vp, i32, vp], i32),
        "hbf_kv_copy": ([ctypes.POINTER(hbf_kv), vp, vp, i32, vp], i32),
        "hbf_kv_compact": ([ctypes.POINTER(hbf_kv), vp, vp, vp, vp], i32),
        "hbf_kv_write": ([ctypes.POINTER(hbf_kv), i32, i32, vp, vp, vp, vp, i32, vp], i32),
        "hbf_kv_get_status": ([ctypes.POINTER(hbf_kv), vp], i32),
        "hbf_kv_attention_workspace_bytes": ([ctypes.POINTER(hbf_kv_layer), ctypes.POINTER(hbf_attention),
                                              ctypes.POINTER(ctypes.c_size_t)], i32),
        "hbf_kv_attention": ([ctypes.POINTER(hbf_kv_layer), ctypes.POINTER(hbf_attention), vp, vp, ctypes.c_size_t,
                              vp], i32),
        "hbf_kv_write_rotated": ([ctypes.POINTER(hbf_kv), i32, ctypes.POINTER(hbf_new_tokens), vp], i32),
        "hbf_kv_chunk_workspace_bytes": ([ctypes.POINTER(hbf_kv), ctypes.POINTER(hbf_kv_layer),
                                          ctypes.POINTER(hbf_chunk), ctypes.POINTER(ctypes.c_size_t)], i32),
        "hbf_kv_chunk_attention": ([ctypes.POINTER(hbf_kv), ctypes.POINTER(hbf_kv_layer), ctypes.POINTER(hbf_chunk),
                                    vp, vp, ctypes.c_size_t, vp], i32),
        "hbf_kv_evict": ([ctypes.POINTER(hbf_kv), ctypes.POINTER(hbf_eviction), vp], i32),
        "hbf_moe_workspace_bytes": ([ctypes.POINTER(hbf_moe), i32, ctypes.POINTER(ctypes.c_size_t)], i32),
        "hbf_moe_layer": ([ctypes.POINTER(hbf_moe), vp, i64, i32, vp, vp, vp, i64, vp, vp, ctypes.c_size_t, vp],
                          i32),
    }
    for name, (args, res) in sig.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = res
    _lib = lib
    return lib


def _dp(t):
    """Device pointer of a torch tensor (or None)."""
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _sp(stream):
    """hipStream_t of a torch stream (None -> current stream)."""
    if stream is None:
        import torch
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


class HbfError(RuntimeError):
    def __init__(self, code, what):
        lib = load_library()
        super().__init__(f"{what}: {lib.hbf_strerror(code).decode()} ({code})")
        self.code = code


def _check(code, what):
    if code != HBF_OK:
        raise HbfError(code, what)
    return code


def _dev(t, what, dtypes, numel=None, shape=None, at_least=False):
    """Fail-closed argument check (Section D1) before any pointer reaches the
    library, which cannot see array lengths: `t` must be a contiguous tensor
    on the GPU with one of `dtypes` (names) and, when given, exactly `numel`
    elements (at least that many with at_least) or exactly `shape`.  Raises
    HbfError(HBF_EINVAL) otherwise."""
    import torch
    bad = None
    if not isinstance(t, torch.Tensor):
        bad = f"not a tensor ({type(t).__name__})"
    elif not t.is_cuda:
        bad = "not in GPU memory"
    elif str(t.dtype).replace("torch.", "") not in dtypes:
        bad = f"dtype {t.dtype}, expected {'/'.join(dtypes)}"
    elif not t.is_contiguous():
        bad = "not contiguous"
    elif shape is not None and tuple(t.shape) != tuple(shape):
        bad = f"shape {tuple(t.shape)}, expected {tuple(shape)}"
    elif numel is not None and (t.numel() < numel if at_least else t.numel() != numel):
        bad = f"{t.numel()} elements, expected {'at least ' if at_least else ''}{numel}"
    if bad is not None:
        raise HbfError(HBF_EINVAL, f"{what}: {bad}")
    return t


_W64 = ("int64", "uint64")   # 8-byte words (addresses are uint64 bit patterns)
_I64 = ("int64",)


class Model:
    """An HBF device model on the current GPU (owns one C handle)."""

    def __init__(self, channels, dies_per_channel, planes_per_die, page_bytes, t_read_ns,
                 channel_bytes_per_s, flags=0):
        self._lib = load_library()
        self.params = hbf_params(channels, dies_per_channel, planes_per_die, page_bytes, t_read_ns,
                                 channel_bytes_per_s, flags)
        h = ctypes.c_void_p()
        _check(self._lib.hbf_model_create(ctypes.byref(self.params), ctypes.byref(h)), "hbf_model_create")
        self._h = h

    @classmethod
    def from_dict(cls, d):
        return cls(**d)

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            self._lib.hbf_model_destroy(self._h)
        self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def handle(self):
        return self._h

    @property
    def xfer_ns(self):
        x = ctypes.c_int64()
        _check(self._lib.hbf_xfer_ns(self._h, ctypes.byref(x)), "hbf_xfer_ns")
        return x.value

    @property
    def n_die_queues(self):
        x = ctypes.c_uint32()
        _check(self._lib.hbf_n_die_queues(self._h, ctypes.byref(x)), "hbf_n_die_queues")
        return x.value

    def register_range(self, base, nbytes):
        rid = ctypes.c_int32(-1)
        rc = self._lib.hbf_register_range(self._h, base, nbytes, ctypes.byref(rid))
        return rc, rid.value

    def reset(self, stream=None):
        _check(self._lib.hbf_model_reset(self._h, _sp(stream)), "hbf_model_reset")

    def workspace_bytes(self, n):
        b = ctypes.c_size_t()
        _check(self._lib.hbf_workspace_bytes(self._h, n, ctypes.byref(b)), "hbf_workspace_bytes")
        return b.value

    def set_workspace(self, tensor):
        if tensor is None:
            return self._lib.hbf_set_workspace(self._h, None, 0)
        _dev(tensor, "workspace", ("uint8", "int8", "int16", "int32", "int64", "float32"))
        return self._lib.hbf_set_workspace(self._h, _dp(tensor), tensor.numel() * tensor.element_size())

    def classify_map(self, addr, out, stream=None):
        """addr: uint64-valued int64 tensor [n] (device); out: int64 tensor [n]."""
        _dev(addr, "addr", _W64)
        _dev(out, "map_out", _W64, numel=addr.numel())
        return self._lib.hbf_classify_map(self._h, _dp(addr), addr.numel(), _dp(out), _sp(stream))

    def time_requests(self, addr, issue, complete, stream=None):
        """addr/issue/complete: int64 device tensors [n] (addr holds uint64 bit patterns)."""
        n = _dev(addr, "addr", _W64).numel()
        _dev(issue, "issue_ns", _I64, numel=n)
        _dev(complete, "complete_ns", _I64, numel=n)
        return self._lib.hbf_time_requests(self._h, _dp(addr), _dp(issue), n, _dp(complete), _sp(stream))

    def time_requests_noalloc(self, addr, issue, complete, stream=None):
        """hbf_time_requests through the entry point that allocates nothing
        (static per-GPU scratch of HBF_NOALLOC_SCRATCH_BYTES; calls on one GPU
        must not overlap)."""
        n = _dev(addr, "addr", _W64).numel()
        _dev(issue, "issue_ns", _I64, numel=n)
        _dev(complete, "complete_ns", _I64, numel=n)
        return self._lib.hbf_time_requests_noalloc(self._h, _dp(addr), _dp(issue), n, _dp(complete),
                                                   _sp(stream))

    def time_layers(self, addr, layer_start, t_start_ns, compute_ns, issue, complete, layer_done, stream=None):
        """Closed-loop layers.  addr/issue/complete: int64 device tensors [n];
        layer_start: host int64 array [L+1]; layer_done: int64 device tensor [L]."""
        import numpy as np
        ls = np.ascontiguousarray(layer_start, dtype=np.int64)
        L = ls.size - 1
        n = _dev(addr, "addr", _W64).numel()
        _dev(issue, "issue_ns", _I64, numel=n)
        _dev(complete, "complete_ns", _I64, numel=n)
        _dev(layer_done, "layer_done_ns", _I64, numel=max(L, 0), at_least=True)
        if ls.ndim != 1 or L < 0:
            raise HbfError(HBF_EINVAL, "layer_start: one-dimensional, at least one entry")
        return self._lib.hbf_time_layers(self._h, _dp(addr), n, ls.ctypes.data_as(ctypes.c_void_p), L,
                                         t_start_ns, compute_ns, _dp(issue), _dp(complete), _dp(layer_done),
                                         _sp(stream))

    def gemv_instrumented(self, W, X, Y, page_issue=None, page_complete=None, measured=None, stream=None):
        """W: int16 [E,N,K] (bf16 bits); X: int16 [E,B,K]; Y: float32 [E,B,N];
        page_issue / page_complete (both or neither) and measured: int64
        [E*N*K*2 / page_bytes], one entry per weight page."""
        _dev(W, "W", ("int16", "uint16", "bfloat16"))
        if W.dim() != 3:
            raise HbfError(HBF_EINVAL, f"W: shape {tuple(W.shape)}, expected [E, N, K]")
        E, N, K = W.shape
        _dev(X, "X", ("int16", "uint16", "bfloat16"))
        if X.dim() != 3 or X.shape[0] != E or X.shape[2] != K:
            raise HbfError(HBF_EINVAL, f"X: shape {tuple(X.shape)}, expected [{E}, B, {K}]")
        B = X.shape[1]
        _dev(Y, "Y", ("float32",), shape=(E, B, N))
        if (page_issue is None) != (page_complete is None):
            raise HbfError(HBF_EINVAL, "page_issue and page_complete: both or neither")
        if measured is not None and page_issue is None:
            raise HbfError(HBF_EINVAL, "measured needs page_issue and page_complete")
        pages = E * N * K * 2 // self.params.page_bytes
        for t, nm in ((page_issue, "page_issue_ns"), (page_complete, "page_complete_ns"),
                      (measured, "measured_delay_ns")):
            if t is not None:
                _dev(t, nm, _I64, numel=pages)
        return self._lib.hbf_gemv_instrumented(self._h, _dp(W), E, K, N, _dp(X), B, _dp(Y), _dp(page_issue),
                                               _dp(page_complete), _dp(measured), _sp(stream))

    def wall_clock_tick_ps(self):
        x = ctypes.c_int64()
        _check(self._lib.hbf_wall_clock_tick_ps(self._h, ctypes.byref(x)), "hbf_wall_clock_tick_ps")
        return x.value

    def get_status(self, stream=None):
        return self._lib.hbf_get_status(self._h, _sp(stream))

    def get_state(self, stream=None):
        import numpy as np
        d = np.zeros(self.n_die_queues, dtype=np.int64)
        c = np.zeros(self.params.channels, dtype=np.int64)
        _check(self._lib.hbf_get_state(self._h, d.ctypes.data_as(ctypes.c_void_p),
                                       c.ctypes.data_as(ctypes.c_void_p), _sp(stream)), "hbf_get_state")
        return d, c

    def set_state(self, die_free, chan_free, stream=None):
        import numpy as np
        d = np.ascontiguousarray(die_free, dtype=np.int64)
        c = np.ascontiguousarray(chan_free, dtype=np.int64)
        return self._lib.hbf_set_state(self._h, d.ctypes.data_as(ctypes.c_void_p),
                                       c.ctypes.data_as(ctypes.c_void_p), _sp(stream))

    # -- the calibrated vmem curve (Section "Discussion"; reading in include/hbf.h)

    def vmem_configure(self, knots_ns):
        """T(1), T(4), T(16), T(64), T(256), T(512) in ns (HBF_FLAG_VMEM_CURVE models)."""
        import numpy as np
        k = np.ascontiguousarray(knots_ns, dtype=np.int64)
        if k.size != 6:
            raise HbfError(HBF_EINVAL, "vmem knots: six values")
        return self._lib.hbf_vmem_configure(self._h, k.ctypes.data_as(ctypes.c_void_p))

    # -- refresh traffic (Section D4; reading in include/hbf.h)

    def refresh_configure(self, t_prog_ns):
        return self._lib.hbf_refresh_configure(self._h, int(t_prog_ns))

    def refresh_submit(self, pages, done, stream=None):
        """pages: host uint64 array of device pages in plan order; done: int64
        device tensor [len(pages)] receiving each quantum's completion."""
        import numpy as np
        pg = np.ascontiguousarray(pages, dtype=np.uint64)
        if done is not None:
            _dev(done, "done_ns", _I64, numel=pg.size, at_least=True)
        return self._lib.hbf_refresh_submit(self._h, pg.ctypes.data_as(ctypes.c_void_p) if pg.size else None,
                                            pg.size, _dp(done), _sp(stream))

    def refresh_drain(self, t_from_ns, t_to_ns, stream=None):
        return self._lib.hbf_refresh_drain(self._h, int(t_from_ns), int(t_to_ns), _sp(stream))

    def refresh_pending(self, stream=None):
        import numpy as np
        out = np.zeros(self.n_die_queues, dtype=np.uint32)
        _check(self._lib.hbf_refresh_pending(self._h, out.ctypes.data_as(ctypes.c_void_p), _sp(stream)),
               "hbf_refresh_pending")
        return out

    def profile(self, enable=True):
        _check(self._lib.hbf_profile(self._h, int(enable)), "hbf_profile")

    def kernel_times(self):
        """[(kernel name, ms)] of the last hbf_time_requests call (profiling on)."""
        ms = (ctypes.c_float * 16)()
        names = (ctypes.c_char_p * 16)()
        cnt = ctypes.c_int(0)
        _check(self._lib.hbf_kernel_times(self._h, ms, names, 16, ctypes.byref(cnt)), "hbf_kernel_times")
        return [(names[i].decode(), ms[i]) for i in range(cnt.value)]


class Cache:
    """Capacity-mode frame cache with the next-page prefetcher on the current
    GPU (one C handle; reading in include/hbf.h)."""

    def __init__(self, frames, prefetch_pages, range_pages):
        self._lib = load_library()
        h = ctypes.c_void_p()
        _check(self._lib.hbf_cache_create(frames, prefetch_pages, range_pages, ctypes.byref(h)), "hbf_cache_create")
        self._h = h

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            self._lib.hbf_cache_destroy(self._h)
        self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def reset(self, stream=None):
        return self._lib.hbf_cache_reset(self._h, _sp(stream))

    def set_chunk(self, accesses):
        """Accesses served together (0 = one after another); see include/hbf.h."""
        _check(self._lib.hbf_cache_set_chunk(self._h, int(accesses)), "hbf_cache_set_chunk")

    def chunk(self):
        x = ctypes.c_uint32()
        _check(self._lib.hbf_cache_get_chunk(self._h, ctypes.byref(x)), "hbf_cache_get_chunk")
        return x.value

    def access(self, pages, hit, counts, pf_page=None, pf_src=None, stream=None):
        """pages: int64 device tensor [n] (page numbers); hit: uint8 [n];
        counts: int64 [8]; pf_page / pf_src: int64 [cap] or None."""
        n = _dev(pages, "pages", _W64).numel()
        _dev(hit, "hit", ("uint8",), numel=n, at_least=True)
        _dev(counts, "counts", _I64, numel=8, at_least=True)
        if (pf_page is None) != (pf_src is None):
            raise HbfError(HBF_EINVAL, "pf_page and pf_src: both or neither")
        cap = 0 if pf_page is None else pf_page.numel()
        if pf_page is not None:
            _dev(pf_page, "pf_page", _W64)
            _dev(pf_src, "pf_src", _I64, numel=cap)
        return self._lib.hbf_cache_access(self._h, _dp(pages), pages.numel(), _dp(hit), _dp(pf_page), _dp(pf_src),
                                          cap, _dp(counts), _sp(stream))


def cache_sweep(frames, prefetch, range_pages, pages, counts, stream=None):
    """Many fresh caches over one stream: frames / prefetch host int lists,
    pages int64 device tensor, counts int64 device tensor [len(frames), 5]."""
    import numpy as np
    lib = load_library()
    f = np.ascontiguousarray(frames, dtype=np.uint32)
    d = np.ascontiguousarray(prefetch, dtype=np.uint32)
    if f.size != d.size:
        raise HbfError(HBF_EINVAL, "frames and prefetch: one entry per cache each")
    _dev(pages, "pages", _W64)
    _dev(counts, "counts", _I64, numel=5 * f.size, at_least=True)
    return lib.hbf_cache_sweep(f.ctypes.data_as(ctypes.c_void_p), d.ctypes.data_as(ctypes.c_void_p), f.size,
                               range_pages, _dp(pages), pages.numel(), _dp(counts), _sp(stream))


_I32 = ("int32",)
_HALF = ("bfloat16", "float16")
torch = None   # the module, once a KvPages or MoeLayer is made: their calls last about 10 us, an import statement 0.2


def _import_torch():
    global torch, _Tensor, _int32, _raw_stream, _device
    import torch
    _Tensor, _int32 = torch.Tensor, torch.int32
    _raw_stream, _device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
    return load_library()


def _raw(stream):
    """hipStream_t of a torch stream (None -> current stream), as a number.
    (torch.cuda.current_stream() builds an object, which takes 2.8 us.)"""
    return _raw_stream(_device()) if stream is None else stream.cuda_stream


def _is(t, dtype):
    """A contiguous tensor of that type on the GPU: what most calls pass."""
    return isinstance(t, _Tensor) and t.is_cuda and t.dtype is dtype and t.is_contiguous()


def _ints(t, what, numel=None):
    """_dev for an int32 tensor; its number of elements."""
    if isinstance(t, _Tensor) and t.is_cuda and t.dtype is _int32 and t.is_contiguous():
        n = t.numel()
        if numel is None or n == numel:
            return n
    _dev(t, what, _I32, numel=numel)
    return t.numel()


def _strided(t, what, dtypes, dim, inner=1):
    """As _dev, for a tensor of `dim` dimensions whose last `inner` are
    contiguous and whose others may be strided (by 16-byte multiples)."""
    bad = None
    if not isinstance(t, torch.Tensor):
        bad = f"not a tensor ({type(t).__name__})"
    elif not t.is_cuda:
        bad = "not in GPU memory"
    elif t.dtype not in dtypes:
        bad = f"dtype {t.dtype}, expected {'/'.join(map(str, dtypes))}"
    elif t.dim() != dim:
        bad = f"{t.dim()} dimensions, expected {dim}"
    elif not t.is_contiguous() or dim > inner and t.shape[-1] * t.element_size() % 16:
        want = 1
        for d in range(dim - 1, dim - 1 - inner, -1):
            if t.shape[d] != 1 and t.stride(d) != want:
                bad = f"strides {tuple(t.stride())}: the last {inner} dimension(s) must be contiguous"
            want *= t.shape[d]
        if any(t.stride(d) * t.element_size() % 16 for d in range(dim - inner) if t.shape[d] > 1):
            bad = f"strides {tuple(t.stride())}: not multiples of 16 bytes"
    if bad is not None:
        raise HbfError(HBF_EINVAL, f"{what}: {bad}")
    return t


def _heads(t, dtype):
    """[rows, heads, head_dim] as a kernel takes it, the strides of two dimensions in elements of 2 bytes (_strided says what is wrong)."""
    if isinstance(t, _Tensor) and t.is_cuda and t.dtype is dtype and t.dim() == 3:
        rows, heads, inner = t.stride()
        return inner == 1 and not (rows | heads) & 7
    return False


def _writable(t, what):
    """An output whose elements must not share memory (an expanded tensor's do)."""
    if not t.is_contiguous() and any(t.stride(d) == 0 and t.shape[d] > 1 for d in range(t.dim())):
        raise HbfError(HBF_EINVAL, f"{what}: an expanded tensor cannot be written")
    return t


def _same_layout(t, like):
    return getattr(t, "is_cuda", False) and t.dtype == like.dtype and t.shape == like.shape and t.stride() == like.stride()


class _Blocks:
    """Device blocks of one object, and the streams that its calls used them
    on: the allocator gives them away only once those are through with them."""

    def __init__(self, *blocks):
        self._blocks = blocks
        self._on = {_raw(None)}   # the allocator knows the stream that they were made on

    def use(self, raw, stream):
        """A call on `stream` (None: the current one), whose number is `raw`, gets them."""
        if raw not in self._on:
            for t in self._blocks:
                t.record_stream(stream if stream is not None else torch.cuda.current_stream())
            self._on.add(raw)


class _Scratch:
    """Device scratch that grows with the calls' needs.  What it grew out of
    stays as long as the object: a captured graph may write to it whenever it is
    replayed.  Each block is at least twice the one before, so that what is kept
    is less than the last."""

    def __init__(self):
        self._t = self._use = None
        self._kept = []

    def get(self, nbytes, device, stream):
        if self._t is None or self._t.numel() < nbytes:
            least = 256
            if self._t is not None:
                self._kept.append(self._t)
                least = 2 * self._t.numel()
            # made on the call's stream: what was freed on another one may still be in use there
            with torch.cuda.stream(stream):
                self._t = torch.empty(max(nbytes, least), dtype=torch.uint8, device=device)
                self._use = _Blocks(self._t)
        self._use.use(_raw(stream), stream)
        return self._t


def _stride(t, d):
    """Stride of a dimension in elements; of one of a single entry, which is never taken, 0."""
    return t.stride(d) if t.shape[d] > 1 else 0


def _zeroed(nbytes, device, zero=256):
    """Device bytes, the first `zero` zero and seen so by every stream."""
    t = torch.empty(max(nbytes, zero), dtype=torch.uint8, device=device)
    t[:zero].zero_()
    torch.cuda.current_stream(device).synchronize()
    return t


def _take_status(word, blocks, stream):
    """A status word of those blocks, read and cleared in the order of `stream`
    (None: the current one), so that a later call's error is not cleared with it."""
    blocks.use(_raw(stream), stream)
    with torch.cuda.stream(stream):
        rc = int(word.item())
        if rc != HBF_OK:
            word.zero_()
    return rc


def _dtype_code(t):
    import torch
    return HBF_BF16 if t.dtype == torch.bfloat16 else HBF_FP16


class KvPages:
    """A KV cache of pages on the current GPU (reading in include/hbf.h).

    pool: bfloat16 or float16 [layers, 2, pages, page_tokens, kv_heads,
    head_dim], contiguous; index 0 of the second dimension is K, 1 is V.
    refs: int32 [pages]; tables: int32 [slots, entries] (rows may be strided);
    lens: int32 [slots].  All stay the caller's; a cache that only
    prefix_attention reads needs the pool alone.  max_list: the longest list
    that extend and fork will be given.  Calls on one object must be ordered
    on one stream, replays of captured ones among them, and the object must
    live as long as a graph that captured its calls."""

    def __init__(self, pool, refs=None, tables=None, lens=None, max_list=1024):
        self._lib = _import_torch()
        _dev(pool, "pool", _HALF)
        if pool.dim() != 6 or pool.shape[1] != 2 or 0 in pool.shape:
            raise HbfError(HBF_EINVAL, f"pool: shape {tuple(pool.shape)}, expected "
                                       "[layers, 2, pages, page_tokens, kv_heads, head_dim]")
        self.pool, self.refs, self.tables, self.lens = pool, refs, tables, lens
        self.layers, _, self.pages, self.page_tokens, self.kv_heads, self.head_dim = pool.shape
        self._attn_ws = _Scratch()
        self._attn_sizes, self._attn_bytes, self._layers = None, 0, {}
        self._chunk_sizes, self._chunk_bytes = None, 0
        nbytes = 512 + 4 * HBF_CHUNK_CTL_WORDS
        words = _zeroed(nbytes, pool.device, nbytes).view(torch.int32)
        self._attn_status, self._attn_ctl, self._chunk_ctl = words[:1], words[64:], words[128:]
        self._attn_args, self._chunk_args, self._new_args = hbf_attention(), hbf_chunk(), hbf_new_tokens()
        self._attn_at = (self._attn_status.data_ptr(), self._attn_ctl.data_ptr())
        self._chunk_at = self._chunk_ctl.data_ptr()
        self._attn_words = _Blocks(words)
        self._kv = None
        if refs is None and tables is None and lens is None:
            return
        _dev(refs, "refs", _I32, shape=(self.pages,))
        if not isinstance(tables, torch.Tensor) or not tables.is_cuda or tables.dtype != torch.int32 \
                or tables.dim() != 2 or 0 in tables.shape or (tables.shape[1] > 1 and tables.stride(1) != 1) \
                or (tables.shape[0] > 1 and tables.stride(0) < tables.shape[1]):
            raise HbfError(HBF_EINVAL, "tables: expected int32 [slots, entries] in GPU memory, rows contiguous")
        _dev(lens, "lens", _I32, shape=(tables.shape[0],))
        tok = self.kv_heads * self.head_dim * 2
        self.max_list = int(max_list)
        self._kv = hbf_kv(pool.data_ptr(), tok * self.page_tokens * self.pages, tok * self.page_tokens, tok,
                          self.layers * 2, self.pages, self.page_tokens, tables.shape[0], tables.shape[1],
                          max(tables.stride(0), tables.shape[1]), refs.data_ptr(), tables.data_ptr(),
                          lens.data_ptr(), None)
        b = ctypes.c_size_t()
        _check(self._lib.hbf_kv_workspace_bytes(ctypes.byref(self._kv), self.max_list, ctypes.byref(b)),
               "hbf_kv_workspace_bytes")
        self._ws = _zeroed(b.value, pool.device)
        self._kv.dev_ws = self._ws.data_ptr()
        self._kv_ref = ctypes.byref(self._kv)
        self._kv_blocks = _Blocks(self._ws)

    def _desc(self):
        if self._kv is None:
            raise HbfError(HBF_EINVAL, "this KvPages was made without refs, tables and lens")
        return self._kv_ref

    def _on(self, stream):
        """A checked call's stream, as a number; the workspace is used on it."""
        raw = _raw(stream)
        self._kv_blocks.use(raw, stream)
        return raw

    def extend(self, slots, add, stream=None):
        """Slot slots[i] grows by add[i] tokens (int32 device tensors [n])."""
        d = self._desc()
        n = _ints(slots, "slots")
        _ints(add, "add", n)
        return self._lib.hbf_kv_extend(d, slots.data_ptr(), add.data_ptr(), n, self.max_list, self._on(stream))

    def fork(self, parents, children, stream=None):
        """The empty slot children[i] gets parents[i]'s tokens (int32 [n])."""
        d = self._desc()
        n = _ints(parents, "parents")
        _ints(children, "children", n)
        return self._lib.hbf_kv_fork(d, parents.data_ptr(), children.data_ptr(), n, self.max_list, self._on(stream))

    def free(self, slots, stream=None):
        """Slots (int32 [n]) become empty and give their pages back."""
        d = self._desc()
        n = _ints(slots, "slots")
        return self._lib.hbf_kv_free(d, slots.data_ptr(), n, self._on(stream))

    def copy(self, src, dst, stream=None):
        """Pages dst[i] become copies of pages src[i] (int32 [n])."""
        d = self._desc()
        n = _ints(src, "src")
        _ints(dst, "dst", n)
        return self._lib.hbf_kv_copy(d, src.data_ptr(), dst.data_ptr(), n, self._on(stream))

    def compact(self, remap, tables_out=None, refs_out=None, stream=None):
        """Pages in use move to the front.  remap: int32 [pages]; tables_out
        (shaped and strided as tables) and refs_out: None for in place."""
        d = self._desc()
        _ints(remap, "remap", self.pages)
        if refs_out is not None:
            _ints(refs_out, "refs_out", self.pages)
        if tables_out is not None and (not getattr(tables_out, "is_cuda", False)
                                       or tables_out.dtype != self.tables.dtype
                                       or tables_out.shape != self.tables.shape
                                       or tables_out.stride() != self.tables.stride()):
            raise HbfError(HBF_EINVAL, "tables_out: expected the shape, strides and type of tables")
        return self._lib.hbf_kv_compact(d, remap.data_ptr(), None if tables_out is None else tables_out.data_ptr(),
                                        None if refs_out is None else refs_out.data_ptr(), self._on(stream))

    def write(self, k, v, slots, pos, first_layer=0, stream=None):
        """Token pos[i] of slot slots[i] (int32 [n]) gets k[:, i] and v[:, i]:
        [layers, n, kv_heads, head_dim] of the pool's type, for the layers from
        first_layer on (or [n, kv_heads, head_dim] for that layer alone)."""
        d = self._desc()
        n = _ints(slots, "slots")
        _ints(pos, "pos", n)
        for t, what in ((k, "k"), (v, "v")):
            if not _is(t, self.pool.dtype):
                _dev(t, what, (str(self.pool.dtype).replace("torch.", ""),))
        shape = k.shape
        layers = shape[0] if len(shape) == 4 else 1
        if shape[-3:] != (n, self.kv_heads, self.head_dim) or len(shape) not in (3, 4) or v.shape != shape:
            raise HbfError(HBF_EINVAL, f"k, v: shapes {tuple(k.shape)}, {tuple(v.shape)}, expected "
                                       f"[layers, {n}, {self.kv_heads}, {self.head_dim}]")
        return self._lib.hbf_kv_write(d, int(first_layer), layers, k.data_ptr(), v.data_ptr(), slots.data_ptr(),
                                      pos.data_ptr(), n, self._on(stream))

    def get_status(self, stream=None):
        """Synchronises; HBF_OK, HBF_EINVAL or HBF_ENOMEM since the last call
        (the attention's status counts too)."""
        rc = HBF_OK
        if self._kv is not None:
            rc = self._lib.hbf_kv_get_status(self._desc(), _sp(stream))
        if rc == HBF_OK:
            rc = _take_status(self._attn_status, self._attn_words, stream)
        return rc

    def prefix_attention(self, layer, q, out, prefix_pages, prefix_len, tables=None, own_lens=None, lse=None,
                         scale=None, stream=None):
        """Attention of q [rows, heads, head_dim] (one token per row) over the
        first prefix_len tokens of the pages prefix_pages (int32; None without
        prefix), shared by all rows, and each row's own_lens[r] tokens of the
        pages tables[r] (int32 [rows, entries], rows may be strided; e.g. the
        columns behind the prefix of a cache's table).  Work is cut for rows
        that fill their columns: where the host knows that all of them are
        shorter, it should pass no more columns than the longest needs (a
        slice).  out: as q; lse: float32 [rows, heads] or None; scale:
        1 / sqrt(head_dim) if None."""
        dtype = self.pool.dtype
        if not 0 <= layer < self.layers:
            raise HbfError(HBF_EINVAL, f"layer {layer}, the pool has {self.layers}")
        if not _is(q, dtype) or q.dim() != 3:
            _strided(q, "q", (dtype,), 3)
        if not _is(out, dtype):
            _writable(_strided(out, "out", (dtype,), 3), "out")
        shape = q.shape
        rows, heads, dim = shape
        if dim != self.head_dim or out.shape != shape:
            raise HbfError(HBF_EINVAL, f"q, out: shapes {tuple(shape)}, {tuple(out.shape)}, expected "
                                       f"[rows, heads, {self.head_dim}]")
        if lse is not None and (not _is(lse, torch.float32) or lse.shape != shape[:2]):
            _dev(lse, "lse", ("float32",), shape=(rows, heads))
        prefix_len = int(prefix_len)
        if prefix_len > 0 and _ints(prefix_pages, "prefix_pages") * self.page_tokens < prefix_len:
            raise HbfError(HBF_EINVAL, f"prefix_pages: {prefix_pages.numel()} pages for {prefix_len} tokens")
        if (tables is None) != (own_lens is None):
            raise HbfError(HBF_EINVAL, "tables and own_lens: both or neither")
        max_own = stride = own = 0
        if tables is not None:
            if not _is(tables, torch.int32) or tables.dim() != 2 or tables.shape[0] != rows:
                if not isinstance(tables, torch.Tensor) or not tables.is_cuda or tables.dtype != torch.int32 \
                        or tables.dim() != 2 or tables.shape[0] != rows \
                        or (tables.shape[1] > 1 and tables.stride(1) != 1):
                    raise HbfError(HBF_EINVAL,
                                   f"tables: expected int32 [{rows}, entries] in GPU memory, rows contiguous")
            _ints(own_lens, "own_lens", rows)
            max_own, stride = min(tables.shape[1] * self.page_tokens, (1 << 31) - 1), _stride(tables, 0)
            own = own_lens.data_ptr()
        kv = self._layer(layer)
        qs, os = q.stride(), out.stride()   # (of a dimension of one entry: never taken, but it may be odd)
        at = self._attn_args   # (filled anew by each call, in a third of the time that making one takes)
        _pack_attention(at, 0, q.data_ptr(), qs[0] if rows > 1 else 0, qs[1] if heads > 1 else 0, rows, heads,
                        dim ** -0.5 if scale is None else scale,
                        prefix_pages.data_ptr() if prefix_len > 0 else 0, prefix_len,
                        tables.data_ptr() if max_own else 0, stride, own, max_own, out.data_ptr(),
                        os[0] if rows > 1 else 0, os[1] if heads > 1 else 0,
                        0 if lse is None else lse.data_ptr(), self._attn_at[1] or 0)
        sizes = (rows, heads, prefix_len, max_own)
        if sizes != self._attn_sizes:
            b = ctypes.c_size_t()
            rc = self._lib.hbf_kv_attention_workspace_bytes(kv, at, ctypes.byref(b))
            if rc != HBF_OK:
                return rc
            self._attn_sizes, self._attn_bytes = sizes, b.value
        ws = self._attn_ws.get(self._attn_bytes, self.pool.device, stream)
        raw = _raw(stream)
        self._attn_words.use(raw, stream)
        return self._lib.hbf_kv_attention(kv, at, self._attn_at[0], ws.data_ptr(), ws.numel(), raw)

    def write_rotated(self, layer, q, k, v, slots, pos, freqs, q_out, q_weight=None, k_weight=None, eps=1e-6,
                      positions=None, interleaved=False, stream=None):
        """New tokens of one layer enter the cache: q [n, heads, head_dim] is
        normed (with q_weight [head_dim]; None: not) and turned to q_out (which
        may be q), k [n, kv_heads, head_dim] likewise and v as it is go to token
        pos[i] of slot slots[i] (int32 [n]).  Rows and heads may be strided, as
        views of one projection's output are.  freqs: float64, radians per
        position of each pair that turns (a multiple of 8, up to head_dim / 2);
        pair i is the values i and i + len(freqs), interleaved: 2 i and 2 i + 1.
        positions: int32 [n], pos if None."""
        d = self._desc()
        dtype = self.pool.dtype
        if not 0 <= layer < self.layers:
            raise HbfError(HBF_EINVAL, f"layer {layer}, the pool has {self.layers}")
        n = _ints(slots, "slots")
        _ints(pos, "pos", n)
        if positions is not None:
            _ints(positions, "positions", n)
        for t, what in ((q, "q"), (k, "k"), (v, "v"), (q_out, "q_out")):
            if not _heads(t, dtype):
                _strided(t, what, (dtype,), 3)
        _writable(q_out, "q_out")
        heads, dim, kv_shape = q.shape[1], self.head_dim, (n, self.kv_heads, self.head_dim)
        if q.shape != (n, heads, dim) or q_out.shape != q.shape or k.shape != kv_shape or v.shape != kv_shape:
            raise HbfError(HBF_EINVAL, f"q, k, v, q_out: shapes {tuple(q.shape)}, {tuple(k.shape)}, {tuple(v.shape)}, "
                                       f"{tuple(q_out.shape)}, expected [{n}, heads, {dim}] and {list(kv_shape)}")
        for t, what in ((q_weight, "q_weight"), (k_weight, "k_weight")):
            if t is not None and (not _is(t, dtype) or t.shape != (dim,)):
                _dev(t, what, (str(dtype).replace("torch.", ""),), shape=(dim,))
        if not _is(freqs, torch.float64):
            _dev(freqs, "freqs", ("float64",))
        qs, ks, vs, os = q.stride(), k.stride(), v.stride(), q_out.stride()
        row = n > 1
        nt = self._new_args
        try:
            _pack_new_tokens(nt, 0, q.data_ptr(), k.data_ptr(), v.data_ptr(), qs[0] if row else 0,
                             qs[1] if heads > 1 else 0, ks[0] if row else 0, ks[1] if self.kv_heads > 1 else 0,
                             vs[0] if row else 0, vs[1] if self.kv_heads > 1 else 0, q_out.data_ptr(),
                             os[0] if row else 0, os[1] if heads > 1 else 0, n, heads, self.kv_heads, dim,
                             HBF_BF16 if dtype is torch.bfloat16 else HBF_FP16, HBF_ROT_PAIRS if interleaved else 0,
                             0 if q_weight is None else q_weight.data_ptr(), 0 if k_weight is None else k_weight.data_ptr(),
                             eps, freqs.numel(), freqs.data_ptr(), slots.data_ptr(), pos.data_ptr(),
                             0 if positions is None else positions.data_ptr())
        except (struct.error, OverflowError):
            raise HbfError(HBF_EINVAL, f"{n} tokens, {freqs.numel()} freqs, eps {eps}: expected what fits 32 bits") from None
        return self._lib.hbf_kv_write_rotated(d, layer, nt, self._on(stream))

    def attention(self, layer, q, out, slots, starts, lse=None, weights=None, scale=None, window=0, sinks=0,
                  stream=None):
        """Causal attention of new tokens over the cache.  Row i's queries are
        q[starts[i]:starts[i + 1]] (q: [tokens, heads, head_dim]; starts: int32
        [rows + 1], slots: int32 [rows]), the last tokens of slot slots[i], whose
        K and V are in the cache already: one per row in a decode step, more for
        a chunk of a prompt, also in one call.  window > 0: a query sees the
        last `window` tokens up to its own, and the first `sinks`.  out: as q
        (not q itself); lse: float32 [tokens, heads] or None; weights: float32
        [slots, kv_heads, tokens] (slots and heads may be strided) or None:
        each cached token's grows by the probabilities that the row's queries
        gave it.  What lies behind starts[rows] is left as it was.  The window
        counts places: after evict, one that reaches past the last `recent` and
        what came behind them sees whichever of the middle lie there.  With
        weights, the object's scratch may hold a float for each query of each
        head and each token that both a table's row and weights have room for,
        up to 512 MiB a call (and what it grew out of, less than that again):
        where sequences are known to be shorter, pass weights[..., :n], n at
        least the longest length."""
        d = self._desc()
        dtype = self.pool.dtype
        if not 0 <= layer < self.layers:
            raise HbfError(HBF_EINVAL, f"layer {layer}, the pool has {self.layers}")
        if not _heads(q, dtype):
            _strided(q, "q", (dtype,), 3)
        if not _heads(out, dtype):
            _strided(out, "out", (dtype,), 3)
        _writable(out, "out")
        shape = q.shape
        tokens, heads, dim = shape
        if dim != self.head_dim or out.shape != shape:
            raise HbfError(HBF_EINVAL, f"q, out: shapes {tuple(shape)}, {tuple(out.shape)}, expected "
                                       f"[tokens, heads, {self.head_dim}]")
        rows = _ints(slots, "slots")
        _ints(starts, "starts", rows + 1)
        if lse is not None and (not _is(lse, torch.float32) or lse.shape != shape[:2]):
            _dev(lse, "lse", ("float32",), shape=(tokens, heads))
        ws, held = (0, 0), 0
        if weights is not None:
            self._check_weights(weights, "weights", (self.tables.shape[0], self.kv_heads))
            ws, held = (_stride(weights, 0), _stride(weights, 1)), weights.shape[2]
        kv = self._layer(layer)
        qs, os = q.stride(), out.stride()
        at = self._chunk_args
        try:
            _pack_chunk(at, 0, q.data_ptr(), qs[0] if tokens > 1 else 0, qs[1] if heads > 1 else 0, tokens, rows, heads,
                        dim ** -0.5 if scale is None else scale, slots.data_ptr(), starts.data_ptr(), int(window),
                        int(sinks), out.data_ptr(), os[0] if tokens > 1 else 0, os[1] if heads > 1 else 0,
                        0 if lse is None else lse.data_ptr(), 0 if weights is None else self._address(weights), *ws,
                        min(held, (1 << 31) - 1), self._chunk_at or 0)
        except (struct.error, OverflowError):
            raise HbfError(HBF_EINVAL, f"{tokens} tokens, {rows} rows, window {window}, sinks {sinks}, scale {scale}: "
                                       "expected what fits 32 bits") from None
        sizes = (tokens, rows, heads, None if weights is None else held)
        if sizes != self._chunk_sizes:
            b = ctypes.c_size_t()
            rc = self._lib.hbf_kv_chunk_workspace_bytes(d, kv, at, ctypes.byref(b))
            if rc != HBF_OK:
                return rc
            self._chunk_sizes, self._chunk_bytes = sizes, b.value
        scratch = self._attn_ws.get(self._chunk_bytes, self.pool.device, stream)
        raw = _raw(stream)
        self._attn_words.use(raw, stream)
        return self._lib.hbf_kv_chunk_attention(d, kv, at, self._attn_at[0], scratch.data_ptr(), scratch.numel(), raw)

    def _check_weights(self, t, what, lead):
        """Accumulated weights: float32 [*lead, tokens], tokens contiguous."""
        if not isinstance(t, _Tensor) or not t.is_cuda or t.dtype is not torch.float32 \
                or tuple(t.shape[:-1]) != lead or (t.shape[-1] > 1 and t.stride(-1) != 1):
            raise HbfError(HBF_EINVAL, f"{what}: expected float32 {[*lead, 'tokens']} in GPU memory, tokens contiguous")
        _writable(t, what)

    def _address(self, weights):
        """Of weights that are given: those that hold no token have none of their own, and NULL says something else."""
        return weights.data_ptr() or self.lens.data_ptr()

    def evict(self, slots, keep, weights, kept, sinks=0, recent=0, weights_out=None, stream=None):
        """Slot slots[i] is cut down to keep[i] tokens (int32 [n]), in every
        layer and KV head its own: the first `sinks`, the last `recent`, and
        those of the largest weights between.  weights: float32 [layers, slots,
        kv_heads, tokens] (as attention's, for each layer; all but the tokens
        may be strided) follow their tokens, in place or to weights_out (shaped
        and strided alike, not overlapping).  kept: int32 [layers, n, kv_heads, max_keep],
        max_keep at least the largest keep, receives each place's token's old
        position, -1 behind them.  The middle is in no order afterwards, and
        attention's window counts places."""
        d = self._desc()
        n = _ints(slots, "slots")
        _ints(keep, "keep", n)
        self._check_weights(weights, "weights", (self.layers, self.tables.shape[0], self.kv_heads))
        if weights_out is not None and (not _same_layout(weights_out, weights)):
            raise HbfError(HBF_EINVAL, "weights_out: expected the shape, strides and type of weights")
        if not _is(kept, _int32) or kept.dim() != 4 or kept.shape[:3] != (self.layers, n, self.kv_heads):
            _dev(kept, "kept", _I32)
            raise HbfError(HBF_EINVAL, f"kept: shape {tuple(kept.shape)}, expected "
                                       f"[{self.layers}, {n}, {self.kv_heads}, max_keep]")
        sinks, recent, max_keep = int(sinks), int(recent), kept.shape[3]
        for value, what in ((n, "slots"), (sinks, "sinks"), (recent, "recent"), (max_keep, "max_keep")):
            if not -(1 << 31) <= value < 1 << 31:   # (ctypes would cut it)
                raise HbfError(HBF_EINVAL, f"{what} {value}: expected what fits 32 bits")
        ev = hbf_eviction(slots.data_ptr(), keep.data_ptr(), n, self.kv_heads, sinks, recent,
                          self._address(weights), _stride(weights, 0), _stride(weights, 1), _stride(weights, 2),
                          min(weights.shape[3], (1 << 31) - 1), None if weights_out is None else weights_out.data_ptr(),
                          kept.data_ptr(), max_keep)
        return self._lib.hbf_kv_evict(d, ev, self._on(stream))

    def _layer(self, layer):
        """The library's description of one layer's pages."""
        kv = self._layers.get(layer)
        if kv is None:
            tok = self.kv_heads * self.head_dim
            plane = self.pages * self.page_tokens * tok * 2
            base = self.pool.data_ptr() + 2 * layer * plane
            kv = self._layers[layer] = hbf_kv_layer(base, base + plane, self.page_tokens * tok, tok, self.head_dim,
                                                    self.pages, self.page_tokens, self.kv_heads, self.head_dim,
                                                    _dtype_code(self.pool))
        return kv


class MoeLayer:
    """A mixture-of-experts layer for a few tokens (reading in include/hbf.h).

    gate_up: [experts, 2 * ffn, hidden], gate rows then up rows; down:
    [experts, hidden, ffn]; the experts may be strided (both may be views of
    one buffer that holds expert after expert).  router: [experts, hidden], or
    None where the caller chooses.  max_tokens: the most tokens of a call (its
    scratch is allocated here; HBF_ENOWORKSPACE beyond).  All bfloat16 or all float16.  renormalize:
    the chosen experts' weights sum to 1.  Calls on one object must be
    ordered on one stream, replays of captured ones among them, and the object
    must live as long as a graph that captured its calls."""

    def __init__(self, gate_up, down, topk, router=None, renormalize=True, max_tokens=64):
        self._lib = _import_torch()
        _strided(gate_up, "gate_up", (torch.bfloat16, torch.float16), 3, 2)
        dtype = gate_up.dtype
        _strided(down, "down", (dtype,), 3, 2)
        E, F2, H = gate_up.shape
        if F2 % 2 or tuple(down.shape) != (E, H, F2 // 2):
            raise HbfError(HBF_EINVAL, f"gate_up, down: shapes {tuple(gate_up.shape)}, {tuple(down.shape)}, expected "
                                       "[experts, 2 * ffn, hidden], [experts, hidden, ffn]")
        if router is not None:
            _dev(router, "router", (str(gate_up.dtype).replace("torch.", ""),), shape=(E, H))
        self._keep = (gate_up, down, router)
        self._dtype, self.topk, self.hidden = dtype, int(topk), H
        self._m = hbf_moe(E, self.topk, H, F2 // 2, _dtype_code(gate_up), HBF_MOE_RENORM if renormalize else 0,
                          None if router is None else router.data_ptr(), gate_up.data_ptr(), down.data_ptr(),
                          _stride(gate_up, 0), _stride(down, 0))
        self._ws = _zeroed(self._bytes(max_tokens), gate_up.device)
        self._status = _zeroed(256, gate_up.device)[:4].view(torch.int32)
        self._blocks = _Blocks(self._ws, self._status)

    def _bytes(self, tokens):
        b = ctypes.c_size_t()
        _check(self._lib.hbf_moe_workspace_bytes(ctypes.byref(self._m), int(tokens), ctypes.byref(b)),
               "hbf_moe_workspace_bytes")
        return b.value

    def forward(self, x, y, ids, weights, stream=None):
        """x, y: [tokens, hidden] (rows may be strided); ids: int32 [tokens,
        topk], weights: float32 [tokens, topk]: outputs, or the caller's
        choices where the layer has no router (-1: none)."""
        dtype = self._dtype
        if not _is(x, dtype) or x.dim() != 2:
            _strided(x, "x", (dtype,), 2)
        if not _is(y, dtype):
            _writable(_strided(y, "y", (dtype,), 2), "y")
        T = x.shape[0]
        if x.shape[1] != self.hidden or y.shape != x.shape:
            raise HbfError(HBF_EINVAL, f"x, y: shapes {tuple(x.shape)}, {tuple(y.shape)}, expected "
                                       f"[tokens, {self.hidden}]")
        for t, what, dt in ((ids, "ids", torch.int32), (weights, "weights", torch.float32)):
            if not _is(t, dt) or t.shape != (T, self.topk):
                _dev(t, what, (str(dt).replace("torch.", ""),), shape=(T, self.topk))
        raw = _raw(stream)
        self._blocks.use(raw, stream)
        return self._lib.hbf_moe_layer(self._m, x.data_ptr(), _stride(x, 0), T, ids.data_ptr(), weights.data_ptr(),
                                       y.data_ptr(), _stride(y, 0), self._status.data_ptr(), self._ws.data_ptr(),
                                       self._ws.numel(), raw)

    def get_status(self, stream=None):
        """Synchronises; HBF_OK, or HBF_EINVAL if an id was out of range since
        the last call."""
        return _take_status(self._status, self._blocks, stream)


def refresh_plan(params, blocks, pages_per_block):
    """Device pages of a refresh plan in the scheduler's order (host-only).
    params: dict of model parameters; blocks: (epoch, zone, channel, die,
    plane, block) tuples.  Returns (status, uint64 array)."""
    import numpy as np
    lib = load_library()
    p = hbf_params(params["channels"], params["dies_per_channel"], params["planes_per_die"],
                   params["page_bytes"], params["t_read_ns"], params["channel_bytes_per_s"],
                   params.get("flags", 0))
    arr = (hbf_refresh_block * max(1, len(blocks)))(*[hbf_refresh_block(*b) for b in blocks])
    out = np.zeros(max(1, len(blocks) * pages_per_block), dtype=np.uint64)
    rc = lib.hbf_refresh_plan(ctypes.byref(p), ctypes.cast(arr, ctypes.c_void_p), len(blocks), pages_per_block,
                              out.ctypes.data_as(ctypes.c_void_p), len(blocks) * pages_per_block)
    return rc, out[:len(blocks) * pages_per_block]


def strerror(code):
    return load_library().hbf_strerror(code).decode()
