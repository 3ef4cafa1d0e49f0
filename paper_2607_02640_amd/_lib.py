"""ctypes binding of libmtn (include/mtn.h).

Argument marshalling only: every step of the attention path runs in the HIP
library.  Device buffers are passed as torch tensors (their data pointers) and
the stream as torch's current HIP stream.  Loading fails loudly when the
library has not been built; there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
# MTN_LIB selects another build of the same library (e.g. a tuning variant)
LIB_PATH = os.environ.get("MTN_LIB") or os.path.join(_HERE, "libmtn.so")

MTN_OK = 0
MTN_ERR_INVALID_ARG = -1
MTN_ERR_BAD_SESSION = -2
MTN_ERR_CHUNK_TOO_LARGE = -3
MTN_ERR_NO_SESSION_SLOT = -4
MTN_ERR_POOL_EXHAUSTED = -5
MTN_ERR_SESSION_FULL = -6
MTN_ERR_DEVICE = -7
MTN_ERR_BAD_STATE = -8
MTN_ERR_UNSUPPORTED = -9
MTN_ERR_HOST_MEMORY = -10

MTN_F32 = 0
MTN_BF16 = 1
MTN_FP8_E4M3 = 2
MTN_INT8_BLOCK = 3
# pool dtype name -> (kv_dtype, io_dtype); "fp8" keeps E4M3 codes, "int8" int8
# codes under one scale per block and head, both with bf16 io
DTYPES = {"f32": (MTN_F32, MTN_F32), "bf16": (MTN_BF16, MTN_BF16),
          "fp8": (MTN_FP8_E4M3, MTN_BF16), "int8": (MTN_INT8_BLOCK, MTN_BF16)}
MTN_WINDOW_UNBOUNDED = -1
MTN_POOL_HOST_ONLY = 1
# rotary forms of Pool.set_rope
ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "base": 2, "yarn": 3}

# every symbol include/mtn.h declares
EXPORTS = [
    "mtn_pool_required_bytes", "mtn_pool_create", "mtn_pool_destroy",
    "mtn_session_open", "mtn_session_close", "mtn_plan_begin", "mtn_plan_commit",
    "mtn_plan_abort",
    "mtn_pool_set_rope", "mtn_pool_set_qk_norm", "mtn_linear_required_bytes",
    "mtn_pool_set_linear", "mtn_session_state_slot", "mtn_attend_linear", "mtn_pool_linear_times", "mtn_session_fork", "mtn_pool_resize",
    "mtn_frame_append_kv", "mtn_attend_chunk_prefill", "mtn_attend_decode",
    "mtn_attend_decode_append", "mtn_attend_decode_noalloc",
    "mtn_frame_step", "mtn_pool_stats", "mtn_session_info", "mtn_session_block_table",
    "mtn_plan_info", "mtn_debug_poison_dead", "mtn_pool_set_timing", "mtn_pool_set_prefill_pass_rows",
    "mtn_pool_kernel_times", "mtn_pool_prefill_merge_times", "mtn_hbm_copy", "mtn_hbm_read", "mtn_status_string", "mtn_pool_last_error",
    "mtn_pool_set_decode_kernel", "mtn_pool_last_split", "mtn_debug_inject_failure",
    "mtn_admission_create", "mtn_admission_destroy", "mtn_admission_offer",
    "mtn_admission_release", "mtn_admission_observe", "mtn_admission_get",
]


class PoolConfig(C.Structure):
    _fields_ = [
        ("n_layers", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
        ("head_dim", C.c_int32), ("block_size", C.c_int32), ("n_sink", C.c_int32),
        ("window", C.c_int32), ("max_chunk", C.c_int32), ("max_sessions", C.c_int32),
        ("max_len", C.c_int32), ("n_blocks", C.c_int64), ("kv_dtype", C.c_int32),
        ("io_dtype", C.c_int32), ("rope_theta", C.c_double), ("softmax_scale", C.c_float),
        ("flags", C.c_uint32),
    ]


class RopeConfig(C.Structure):
    _fields_ = [
        ("layout", C.c_int32), ("rotary_dim", C.c_int32), ("scaling", C.c_int32),
        ("original_len", C.c_int32), ("factor", C.c_double), ("beta_fast", C.c_double),
        ("beta_slow", C.c_double), ("magnitude", C.c_double),
    ]


class QkNormConfig(C.Structure):
    _fields_ = [("q_weight", C.POINTER(C.c_float)), ("k_weight", C.POINTER(C.c_float)), ("eps", C.c_double)]


class LinearConfig(C.Structure):
    _fields_ = [
        ("n_layers", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
        ("head_dim", C.c_int32), ("io_dtype", C.c_int32), ("scale", C.c_float),
        ("log_decay", C.POINTER(C.c_float)),
    ]


class PoolStats(C.Structure):
    _fields_ = [
        ("capacity", C.c_int64), ("assigned", C.c_int64), ("reserved", C.c_int64),
        ("open_sessions", C.c_int32), ("blocks_per_session", C.c_int32),
        ("ring_tokens", C.c_int32), ("sink_blocks", C.c_int32),
    ]


class AdmissionConfig(C.Structure):
    _fields_ = [
        ("target_ms", C.c_double), ("backoff", C.c_double), ("increase", C.c_int32),
        ("initial_cap", C.c_int32), ("min_cap", C.c_int32), ("max_cap", C.c_int32),
        ("hold_ticks", C.c_int32),
    ]


class AdmissionState(C.Structure):
    _fields_ = [
        ("cap", C.c_int32), ("admitted", C.c_int32), ("hold", C.c_int32),
        ("offered", C.c_int64), ("rejected", C.c_int64), ("ticks", C.c_int64),
        ("decreases", C.c_int64), ("increases", C.c_int64),
    ]


class FrameBatch(C.Structure):
    _fields_ = [
        ("n_seq", C.c_int32),
        ("sids", C.POINTER(C.c_int32)), ("chunk_len", C.POINTER(C.c_int32)),
        ("n_decode", C.POINTER(C.c_int32)),
        ("q_chunk", C.c_void_p), ("k_chunk", C.c_void_p), ("v_chunk", C.c_void_p),
        ("out_chunk", C.c_void_p), ("lse_chunk", C.c_void_p),
        ("q_dec", C.c_void_p), ("k_dec", C.c_void_p), ("v_dec", C.c_void_p),
        ("out_dec", C.c_void_p), ("lse_dec", C.c_void_p),
        ("n_split", C.c_int32),
    ]


_lib = None


def load() -> C.CDLL:
    """Load libmtn.so (built by paper_2607_02640_amd.build); raise if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it with paper_2607_02640_amd.build.build() "
            "(the attention path has no non-HIP fallback)")
    lib = C.CDLL(LIB_PATH)
    i32, i64, vp = C.c_int32, C.c_int64, C.c_void_p
    P32, P64 = C.POINTER(C.c_int32), C.POINTER(C.c_int64)
    sig = {
        "mtn_pool_required_bytes": (i32, [C.POINTER(PoolConfig), C.POINTER(C.c_size_t)]),
        "mtn_pool_create": (i32, [C.POINTER(PoolConfig), vp, C.c_size_t, vp, C.POINTER(vp)]),
        "mtn_pool_destroy": (None, [vp]),
        "mtn_pool_set_rope": (i32, [vp, C.POINTER(RopeConfig)]),
        "mtn_pool_set_qk_norm": (i32, [vp, C.POINTER(QkNormConfig)]),
        "mtn_linear_required_bytes": (i32, [vp, C.POINTER(LinearConfig), C.POINTER(C.c_size_t)]),
        "mtn_pool_set_linear": (i32, [vp, C.POINTER(LinearConfig), vp, C.c_size_t]),
        "mtn_session_state_slot": (i32, [vp, i32, P32]),
        "mtn_attend_linear": (i32, [vp, i32, vp, vp, vp, vp, vp]),
        "mtn_pool_linear_times": (i32, [vp, P64, C.POINTER(C.c_double)]),
        "mtn_session_fork": (i32, [vp, i32, i32, P32, vp]),
        "mtn_pool_resize": (i32, [vp, i64, vp, C.c_size_t, vp]),
        "mtn_session_open": (i32, [vp, P32]),
        "mtn_session_close": (i32, [vp, i32]),
        "mtn_plan_begin": (i32, [vp, i32, P32, P32, vp]),
        "mtn_plan_commit": (i32, [vp]),
        "mtn_plan_abort": (i32, [vp]),
        "mtn_pool_set_decode_kernel": (i32, [vp, i32]),
        "mtn_pool_last_split": (i32, [vp, P32]),
        "mtn_debug_inject_failure": (i32, [vp, i64]),
        "mtn_frame_append_kv": (i32, [vp, i32, vp, vp, vp]),
        "mtn_attend_chunk_prefill": (i32, [vp, i32, vp, vp, vp, vp]),
        "mtn_attend_decode": (i32, [vp, i32, vp, vp, vp, i32, vp]),
        "mtn_attend_decode_append": (i32, [vp, i32, vp, vp, vp, vp, vp, i32, vp]),
        "mtn_attend_decode_noalloc": (i32, [vp, i32, vp, vp, vp, i32, vp]),
        "mtn_frame_step": (i32, [vp, C.POINTER(FrameBatch), vp]),
        "mtn_pool_stats": (i32, [vp, C.POINTER(PoolStats)]),
        "mtn_session_info": (i32, [vp, i32, P64, P32]),
        "mtn_session_block_table": (i32, [vp, i32, P32, i32, P32]),
        "mtn_plan_info": (i32, [vp, P64, P32, P32, i32, P64, P64, P32]),
        "mtn_debug_poison_dead": (i32, [vp, vp]),
        "mtn_pool_set_timing": (i32, [vp, i32]),
        "mtn_pool_set_prefill_pass_rows": (i32, [vp, i32]),
        "mtn_pool_kernel_times": (i32, [vp, P64, C.POINTER(C.c_double)]),
        "mtn_pool_prefill_merge_times": (i32, [vp, P64, C.POINTER(C.c_double)]),
        "mtn_hbm_copy": (i32, [vp, vp, C.c_size_t, vp]),
        "mtn_hbm_read": (i32, [vp, C.c_size_t, vp]),
        "mtn_admission_create": (i32, [C.POINTER(AdmissionConfig), C.POINTER(vp)]),
        "mtn_admission_destroy": (None, [vp]),
        "mtn_admission_offer": (i32, [vp, P32]),
        "mtn_admission_release": (i32, [vp]),
        "mtn_admission_observe": (i32, [vp, C.c_double]),
        "mtn_admission_get": (i32, [vp, C.POINTER(AdmissionState)]),
        "mtn_status_string": (C.c_char_p, [i32]),
        "mtn_pool_last_error": (C.c_char_p, [vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


class MtnError(RuntimeError):
    def __init__(self, code: int, where: str, detail: str = ""):
        lib = load()
        super().__init__(f"{where}: {lib.mtn_status_string(code).decode()} ({code})"
                         + (f": {detail}" if detail else ""))
        self.code = code


def _arr32(xs: Sequence[int]):
    return (C.c_int32 * len(xs))(*[int(x) for x in xs])


def _host_floats(x, where: str, n: int):
    """``n`` host floats of a tensor, array or nested list, or None (NULL)."""
    if x is None:
        return None
    import numpy as np
    a = x.detach().to("cpu").float().numpy() if hasattr(x, "detach") else x
    a = np.ascontiguousarray(a, dtype=np.float32).reshape(-1)
    if a.size != n:
        raise MtnError(MTN_ERR_INVALID_ARG, where, f"{a.size} values instead of {n}")
    return (C.c_float * n)(*a.tolist())


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    return t.data_ptr()


_torch = None  # once _stream has been asked


def _stream(stream) -> Optional[int]:
    global _torch
    if stream is not None:
        return stream
    if _torch is None:
        import torch as _torch
    torch = _torch
    if torch.cuda.is_initialized():
        # what current_stream().cuda_stream returns, without the Stream object, which
        # took half of a call's time on the host (3.4 of 6.6 us); the names are torch's
        # own, and a torch without them is asked the public way
        try:
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        except AttributeError:
            return torch.cuda.current_stream().cuda_stream
    if torch.cuda.is_available():
        return torch.cuda.current_stream().cuda_stream
    return None


class Pool:
    """A KV pool (mtn_pool) with the C ABI's calls as methods.

    ``kv`` is a caller-owned device tensor of at least ``required_bytes``;
    pass ``host_only=True`` to exercise planning without a device.
    """

    def __init__(self, *, n_layers, n_q_heads, n_kv_heads, head_dim, n_sink, window,
                 max_chunk, max_sessions, n_blocks, dtype="bf16", max_len=0,
                 rope_theta=10000.0, softmax_scale=0.0, block_size=16, host_only=False,
                 kv=None, stream=None):
        self.lib = load()
        kvt, iot = DTYPES[dtype]
        self.cfg = PoolConfig(
            n_layers, n_q_heads, n_kv_heads, head_dim, block_size, n_sink,
            MTN_WINDOW_UNBOUNDED if window is None else window, max_chunk, max_sessions,
            max_len, n_blocks, kvt, iot, rope_theta, softmax_scale,
            MTN_POOL_HOST_ONLY if host_only else 0)
        self.dtype = dtype
        self.host_only = host_only
        nbytes = C.c_size_t()
        self._check(self.lib.mtn_pool_required_bytes(C.byref(self.cfg), C.byref(nbytes)),
                    "required_bytes")
        self.required_bytes = nbytes.value
        self.kv = kv
        self.states = None  # of the linear layers: set_linear
        # their rows: torch dtype, device's index, elements of a query's and a KV row, device, head dim
        self._linear_rows = None
        self._plan_tokens = 0  # of the open plan
        h = C.c_void_p()
        st = self.lib.mtn_pool_create(C.byref(self.cfg), _ptr(kv) if kv is not None else None,
                                      C.c_size_t(kv.numel() * kv.element_size() if kv is not None else 0),
                                      None if host_only else _stream(stream), C.byref(h))
        self._check(st, "pool_create")
        self.h = h

    @staticmethod
    def required(**kw) -> int:
        lib = load()
        kvt, iot = DTYPES[kw.get("dtype", "bf16")]
        w = kw["window"]
        cfg = PoolConfig(kw["n_layers"], kw["n_q_heads"], kw["n_kv_heads"], kw["head_dim"],
                         kw.get("block_size", 16), kw["n_sink"],
                         MTN_WINDOW_UNBOUNDED if w is None else w, kw["max_chunk"],
                         kw["max_sessions"], kw.get("max_len", 0), kw["n_blocks"], kvt, iot,
                         kw.get("rope_theta", 1e4), 0.0, 0)
        n = C.c_size_t()
        st = lib.mtn_pool_required_bytes(C.byref(cfg), C.byref(n))
        if st:
            raise MtnError(st, "required_bytes")
        return n.value

    # -- helpers -------------------------------------------------------------
    def _check(self, st, where):
        if st != MTN_OK:
            detail = ""
            if getattr(self, "h", None) is not None:
                detail = (self.lib.mtn_pool_last_error(self.h) or b"").decode()
            raise MtnError(st, where, detail)

    def close(self):
        if getattr(self, "h", None) is not None and self.h.value:
            self.lib.mtn_pool_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- C ABI ---------------------------------------------------------------
    def session_open(self) -> int:
        sid = C.c_int32()
        self._check(self.lib.mtn_session_open(self.h, C.byref(sid)), "session_open")
        return sid.value

    def session_close(self, sid: int) -> None:
        self._check(self.lib.mtn_session_close(self.h, sid), "session_close")

    def session_fork(self, sid: int, copies: int = 1, stream=None) -> list:
        """New sessions that hold what session ``sid`` holds; their ids."""
        out = (C.c_int32 * max(copies, 1))()
        self._check(self.lib.mtn_session_fork(self.h, sid, copies, out,
                                              None if self.host_only else _stream(stream)), "session_fork")
        return list(out[:copies])

    def resize(self, n_blocks: int, kv=None, stream=None) -> None:
        """Move every page into the buffer ``kv`` with ``n_blocks`` blocks; the
        pool then holds ``kv`` and no longer the buffer before it."""
        if not self.host_only and kv is not None and not (kv.device == self.kv.device and kv.is_contiguous()):
            raise MtnError(MTN_ERR_INVALID_ARG, "resize", "kv: not contiguous, or on another device")
        size = C.c_size_t(kv.numel() * kv.element_size() if kv is not None else 0)
        if self.kv is not None:  # torch may not hand the old buffer out before the copy has run
            import torch
            self.kv.record_stream(torch.cuda.current_stream() if stream is None
                                  else torch.cuda.ExternalStream(stream))
        self._check(self.lib.mtn_pool_resize(self.h, n_blocks, _ptr(kv), size,
                                             None if self.host_only else _stream(stream)), "resize")
        self.cfg.n_blocks = n_blocks
        n = C.c_size_t()
        self._check(self.lib.mtn_pool_required_bytes(C.byref(self.cfg), C.byref(n)), "resize")
        self.required_bytes, self.kv = n.value, kv

    def plan_begin(self, sids, n_tok, stream=None) -> None:
        n_tok = [int(x) for x in n_tok]
        st = self.lib.mtn_plan_begin(self.h, len(sids), _arr32(sids), (C.c_int32 * len(n_tok))(*n_tok),
                                     None if self.host_only else _stream(stream))
        self._check(st, "plan_begin")
        if self._linear_rows is not None:
            self._plan_tokens = sum(n_tok[:len(sids)])

    def plan_commit(self) -> None:
        self._check(self.lib.mtn_plan_commit(self.h), "plan_commit")
        self._plan_tokens = 0

    def plan_abort(self) -> None:
        self._check(self.lib.mtn_plan_abort(self.h), "plan_abort")
        self._plan_tokens = 0

    def _not_captured(self, where: str) -> None:
        if not self.host_only:
            import torch
            if torch.cuda.is_current_stream_capturing():
                raise MtnError(MTN_ERR_BAD_STATE, where, "the current stream is being captured")

    def set_rope(self, *, layout="half", rotary_dim=0, scaling="none", factor=1.0, original_len=0,
                 beta_fast=0.0, beta_slow=0.0, magnitude=0.0) -> None:
        """Rotary positions of later appends and queries (mtn_pool_set_rope): layout
        "half" or "interleaved", scaling "none", "linear", "base" or "yarn"."""
        self._not_captured("set_rope")
        cfg = RopeConfig(ROPE_LAYOUTS[layout], rotary_dim, ROPE_SCALINGS[scaling], original_len,
                         factor, beta_fast, beta_slow, magnitude)
        self._check(self.lib.mtn_pool_set_rope(self.h, C.byref(cfg)), "set_rope")

    def set_qk_norm(self, q_weight=None, k_weight=None, eps: float = 1e-6) -> None:
        """Norm every query and key row before it is rotated (mtn_pool_set_qk_norm).
        Weights: [n_layers][head_dim], a tensor of any device, an array or lists;
        None is all ones."""
        self._not_captured("set_qk_norm")
        n = self.cfg.n_layers * self.cfg.head_dim
        w = [_host_floats(x, "set_qk_norm", n) for x in (q_weight, k_weight)]
        cfg = QkNormConfig(*(C.cast(x, C.POINTER(C.c_float)) for x in w), eps)
        self._check(self.lib.mtn_pool_set_qk_norm(self.h, C.byref(cfg)), "set_qk_norm")

    def clear_qk_norm(self) -> None:
        """Back to rows that are only rotated."""
        self._not_captured("clear_qk_norm")
        self._check(self.lib.mtn_pool_set_qk_norm(self.h, None), "clear_qk_norm")

    @staticmethod
    def linear_shape(max_sessions, n_layers, n_kv_heads, head_dim) -> tuple:
        """Shape of the float32 tensor that holds the linear layers' states."""
        return (max_sessions, 2, n_layers, n_kv_heads, head_dim, head_dim)

    def set_linear(self, *, n_layers, n_q_heads, n_kv_heads, head_dim, log_decay, states=None, dtype="bf16",
                   scale=0.0) -> None:
        """Linear-attention layers beside the pool's own (mtn_pool_set_linear).
        ``log_decay``: [n_layers][n_kv_heads], a tensor, an array or lists;
        ``states``: a contiguous float32 device tensor of ``linear_shape``, which the
        pool then holds (host-only pools: None)."""
        where = "set_linear"
        self._not_captured(where)
        if dtype not in ("f32", "bf16"):
            raise MtnError(MTN_ERR_UNSUPPORTED, where, f"dtype {dtype}")
        if states is not None and not self.host_only:
            import torch
            shape = self.linear_shape(self.cfg.max_sessions, n_layers, n_kv_heads, head_dim)
            if tuple(states.shape) != shape or states.dtype != torch.float32 or not states.is_contiguous() \
                    or states.device != self.kv.device:
                raise MtnError(MTN_ERR_INVALID_ARG, where, f"states: not a contiguous float32 tensor {shape} on the "
                               "pool's device")
        decay = _host_floats(log_decay, where, max(n_layers, 0) * max(n_kv_heads, 0))
        cfg = LinearConfig(n_layers, n_q_heads, n_kv_heads, head_dim, DTYPES[dtype][1], scale,
                           C.cast(decay, C.POINTER(C.c_float)))
        size = C.c_size_t(states.numel() * states.element_size() if states is not None else 0)
        self._check(self.lib.mtn_pool_set_linear(self.h, C.byref(cfg), _ptr(states), size), where)
        self.states = states
        self._linear_rows = None
        if states is not None:
            import torch
            self._linear_rows = (torch.float32 if dtype == "f32" else torch.bfloat16,
                                 None if self.host_only else states.get_device(), n_q_heads * head_dim,
                                 n_kv_heads * head_dim, states.device, head_dim)

    def clear_linear(self) -> None:
        """Take the linear layers away; the pool then holds their states no longer."""
        self._not_captured("clear_linear")
        self._check(self.lib.mtn_pool_set_linear(self.h, None, None, C.c_size_t(0)), "clear_linear")
        self.states = self._linear_rows = None

    def state_slot(self, sid: int) -> int:
        """Which of session ``sid``'s two slots of the states is the committed one."""
        slot = C.c_int32()
        self._check(self.lib.mtn_session_state_slot(self.h, sid, C.byref(slot)), "state_slot")
        return slot.value

    def session_state(self, sid: int):
        """The committed state of session ``sid``: a view [layers][KV heads][D][D] of
        the states (undefined while the session has no tokens)."""
        return self.states[sid, self.state_slot(sid)]

    def attend_linear(self, layer, q, k, v, out, stream=None) -> None:
        """One linear layer of the open plan (mtn_attend_linear): contiguous tensors of
        the linear layers' dtype on the pool's device, q and out [T][Hq][D], k and v
        [T][Hkv][D] or more rows (those behind the plan's are left alone)."""
        if self._linear_rows is not None:
            io, dev, per_q, per_kv, *_ = self._linear_rows
            nq, nkv = self._plan_tokens * per_q, self._plan_tokens * per_kv
            # (one pass over what nearly every call brings; a layer's call is 5 us of host time)
            for t, n, per in (q, nq, per_q), (k, nkv, per_kv), (v, nkv, per_kv), (out, nq, per_q):
                if t is None or not (t.dtype is io and t.numel() == n and t.get_device() == dev and t.is_contiguous()):
                    self._check_linear_rows(t, n, per)
        st = self.lib.mtn_attend_linear(self.h, layer, None if q is None else q.data_ptr(),
                                        None if k is None else k.data_ptr(), None if v is None else v.data_ptr(),
                                        None if out is None else out.data_ptr(), _stream(stream))
        if st:
            self._check(st, "attend_linear")

    def _check_linear_rows(self, t, n: int, per: int) -> None:
        """At least ``n`` elements in rows of ``per``, which are heads of D where the
        shape says how a row is cut; the library refuses None."""
        io, _, _, _, device, d = self._linear_rows
        if t is None:
            return
        if not (t.dtype == io and t.device == device and t.is_contiguous()):
            raise MtnError(MTN_ERR_INVALID_ARG, "attend_linear", "rows: not a contiguous tensor of the linear "
                           "layers' dtype on the pool's device")
        cut = tuple(t.shape[-2:] if t.dim() > 2 else t.shape[1:])
        if n and not (t.numel() >= n and cut in ((per // d, d), (per,), ())):
            raise MtnError(MTN_ERR_INVALID_ARG, "attend_linear",
                           f"rows {tuple(t.shape)}: not {n // per} rows of {per // d} x {d} elements or more")

    def set_decode_kernel(self, kind: int) -> None:
        """0 = by shape, 1 = vector kernel, 2 = matrix-core kernel."""
        self._check(self.lib.mtn_pool_set_decode_kernel(self.h, kind), "set_decode_kernel")

    def last_split(self) -> int:
        n = C.c_int32()
        self._check(self.lib.mtn_pool_last_split(self.h, C.byref(n)), "last_split")
        return n.value

    def inject_failure(self, launch_index: int) -> None:
        self._check(self.lib.mtn_debug_inject_failure(self.h, launch_index), "inject_failure")

    def frame_append_kv(self, layer, k, v, stream=None) -> None:
        self._check(self.lib.mtn_frame_append_kv(self.h, layer, _ptr(k), _ptr(v), _stream(stream)),
                    "frame_append_kv")

    def attend_chunk_prefill(self, layer, q, out, lse=None, stream=None) -> None:
        self._check(self.lib.mtn_attend_chunk_prefill(self.h, layer, _ptr(q), _ptr(out), _ptr(lse),
                                                      _stream(stream)), "attend_chunk_prefill")

    def attend_decode(self, layer, q, out, lse=None, n_split=0, stream=None) -> None:
        self._check(self.lib.mtn_attend_decode(self.h, layer, _ptr(q), _ptr(out), _ptr(lse),
                                               n_split, _stream(stream)), "attend_decode")

    def attend_decode_noalloc(self, layer, q, out, lse=None, n_split=0, stream=None) -> None:
        self._check(self.lib.mtn_attend_decode_noalloc(self.h, layer, _ptr(q), _ptr(out),
                                                       _ptr(lse), n_split, _stream(stream)),
                    "attend_decode_noalloc")

    def attend_decode_append(self, layer, k, v, q, out, lse=None, n_split=0,
                             stream=None) -> None:
        self._check(self.lib.mtn_attend_decode_append(self.h, layer, _ptr(k), _ptr(v), _ptr(q),
                                                      _ptr(out), _ptr(lse), n_split,
                                                      _stream(stream)), "attend_decode_append")

    def frame_step(self, sids, chunk_len, n_decode, q_chunk, k_chunk, v_chunk, out_chunk,
                   q_dec=None, k_dec=None, v_dec=None, out_dec=None, lse_chunk=None,
                   lse_dec=None, n_split=0, stream=None) -> None:
        b = FrameBatch()
        b.n_seq = len(sids)
        self._keep = (_arr32(sids), _arr32(chunk_len), _arr32(n_decode))
        b.sids, b.chunk_len, b.n_decode = (C.cast(a, C.POINTER(C.c_int32)) for a in self._keep)
        b.q_chunk, b.k_chunk, b.v_chunk = _ptr(q_chunk), _ptr(k_chunk), _ptr(v_chunk)
        b.out_chunk, b.lse_chunk = _ptr(out_chunk), _ptr(lse_chunk)
        b.q_dec, b.k_dec, b.v_dec = _ptr(q_dec), _ptr(k_dec), _ptr(v_dec)
        b.out_dec, b.lse_dec = _ptr(out_dec), _ptr(lse_dec)
        b.n_split = n_split
        self._check(self.lib.mtn_frame_step(self.h, C.byref(b),
                                            None if self.host_only else _stream(stream)),
                    "frame_step")

    def stats(self) -> dict:
        s = PoolStats()
        self._check(self.lib.mtn_pool_stats(self.h, C.byref(s)), "pool_stats")
        return {k: getattr(s, k) for k, _ in PoolStats._fields_}

    def session_info(self, sid):
        ln, na = C.c_int64(), C.c_int32()
        self._check(self.lib.mtn_session_info(self.h, sid, C.byref(ln), C.byref(na)), "session_info")
        return ln.value, na.value

    def block_table(self, sid):
        n = self.stats()["blocks_per_session"]
        buf = (C.c_int32 * n)()
        cnt = C.c_int32()
        self._check(self.lib.mtn_session_block_table(self.h, sid, buf, n, C.byref(cnt)),
                    "session_block_table")
        return list(buf[:cnt.value])

    def plan_info(self, n_seq: int, cap: int = 1 << 16):
        pos = (C.c_int64 * cap)()
        blk = (C.c_int32 * cap)()
        off = (C.c_int32 * cap)()
        lo = (C.c_int64 * cap)()
        hi = (C.c_int64 * cap)()
        n = C.c_int32()
        self._check(self.lib.mtn_plan_info(self.h, pos, blk, off, cap, lo, hi, C.byref(n)),
                    "plan_info")
        return (list(pos[:n.value]), list(blk[:n.value]), list(off[:n.value]),
                list(lo[:n_seq]), list(hi[:n_seq]))

    def poison_dead(self, stream=None) -> None:
        self._check(self.lib.mtn_debug_poison_dead(self.h, _stream(stream)), "debug_poison_dead")

    def set_prefill_pass_rows(self, rows: int) -> None:
        """Query rows per chunk-prefill pass: 0 = per plan, or 128 / 256."""
        self._check(self.lib.mtn_pool_set_prefill_pass_rows(self.h, rows), "set_prefill_pass_rows")

    def set_timing(self, on: bool) -> None:
        self._check(self.lib.mtn_pool_set_timing(self.h, 1 if on else 0), "set_timing")

    def kernel_times(self):
        n = (C.c_int64 * 4)()
        ms = (C.c_double * 4)()
        self._check(self.lib.mtn_pool_kernel_times(self.h, n, ms), "kernel_times")
        names = ("append", "prefill", "decode", "merge")
        times = {names[i]: (n[i], ms[i]) for i in range(4)}
        # the chunk prefill's share of the merges
        self._check(self.lib.mtn_pool_prefill_merge_times(self.h, n, ms), "kernel_times")
        times["prefill_merge"] = (n[0], ms[0])
        self._check(self.lib.mtn_pool_linear_times(self.h, n, ms), "kernel_times")
        times["linear"] = (n[0], ms[0])
        return times


def hbm_copy(src, dst, nbytes: int, stream=None) -> None:
    lib = load()
    st = lib.mtn_hbm_copy(_ptr(src), _ptr(dst), C.c_size_t(nbytes), _stream(stream))
    if st != MTN_OK:
        raise MtnError(st, "hbm_copy")


def hbm_read(src, nbytes: int, stream=None) -> None:
    lib = load()
    st = lib.mtn_hbm_read(_ptr(src), C.c_size_t(nbytes), _stream(stream))
    if st != MTN_OK:
        raise MtnError(st, "hbm_read")


class Admission:
    """AIMD admission controller on the per-frame latency (host only; see
    mtn_admission_* in include/mtn.h)."""

    def __init__(self, *, target_ms, backoff, increase, initial_cap, min_cap, max_cap,
                 hold_ticks):
        self._lib = load()
        cfg = AdmissionConfig(float(target_ms), float(backoff), int(increase), int(initial_cap),
                              int(min_cap), int(max_cap), int(hold_ticks))
        h = C.c_void_p()
        st = self._lib.mtn_admission_create(C.byref(cfg), C.byref(h))
        if st != MTN_OK:
            raise MtnError(st, "mtn_admission_create")
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            self._lib.mtn_admission_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def offer(self) -> bool:
        out = C.c_int32()
        st = self._lib.mtn_admission_offer(self._h, C.byref(out))
        if st != MTN_OK:
            raise MtnError(st, "mtn_admission_offer")
        return bool(out.value)

    def release(self) -> None:
        st = self._lib.mtn_admission_release(self._h)
        if st != MTN_OK:
            raise MtnError(st, "mtn_admission_release")

    def observe(self, tick_ms: float) -> None:
        st = self._lib.mtn_admission_observe(self._h, C.c_double(tick_ms))
        if st != MTN_OK:
            raise MtnError(st, "mtn_admission_observe")

    def state(self) -> dict:
        s = AdmissionState()
        st = self._lib.mtn_admission_get(self._h, C.byref(s))
        if st != MTN_OK:
            raise MtnError(st, "mtn_admission_get")
        return {k: getattr(s, k) for k, _ in AdmissionState._fields_}
