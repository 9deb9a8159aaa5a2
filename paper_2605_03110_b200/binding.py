"""Binding of libada.so -- same names as include/ada.h, marshalling only (ctypes; the calls of the
selection and attention path through the native _pycall module).

Every step of the selection runs inside the CUDA library; this module converts
torch tensors to pointers, allocates output tensors, and raises on any
non-zero status.  There is no fallback: if the shared library has not been
built (python -m paper_2605_03110_b200.build) loading fails loudly.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libada.so")

ADA_OK = 0
ADA_F32, ADA_BF16 = 0, 1
ADA_CROSS_CAUSAL = 1
ADA_ATTN_CAUSAL = 1
ADA_ROPE_PAIRS = 1
ADA_ENGINE_AUTO, ADA_ENGINE_FFMA, ADA_ENGINE_TCGEN05, ADA_ENGINE_TCGEN05_PAIR = 0, 1, 2, 3

SYMBOLS = [
    "ada_create", "ada_destroy", "ada_set_engine", "ada_normalize", "ada_select_full",
    "ada_cascade_step", "ada_select_full_host", "ada_cascade_step_host", "ada_gram_op_count",
    "ada_device_status", "ada_profile_enable", "ada_profile_read", "ada_status_string",
    "ada_select_full_noalloc", "ada_set_cooperative", "ada_selftest_wait_timeout",
    "ada_selftest_launches_alone", "ada_nearest_rep",
    "ada_select_full_heads", "ada_cascade_step_heads", "ada_set_dependent_launch",
    "ada_cascade_step_adaptive", "ada_attention_reps", "ada_set_row_compaction",
    "ada_cache_append", "ada_attention_cached", "ada_select_blocks", "ada_attention_blocks",
]
ADA_NOALLOC_MAX_T = 16384

_lib = None
_fast = None             # the _pycall module, once the library is loaded


class TauPolicy(C.Structure):
    """ada_tau_policy: tau' = clip(tau + gain * (target_turnover - rho), tau_min, tau_max)."""
    _fields_ = [("target_turnover", C.c_double), ("gain", C.c_double), ("tau_min", C.c_double),
                ("tau_max", C.c_double)]


class _KVCacheStruct(C.Structure):
    """ada_kv_cache"""
    _fields_ = [(n, C.c_void_p) for n in ("k", "v", "kmin", "kmax", "table")] + \
        [(n, C.c_int64) for n in ("table_ld", "max_pages", "n_pages", "page_stride", "page_size", "h_kv", "d_h")]


class AdaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


def lib() -> C.CDLL:
    global _lib, _fast
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2605_03110_b200.build`; "
                "there is no CPU fallback")
        L = C.CDLL(LIB_PATH)
        vp, i64, i32p, fp = C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p
        L.ada_create.argtypes = [C.POINTER(vp), C.c_int, i64, i64, i64, C.c_int]
        L.ada_destroy.argtypes = [vp]
        L.ada_set_engine.argtypes = [vp, C.c_int]
        L.ada_set_cooperative.argtypes = [vp, C.c_int]
        L.ada_set_dependent_launch.argtypes = [vp, C.c_int]
        L.ada_set_row_compaction.argtypes = [vp, i64]
        L.ada_selftest_wait_timeout.argtypes = [vp, C.c_int, vp]
        L.ada_selftest_launches_alone.argtypes = [C.c_int, vp]
        L.ada_normalize.argtypes = [vp, vp, i64, i64, i64, i64, C.c_int, vp, fp, i32p, i32p, vp, vp]
        L.ada_select_full.argtypes = [vp, vp, i64, i64, i64, i64, C.c_int, C.c_double, i32p, i32p,
                                      fp, vp]
        L.ada_cascade_step.argtypes = [vp, vp, i64, i64, i64, i64, C.c_int, C.c_double,
                                       i32p, i32p, i32p, i32p, i32p, i32p, i32p, i32p, fp, fp,
                                       C.c_uint32, vp]
        L.ada_cascade_step_adaptive.argtypes = [vp, vp, i64, i64, i64, i64, C.c_int, vp,
                                                C.POINTER(TauPolicy), i32p, i32p, i32p, i32p, i32p,
                                                i32p, i32p, i32p, fp, fp, fp, C.c_uint32, vp]
        L.ada_select_full_heads.argtypes = L.ada_select_full.argtypes
        L.ada_cascade_step_heads.argtypes = L.ada_cascade_step.argtypes
        L.ada_nearest_rep.argtypes = [vp, vp, i64, i64, i64, i64, C.c_int, i32p, i32p, i32p, fp, vp]
        L.ada_attention_reps.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, C.c_int, i32p, i32p, i32p, fp,
                                         i64, C.c_uint32, vp]
        kv = C.POINTER(_KVCacheStruct)
        L.ada_cache_append.argtypes = [vp, kv, i64, i32p, i32p, i32p, i64, vp, i64, vp, i64, C.c_int, vp, i64, i64, vp,
                                       i64, vp, vp, C.c_double, vp, i64, i32p, i32p, i32p, C.c_uint32, vp]
        L.ada_attention_cached.argtypes = [vp, kv, i64, i32p, i32p, i64, i64, vp, i64, i64, C.c_int, C.c_double, vp, i64,
                                           C.c_uint32, vp]
        L.ada_select_blocks.argtypes = [vp, kv, i64, i32p, i32p, i64, vp, i64, i64, C.c_int, i64, i64, i64, i32p, i32p,
                                        C.c_uint32, vp]
        L.ada_attention_blocks.argtypes = [vp, kv, i64, i32p, i32p, i64, vp, i64, i64, C.c_int, i32p, i32p, i64,
                                           C.c_double, vp, i64, C.c_uint32, vp]
        L.ada_select_full_host.argtypes = [vp, vp, i64, i64, i64, C.c_int, C.c_double, i32p, i32p, fp, vp]
        L.ada_cascade_step_host.argtypes = [vp, vp, i64, i64, i64, C.c_int, C.c_double,
                                            i32p, i32p, i32p, i32p, i32p, i32p, i32p, i32p, fp, fp,
                                            C.c_uint32, vp]
        L.ada_select_full_noalloc.argtypes = [vp, i64, i64, i64, C.c_int, C.c_double, i32p, i32p,
                                              fp, vp]
        L.ada_gram_op_count.argtypes = [C.c_int, i64, i64, i64]
        L.ada_gram_op_count.restype = C.c_uint64
        L.ada_device_status.argtypes = [vp, vp, C.POINTER(i64)]
        L.ada_profile_enable.argtypes = [vp, C.c_int]
        L.ada_profile_read.argtypes = [vp, C.POINTER(C.c_char_p), C.POINTER(i64),
                                       C.POINTER(C.c_double), C.c_int]
        L.ada_status_string.argtypes = [C.c_int]
        L.ada_status_string.restype = C.c_char_p
        for name in SYMBOLS:
            if name not in ("ada_gram_op_count", "ada_status_string"):
                getattr(L, name).restype = C.c_int
        try:
            from . import _pycall
        except ImportError as e:
            raise RuntimeError(
                "the native marshalling module of this interpreter is missing or does not load: build it with "
                f"`python -m paper_2605_03110_b200.build` ({e})") from e
        _lib, _fast = L, _pycall
    return _lib


def status_string(s: int) -> str:
    return lib().ada_status_string(int(s)).decode()


def _check(st: int, where: str) -> None:
    if st != ADA_OK:
        raise AdaError(st, where)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


# the current stream's handle without a Stream object around it, where torch has these functions
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is None:
            return torch.cuda.current_stream().cuda_stream
        return _raw_stream(_current_device())
    return stream.cuda_stream


def _stream_of(ctx, stream) -> int:
    """The current stream of the context's device, whichever device is the current one."""
    if stream is None:
        if _raw_stream is None:
            return torch.cuda.current_stream(ctx.device).cuda_stream
        return _raw_stream(ctx.device)
    return stream.cuda_stream


_NO_SWITCH = contextlib.nullcontext()


def _on(stream, like: torch.Tensor):
    """Where a call makes its own outputs: on the stream that its kernels run on.  Filled on another one, they could be
    cleared after the kernel has written them, and their memory could still be in use there."""
    return _NO_SWITCH if stream is None or like.get_device() < 0 else torch.cuda.stream(stream)


def _fresh(stream, make, like: torch.Tensor, shape):
    """_on for one tensor make(shape), with less to do where no stream was passed."""
    if stream is None:
        return make(shape)
    with _on(stream, like):
        return make(shape)


def _raise(st: int, where: str) -> None:
    raise AdaError(st, where)


def dtype_of(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return ADA_F32
    if t.dtype == torch.bfloat16:
        return ADA_BF16
    raise TypeError(f"unsupported activation dtype {t.dtype}")


def _shape(X: torch.Tensor):
    if X.dim() == 2:
        X = X.unsqueeze(0)
    if X.dim() == 3:
        B, T, d = X.shape
        sb, st, sd = X.stride()
        if sd == 1 and (B <= 1 or sb == T * st):
            return X, B, T, d, st
    raise ValueError("X must be (B,)T x d, unit inner stride, sequences densely stacked")


class Context:
    """Owner of an ada_ctx handle."""

    def __init__(self, maxB: int, maxT: int, maxd: int, dtype: int, device: int = 0):
        h = C.c_void_p()
        _check(lib().ada_create(C.byref(h), device, maxB, maxT, maxd, dtype), "ada_create")
        self.h, self.device, self.dtype = h, device, dtype
        self.addr = h.value              # None once closed: the library then reports an invalid argument
        self.maxB, self.maxT, self.maxd = maxB, maxT, maxd

    def close(self):
        if self.h:
            lib().ada_destroy(self.h)
            self.h = self.addr = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def ada_create(maxB: int, maxT: int, maxd: int, dtype: int, device: int = 0) -> Context:
    return Context(maxB, maxT, maxd, dtype, device)


def ada_destroy(ctx: Context) -> None:
    ctx.close()


def ada_set_engine(ctx: Context, engine: int) -> None:
    _check(lib().ada_set_engine(ctx.h, engine), "ada_set_engine")


def ada_set_cooperative(ctx: Context, on: bool) -> None:
    _check(lib().ada_set_cooperative(ctx.h, int(bool(on))), "ada_set_cooperative")


def ada_set_row_compaction(ctx: Context, min_rows: int) -> None:
    """Sequence length from which a large inherited set's complement is copied out for the cross step."""
    _check(lib().ada_set_row_compaction(ctx.h, int(min_rows)), "ada_set_row_compaction")


def ada_set_dependent_launch(ctx: Context, on: bool) -> None:
    _check(lib().ada_set_dependent_launch(ctx.h, int(bool(on))), "ada_set_dependent_launch")


def ada_selftest_wait_timeout(ctx: Context, limit_ms: int = 50, stream=None) -> None:
    """Enqueue the bounded-wait self-test; ada_device_status then reports ADA_ERR_TIMEOUT."""
    _check(lib().ada_selftest_wait_timeout(ctx.h, int(limit_ms), _stream(stream)),
           "ada_selftest_wait_timeout")


def ada_selftest_launches_alone(stream=None, device: int = 0) -> bool:
    """Is `stream` the one stream of the device whose launches go without the cooperative attribute?"""
    return bool(lib().ada_selftest_launches_alone(device, _stream(stream)))


def ada_gram_op_count(cascade: bool, T: int, d: int, r: int = 0) -> int:
    return int(lib().ada_gram_op_count(int(bool(cascade)), T, d, r))


def ada_device_status(ctx: Context, stream=None):
    """Returns (status, n_zero_norm_rows); synchronises the stream."""
    n = C.c_int64(0)
    st = lib().ada_device_status(ctx.h, _stream(stream), C.byref(n))
    return st, n.value


def ada_normalize(ctx: Context, X: torch.Tensor, want_xhat=False, rep_idx=None, rep_cnt=None,
                  stream=None):
    """Returns (inv_norm, Xhat or None, Xrep or None)."""
    X, B, T, d, ldx = _shape(X)
    with _on(stream, X):
        inv = torch.empty((B, T), dtype=torch.float32, device=X.device)
        xhat = torch.empty((B, T, d), dtype=X.dtype, device=X.device) if want_xhat else None
        xrep = torch.zeros((B, T, d), dtype=X.dtype, device=X.device) if rep_idx is not None else None
    _check(lib().ada_normalize(ctx.h, X.data_ptr(), B, T, d, ldx, dtype_of(X), _ptr(xhat),
                               inv.data_ptr(), _ptr(rep_idx), _ptr(rep_cnt), _ptr(xrep),
                               _stream(stream)), "ada_normalize")
    return inv, xhat, xrep


def ada_select_full(ctx: Context, X: torch.Tensor, tau: float, rep_idx=None, rep_cnt=None,
                    gamma=None, want_gamma=True, stream=None):
    """Definition 1.  Returns (rep_idx[B,T] int32, rep_cnt[B] int32, gamma[B,T] or None)."""
    X, B, T, d, ldx = _shape(X)
    dev = X.device
    with _on(stream, X):
        if rep_idx is None:
            rep_idx = torch.empty((B, T), dtype=torch.int32, device=dev)
        if rep_cnt is None:
            rep_cnt = torch.empty((B,), dtype=torch.int32, device=dev)
        if gamma is None and want_gamma:
            gamma = torch.empty((B, T), dtype=torch.float32, device=dev)
    st = _fast.select_full(ctx.addr, X, B, T, d, ldx, dtype_of(X), tau, rep_idx, rep_cnt, gamma, _stream(stream))
    if st:
        _raise(st, "ada_select_full")
    return rep_idx, rep_cnt, gamma


class CascadeOut:
    __slots__ = ("rep_out", "rep_out_cnt", "add_idx", "add_cnt", "rem_idx", "rem_cnt",
                 "gamma_rep", "gamma_cross")

    def __init__(self, B, T, dev, want_gamma):
        i32 = dict(dtype=torch.int32, device=dev)
        self.rep_out = torch.empty((B, T), **i32)
        self.add_idx = torch.empty((B, T), **i32)
        self.rem_idx = torch.empty((B, T), **i32)
        self.rep_out_cnt = torch.empty((B,), **i32)
        self.add_cnt = torch.empty((B,), **i32)
        self.rem_cnt = torch.empty((B,), **i32)
        self.gamma_rep = torch.empty((B, T), dtype=torch.float32, device=dev) if want_gamma else None
        self.gamma_cross = torch.empty((B, T), dtype=torch.float32, device=dev) if want_gamma else None


def ada_cascade_step(ctx: Context, X: torch.Tensor, tau: float, rep_in: torch.Tensor,
                     rep_in_cnt: torch.Tensor, out: Optional[CascadeOut] = None, flags: int = 0,
                     want_gamma=True, stream=None) -> CascadeOut:
    """Algorithm 1.  `out` buffers are reused when given."""
    X, B, T, d, ldx = _shape(X)
    if out is None:
        with _on(stream, X):
            out = CascadeOut(B, T, X.device, want_gamma)
    st = _fast.cascade_step(ctx.addr, X, B, T, d, ldx, dtype_of(X), tau, rep_in, rep_in_cnt, out.rep_out,
                            out.rep_out_cnt, out.add_idx, out.add_cnt, out.rem_idx, out.rem_cnt, out.gamma_rep,
                            out.gamma_cross, flags, _stream(stream))
    if st:
        _raise(st, "ada_cascade_step")
    return out


def ada_cascade_step_adaptive(ctx: Context, X: torch.Tensor, tau_state: torch.Tensor,
                              policy: Optional[TauPolicy], rep_in: torch.Tensor,
                              rep_in_cnt: torch.Tensor, out: Optional[CascadeOut] = None,
                              flags: int = 0, want_gamma=True, turnover: Optional[torch.Tensor] = None,
                              stream=None) -> CascadeOut:
    """Section 8.1: Algorithm 1 with the per-sequence threshold tau_state (float64[B] on the
    device, updated in place when a policy is given); `turnover` (float32[B]) receives Eq. 6."""
    X, B, T, d, ldx = _shape(X)
    assert tau_state.dtype == torch.float64 and tau_state.is_cuda and tau_state.numel() == B
    if policy is not None and not isinstance(policy, TauPolicy):
        raise C.ArgumentError("policy must be a TauPolicy")
    if out is None:
        with _on(stream, X):
            out = CascadeOut(B, T, X.device, want_gamma)
    st = _fast.cascade_step_adaptive(
        ctx.addr, X, B, T, d, ldx, dtype_of(X), tau_state, None if policy is None else C.addressof(policy), rep_in,
        rep_in_cnt, out.rep_out, out.rep_out_cnt, out.add_idx, out.add_cnt, out.rem_idx, out.rem_cnt, out.gamma_rep,
        out.gamma_cross, turnover, flags, _stream(stream))
    if st:
        _raise(st, "ada_cascade_step_adaptive")
    return out


def _shape_heads(X: torch.Tensor):
    if X.dim() == 3:
        T, h, d_h = X.shape
        st, sh, sd = X.stride()
        if sd == 1 and sh == d_h:
            return T, h, d_h, st
    raise ValueError("X must be T x h x d_h with the heads of a token side by side")


def ada_select_full_heads(ctx: Context, X: torch.Tensor, tau: float, rep_idx=None, rep_cnt=None,
                          gamma=None, want_gamma=True, stream=None):
    """Section 8.5: Definition 1 per head of X (T, h, d_h).  Returns (rep_idx[h,T], rep_cnt[h],
    gamma[h,T] or None)."""
    T, h, d_h, ldx = _shape_heads(X)
    dev = X.device
    with _on(stream, X):
        if rep_idx is None:
            rep_idx = torch.empty((h, T), dtype=torch.int32, device=dev)
        if rep_cnt is None:
            rep_cnt = torch.empty((h,), dtype=torch.int32, device=dev)
        if gamma is None and want_gamma:
            gamma = torch.empty((h, T), dtype=torch.float32, device=dev)
    st = _fast.select_full_heads(ctx.addr, X, T, h, d_h, ldx, dtype_of(X), tau, rep_idx, rep_cnt, gamma,
                                 _stream(stream))
    if st:
        _raise(st, "ada_select_full_heads")
    return rep_idx, rep_cnt, gamma


def ada_cascade_step_heads(ctx: Context, X: torch.Tensor, tau: float, rep_in: torch.Tensor,
                           rep_in_cnt: torch.Tensor, out: Optional[CascadeOut] = None,
                           flags: int = 0, want_gamma=True, stream=None) -> CascadeOut:
    """Section 8.5: Algorithm 1 per head of X (T, h, d_h); lists are [h, T], counts [h]."""
    T, h, d_h, ldx = _shape_heads(X)
    if out is None:
        with _on(stream, X):
            out = CascadeOut(h, T, X.device, want_gamma)
    st = _fast.cascade_step_heads(ctx.addr, X, T, h, d_h, ldx, dtype_of(X), tau, rep_in, rep_in_cnt, out.rep_out,
                                  out.rep_out_cnt, out.add_idx, out.add_cnt, out.rem_idx, out.rem_cnt, out.gamma_rep,
                                  out.gamma_cross, flags, _stream(stream))
    if st:
        _raise(st, "ada_cascade_step_heads")
    return out


def ada_nearest_rep(ctx: Context, X: torch.Tensor, rep_idx: torch.Tensor, rep_cnt: torch.Tensor,
                    want_gamma=True, stream=None):
    """Section 2.3.  Returns (nearest_idx[B,T] int32, nearest_gamma[B,T] or None)."""
    X, B, T, d, ldx = _shape(X)
    with _on(stream, X):
        near = torch.empty((B, T), dtype=torch.int32, device=X.device)
        g = torch.empty((B, T), dtype=torch.float32, device=X.device) if want_gamma else None
    st = _fast.nearest_rep(ctx.addr, X, B, T, d, ldx, dtype_of(X), rep_idx, rep_cnt, near, g, _stream(stream))
    if st:
        _raise(st, "ada_nearest_rep")
    return near, g


def ada_attention_reps(ctx: Context, Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor,
                       rep_idx: torch.Tensor, rep_cnt: torch.Tensor, nearest_idx=None, out=None,
                       flags: int = 0, stream=None) -> torch.Tensor:
    """Section 2.3, Eq. 2: attention on the representative rows of Q, K, V (each T x h x d_h,
    bf16), expanded to every token through nearest_idx when given.  Returns out fp32 [T, h, d_h]
    (rows that receive nothing are left as they are: zeros in a fresh tensor)."""
    T, h, d_h, ld = _shape_heads(Q)
    shape, strides = Q.shape, Q.stride()
    if K.shape != shape or V.shape != shape or K.stride() != strides or V.stride() != strides:
        raise ValueError("Q, K, V must share shape and strides")
    if out is None:
        with _on(stream, Q):
            out = torch.zeros((T, h, d_h), dtype=torch.float32, device=Q.device)
    st = _fast.attention_reps(ctx.addr, Q, K, V, T, h, d_h, ld, dtype_of(Q), rep_idx, rep_cnt, nearest_idx, out,
                              out.stride(0), flags, _stream(stream))
    if st:
        _raise(st, "ada_attention_reps")
    return out


class KVCache:
    """Paged key / value cache: K and V (n_pages, h_kv, page_size, d_h) bf16, planes of one tensor or tensors of their
    own with the same page stride; table (B, pages of a sequence) int32; kmin, kmax (n_pages, h_kv, d_h) bf16, the
    bounds of every page's keys (both or neither; ada_select_blocks needs them).  The tensors are the caller's.  Of a
    table that is much wider than the longest sequence, table[:, :pages] makes ada_select_blocks faster."""

    def __init__(self, K: torch.Tensor, V: torch.Tensor, table: torch.Tensor, kmin: Optional[torch.Tensor] = None,
                 kmax: Optional[torch.Tensor] = None):
        if K.dim() != 4 or V.shape != K.shape or V.stride(0) != K.stride(0) and K.shape[0] > 1:
            raise ValueError("K and V must be (n_pages, h_kv, page_size, d_h) with the same page stride")
        n, h_kv, ps, d = K.shape
        for t in (K, V):
            if t.stride()[1:] != (ps * d, d, 1):
                raise ValueError("a page of K or V must be dense: (h_kv, page_size, d_h)")
        if table.dim() != 2 or table.stride(1) != 1:
            raise ValueError("table must be (B, pages) with unit inner stride")
        if table.shape[0] > 1 and table.stride(0) < table.shape[1]:
            raise ValueError("the rows of table must not overlap")
        _int32(table, "table")
        if (kmin is None) != (kmax is None):
            raise ValueError("kmin and kmax belong together")
        for t in (kmin, kmax):
            if t is not None and (t.shape != (n, h_kv, d) or not t.is_contiguous()):
                raise ValueError("kmin and kmax must be dense (n_pages, h_kv, d_h)")
        dtype = dtype_of(K)
        if any(t is not None and t.dtype != K.dtype for t in (V, kmin, kmax)):
            raise TypeError("K, V, kmin and kmax must have one type")
        if any(t is not None and t.device != K.device for t in (V, table, kmin, kmax)):
            raise ValueError("the cache's tensors must be on one device")
        self.K, self.V, self.table, self.kmin, self.kmax = K, V, table, kmin, kmax
        self.K_dtype, self.index = K.dtype, K.get_device()
        self.dtype, self.h_kv, self.d_h, self.page_size, self.B = dtype, h_kv, d, ps, table.shape[0]
        self._c = _KVCacheStruct(K.data_ptr(), V.data_ptr(), _ptr(kmin), _ptr(kmax), table.data_ptr(),
                                 table.stride(0) if table.shape[0] > 1 else table.shape[1], table.shape[1], n,
                                 K.stride(0) if n > 1 else h_kv * ps * d, ps, h_kv, d)
        self.addr = C.addressof(self._c)


def _int32(t: torch.Tensor, name: str, n: Optional[int] = None, device: Optional[int] = None) -> None:
    if t.dtype is not torch.int32:
        raise TypeError(f"{name} must be int32")
    if device is not None and t.get_device() != device:
        raise ValueError(f"{name} must be on the cache's device")
    if n is not None and (t.numel() < n or not t.is_contiguous()):
        raise ValueError(f"{name} must be dense with at least {n} entries")


def _elsewhere(where: str) -> None:
    """The tensors have been compared with the cache's device, and the cache with the context's."""
    raise AdaError(1, f"{where}: the cache is not on the context's device")


def _ragged(cache: KVCache, off: torch.Tensor, length: torch.Tensor) -> int:
    """Sequences of a call: off has one entry more than there are, the table and the lengths one for each."""
    B = off.numel() - 1
    if B < 1 or B > cache.B:
        raise ValueError("off must have B + 1 entries, the cache's table at least B rows")
    _int32(off, "off", B + 1, cache.index)
    _int32(length, "the lengths", B, cache.index)
    return B


def _rows_of(X: torch.Tensor, name: str, cache: KVCache, N: Optional[int] = None, heads: Optional[int] = None):
    """(N, heads, row stride) of per-token rows (N, heads, d_h), heads side by side."""
    shape, strides, d = X.shape, X.stride(), cache.d_h      # (each once: a call's checks are on the way of every token)
    if len(shape) != 3 or shape[2] != d or N is not None and shape[0] != N or heads is not None and shape[1] != heads:
        raise ValueError(f"{name} must be {'N' if N is None else N} x {'heads' if heads is None else heads} x d_h")
    if X.dtype is not cache.K_dtype:
        raise TypeError(f"{name} must have the cache's type")
    if X.get_device() != cache.index:
        raise ValueError(f"{name} must be on the cache's device")
    if strides[2] != 1 or strides[1] != d and shape[1] > 1:
        raise ValueError(f"{name} must hold the heads of a token side by side")
    return shape[0], shape[1], strides[0] if shape[0] > 1 else shape[1] * d


def ada_cache_append(ctx: Context, cache: KVCache, K: torch.Tensor, V: torch.Tensor, off: torch.Tensor,
                     length: torch.Tensor, len_out: Optional[torch.Tensor] = None, Q: Optional[torch.Tensor] = None,
                     q_out: Optional[torch.Tensor] = None, q_norm: Optional[torch.Tensor] = None,
                     k_norm: Optional[torch.Tensor] = None, eps: float = 1e-6,
                     inv_freq: Optional[torch.Tensor] = None, pos0: Optional[torch.Tensor] = None,
                     rep_idx: Optional[torch.Tensor] = None, rep_cnt: Optional[torch.Tensor] = None, flags: int = 0,
                     stream=None):
    """Appends the new tokens' keys and values (N, h_kv, d_h) behind the `length` int32[B] tokens that the sequences
    have; sequence b has rows off[b] .. off[b + 1].  Q (N, h, d_h) is normed and rotated alongside.  rep_idx, rep_cnt:
    only these tokens are kept (the lists of a selection call).  Returns (q_out or None, len_out)."""
    B = _ragged(cache, off, length)
    N, _, ldk = _rows_of(K, "K", cache, None, cache.h_kv)
    _, _, ldv = _rows_of(V, "V", cache, N, cache.h_kv)
    if len_out is None:
        len_out = _fresh(stream, length.new_empty, length, B)
    else:
        _int32(len_out, "len_out", B, cache.index)
    h = ldq = ldqo = 0
    if Q is not None:
        _, h, ldq = _rows_of(Q, "Q", cache, N)
        if q_out is None:
            q_out = _fresh(stream, Q.new_empty, Q, (N, h, cache.d_h))
            ldqo = h * cache.d_h
        else:
            _, _, ldqo = _rows_of(q_out, "q_out", cache, N, h)
    for w in (q_norm, k_norm):
        if w is not None:
            if w.dtype is not cache.K_dtype:
                raise TypeError("the norms' weights must have the cache's type")
            if w.get_device() != cache.index:
                raise ValueError("the norms' weights must be on the cache's device")
            if w.shape != (cache.d_h,) or not w.is_contiguous():
                raise ValueError("the norms' weights must be d_h dense elements")
    if inv_freq is not None:
        if inv_freq.dtype is not torch.float64 or inv_freq.dim() != 1 or not inv_freq.is_contiguous():
            raise TypeError("inv_freq must be a dense float64 vector")
        if inv_freq.get_device() != cache.index:
            raise ValueError("inv_freq must be on the cache's device")
    if pos0 is not None:
        _int32(pos0, "pos0", B, cache.index)
    if rep_idx is not None:
        _int32(rep_idx, "rep_idx", N, cache.index)
    if rep_cnt is not None:
        _int32(rep_cnt, "rep_cnt", B, cache.index)
    if cache.index != ctx.device or cache.index < 0:
        _elsewhere("ada_cache_append")
    st = _fast.cache_append(ctx.addr, cache.addr, B, off, length, len_out, N, K, ldk, V, ldv, cache.dtype, Q, h, ldq, q_out,
                            ldqo, q_norm, k_norm, eps, inv_freq, 0 if inv_freq is None else 2 * inv_freq.numel(), pos0,
                            rep_idx, rep_cnt, flags, _stream_of(ctx, stream))
    if st:
        _raise(st, "ada_cache_append")
    return q_out, len_out


def ada_attention_cached(ctx: Context, cache: KVCache, Q: torch.Tensor, off: torch.Tensor, length: torch.Tensor,
                         max_new: int, out: Optional[torch.Tensor] = None, scale: float = 0.0,
                         flags: int = ADA_ATTN_CAUSAL, stream=None) -> torch.Tensor:
    """Attention of new tokens Q (N, h, d_h) over their sequence's cache, whose `length` int32[B] counts them too;
    max_new: the most new tokens that a sequence has.  Returns out (N, h, d_h) bf16; rows behind the last sequence are
    left as they are (zeros in a fresh tensor)."""
    B = _ragged(cache, off, length)
    N, h, ldq = _rows_of(Q, "Q", cache)
    if out is None:
        out = _fresh(stream, Q.new_zeros, Q, (N, h, cache.d_h))
    _, _, ldo = _rows_of(out, "out", cache, N, h)
    if cache.index != ctx.device or cache.index < 0:
        _elsewhere("ada_attention_cached")
    st = _fast.attention_cached(ctx.addr, cache.addr, B, off, length, N, max_new, Q, h, ldq, cache.dtype, scale, out, ldo,
                                flags, _stream_of(ctx, stream))
    if st:
        _raise(st, "ada_attention_cached")
    return out


def _lists_of(cache: KVCache, N: int, blk_idx: torch.Tensor, blk_cnt: torch.Tensor, k: Optional[int] = None) -> int:
    shape = blk_idx.shape
    if len(shape) != 3 or shape[0] != N or shape[1] != cache.h_kv or k is not None and shape[2] != k:
        raise ValueError("blk_idx must be N x h_kv x k")
    _int32(blk_idx, "blk_idx", N * cache.h_kv * shape[2], cache.index)
    _int32(blk_cnt, "blk_cnt", N * cache.h_kv, cache.index)
    return shape[2]


def ada_select_blocks(ctx: Context, cache: KVCache, Q: torch.Tensor, off: torch.Tensor, length: torch.Tensor, k: int,
                      n_first: int = 1, n_last: int = 1, blk_idx: Optional[torch.Tensor] = None,
                      blk_cnt: Optional[torch.Tensor] = None, flags: int = ADA_ATTN_CAUSAL, stream=None):
    """Per new token and key head the k pages with the largest bound of q . key.  Returns (blk_idx int32 (N, h_kv, k),
    blk_cnt int32 (N, h_kv)); rows behind the last sequence are left as they are."""
    B = _ragged(cache, off, length)
    N, h, ldq = _rows_of(Q, "Q", cache)
    if blk_idx is None and blk_cnt is None:
        blk_idx = _fresh(stream, length.new_empty, length, (N, cache.h_kv, k))
        blk_cnt = _fresh(stream, length.new_empty, length, (N, cache.h_kv))
    elif blk_idx is None or blk_cnt is None:
        raise ValueError("blk_idx and blk_cnt are given together")
    else:
        _lists_of(cache, N, blk_idx, blk_cnt, k)
    if cache.index != ctx.device or cache.index < 0:
        _elsewhere("ada_select_blocks")
    st = _fast.select_blocks(ctx.addr, cache.addr, B, off, length, N, Q, h, ldq, cache.dtype, k, n_first, n_last, blk_idx,
                             blk_cnt, flags, _stream_of(ctx, stream))
    if st:
        _raise(st, "ada_select_blocks")
    return blk_idx, blk_cnt


def ada_attention_blocks(ctx: Context, cache: KVCache, Q: torch.Tensor, off: torch.Tensor, length: torch.Tensor,
                         blk_idx: torch.Tensor, blk_cnt: torch.Tensor, out: Optional[torch.Tensor] = None,
                         scale: float = 0.0, flags: int = ADA_ATTN_CAUSAL, stream=None) -> torch.Tensor:
    """ada_attention_cached over the pages that blk_idx (N, h_kv, k), blk_cnt (N, h_kv) list."""
    B = _ragged(cache, off, length)
    N, h, ldq = _rows_of(Q, "Q", cache)
    k = _lists_of(cache, N, blk_idx, blk_cnt)
    if out is None:
        out = _fresh(stream, Q.new_zeros, Q, (N, h, cache.d_h))
    _, _, ldo = _rows_of(out, "out", cache, N, h)
    if cache.index != ctx.device or cache.index < 0:
        _elsewhere("ada_attention_blocks")
    st = _fast.attention_blocks(ctx.addr, cache.addr, B, off, length, N, Q, h, ldq, cache.dtype, blk_idx, blk_cnt, k, scale,
                                out, ldo, flags, _stream_of(ctx, stream))
    if st:
        _raise(st, "ada_attention_blocks")
    return out


def ada_select_full_host(ctx: Context, X: torch.Tensor, tau: float, rep_idx: torch.Tensor,
                         rep_cnt: torch.Tensor, gamma: Optional[torch.Tensor] = None,
                         stream=None) -> None:
    """HOST tensors in and out (pinned memory recommended); returns after `stream` is idle."""
    X, B, T, d, ldx = _shape(X)
    assert not X.is_cuda and ldx == d
    _check(lib().ada_select_full_host(ctx.h, X.data_ptr(), B, T, d, dtype_of(X), float(tau),
                                      rep_idx.data_ptr(), rep_cnt.data_ptr(), _ptr(gamma),
                                      _stream(stream)), "ada_select_full_host")


def ada_cascade_step_host(ctx: Context, X: torch.Tensor, tau: float, rep_in, rep_in_cnt, rep_out,
                          rep_out_cnt, add_idx, add_cnt, rem_idx, rem_cnt, gamma_rep=None,
                          gamma_cross=None, flags: int = 0, stream=None) -> None:
    X, B, T, d, ldx = _shape(X)
    assert not X.is_cuda and ldx == d
    _check(lib().ada_cascade_step_host(ctx.h, X.data_ptr(), B, T, d, dtype_of(X), float(tau),
                                       rep_in.data_ptr(), rep_in_cnt.data_ptr(), rep_out.data_ptr(),
                                       rep_out_cnt.data_ptr(), add_idx.data_ptr(), add_cnt.data_ptr(),
                                       rem_idx.data_ptr(), rem_cnt.data_ptr(), _ptr(gamma_rep),
                                       _ptr(gamma_cross), flags, _stream(stream)),
           "ada_cascade_step_host")


def ada_select_full_noalloc(X: torch.Tensor, tau: float, rep_idx: torch.Tensor,
                            rep_cnt: torch.Tensor, gamma: Optional[torch.Tensor] = None,
                            stream=None) -> None:
    """Full selection of ONE sequence (T x d) with no context and no allocation inside the
    library: the caller passes every buffer (rep_idx: T int32, rep_cnt: 1 int32, gamma:
    optional T float32) and the library's scratch is a fixed device array, so this is the
    call for code that may not allocate device memory.  T <= ADA_NOALLOC_MAX_T; calls on
    one device must not overlap on the GPU (they share the scratch)."""
    if X.dim() == 3 and X.shape[0] == 1:
        X = X[0]
    if X.dim() != 2 or X.stride(1) != 1:
        raise ValueError("X must be T x d with unit inner stride")
    T, d = X.shape
    st = lib().ada_select_full_noalloc(X.data_ptr(), T, d, X.stride(0), dtype_of(X), float(tau),
                                       rep_idx.data_ptr(), rep_cnt.data_ptr(), _ptr(gamma),
                                       _stream(stream))
    if st == 3:
        raise AdaError(st, f"ada_select_full_noalloc: T={T} exceeds ADA_NOALLOC_MAX_T="
                           f"{ADA_NOALLOC_MAX_T}")
    _check(st, "ada_select_full_noalloc")


def ada_profile_enable(ctx: Context, on: bool) -> None:
    _check(lib().ada_profile_enable(ctx.h, int(on)), "ada_profile_enable")


def ada_profile_read(ctx: Context):
    """Returns {kernel name: (launches, total_ms)} since the last read."""
    cap = 32
    names = (C.c_char_p * cap)()
    cnt = (C.c_int64 * cap)()
    ms = (C.c_double * cap)()
    n = lib().ada_profile_read(ctx.h, names, cnt, ms, cap)
    return {names[i].decode(): (int(cnt[i]), float(ms[i])) for i in range(min(n, cap))}
