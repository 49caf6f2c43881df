"""Thin ctypes binding of libfsharp.so: the same names as include/fsharp.h, argument
marshalling only.  torch is used for device memory and streams; every step of the path
runs in the library's CUDA kernels.  There is no CPU fallback: if the library is missing
or a call fails, an exception is raised."""
from __future__ import annotations

import ctypes as C
import functools
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# FSHARP_LIB selects another build of the library (the debug build with index checks: lib/libfsharp_debug.so)
LIB_PATH = os.environ.get("FSHARP_LIB") or os.path.join(_HERE, "lib", "libfsharp.so")

FSHARP_F32, FSHARP_BF16 = 0, 1
VARIANTS = {"posrf": 0, "gerf": 1, "saderf": 2, "aderf": 3, "sderf": 4}
POOL_PER_BH, POOL_PER_HEAD = 0, 1
STAB_NONE, STAB_ROW, STAB_GROUP = 0, 1, 2
IMPL_AUTO, IMPL_SIMT, IMPL_TENSOR = 0, 1, 2

EXPORTS = [
    "fsharp_create", "fsharp_destroy", "fsharp_set_stream", "fsharp_set_impl", "fsharp_status",
    "fsharp_launch_count", "fsharp_workspace_bytes", "fsharp_strerror", "fsharp_stats_doubles",
    "fsharp_params_doubles", "fsharp_stats", "fsharp_fit_params", "fsharp_featurize", "fsharp_attend",
    "fsharp_forward_host", "fsharp_pair_estimate", "fsharp_set_timing", "fsharp_read_timing",
    "fsharp_kernel_name", "fsharp_static_scratch_bytes", "fsharp_featurize_static", "fsharp_kernel_apply",
    "fsharp_key_state_splits", "fsharp_attend_key_state", "fsharp_attend_with_state", "fsharp_attend_backward",
    "fsharp_selftest_bounded_wait", "fsharp_rotate", "fsharp_cross_scratch_bytes", "fsharp_cross_attend",
    "fsharp_cross_attend_backward",
]


class FsharpError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {strerror(code)} ({code})")


class fsharp_dims(C.Structure):
    _fields_ = [("B", C.c_int32), ("H", C.c_int32), ("Lq", C.c_int32), ("Lk", C.c_int32),
                ("d", C.c_int32), ("dv", C.c_int32), ("M", C.c_int32), ("pool", C.c_int32),
                ("q_stride", C.c_int64 * 3), ("k_stride", C.c_int64 * 3),
                ("v_stride", C.c_int64 * 3), ("y_stride", C.c_int64 * 3),
                ("omega_head_stride", C.c_int64)]


ROT_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "parts": 3}


class fsharp_rope(C.Structure):
    _fields_ = [("rot", C.c_int32), ("layout", C.c_int32), ("scaling", C.c_int32), ("reserved", C.c_int32),
                ("base", C.c_double), ("factor", C.c_double), ("original", C.c_double), ("slow", C.c_double),
                ("fast", C.c_double), ("gain", C.c_double)]


class fsharp_rotate_dims(C.Structure):
    _fields_ = [("B", C.c_int32), ("L", C.c_int32), ("H", C.c_int32), ("Hk", C.c_int32), ("d", C.c_int32),
                ("q_stride", C.c_int64 * 3), ("k_stride", C.c_int64 * 3),
                ("qo_stride", C.c_int64 * 3), ("ko_stride", C.c_int64 * 3)]


class fsharp_cross_dims(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("B", "H", "Hk", "Lq", "Lk", "d", "dv")]
                + [(n + "_stride", C.c_int64 * 3) for n in ("q", "k", "v", "y", "dy", "dq", "dk", "dv")]
                + [("mask_stride", C.c_int64)])


_lib = None


def load_library() -> C.CDLL:
    """Loads lib/libfsharp.so (built by build.py); raises if it is not there."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} not found: build it with `python -m paper_2302_00787_b200.build` "
            "(there is no fallback implementation)")
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, f32, f64 = C.c_void_p, C.c_int, C.c_int64, C.c_float, C.c_double
    dims_p = C.POINTER(fsharp_dims)
    sig = {
        "fsharp_create": (i32, [C.POINTER(vp), i32, vp]),
        "fsharp_destroy": (i32, [vp]),
        "fsharp_set_stream": (i32, [vp, vp]),
        "fsharp_set_impl": (i32, [vp, i32]),
        "fsharp_status": (i32, [vp, C.POINTER(i32)]),
        "fsharp_launch_count": (i64, [vp]),
        "fsharp_workspace_bytes": (C.c_size_t, [vp]),
        "fsharp_strerror": (C.c_char_p, [i32]),
        "fsharp_stats_doubles": (C.c_size_t, [i32]),
        "fsharp_params_doubles": (C.c_size_t, [i32]),
        "fsharp_stats": (i32, [vp, vp, vp, dims_p, i32, f32, vp]),
        "fsharp_fit_params": (i32, [vp, vp, i32, i32, i32, f64, vp]),
        "fsharp_featurize": (i32, [vp, vp, vp, vp, i32, dims_p, i32, f32, i32, vp, vp]),
        "fsharp_attend": (i32, [vp, vp, vp, vp, vp, vp, dims_p, i32, i32, i32, f32, vp]),
        "fsharp_kernel_apply": (i32, [vp, vp, vp, vp, vp, vp, f64, dims_p, i32, f32, vp]),
        "fsharp_attend_backward": (i32, [vp, vp, vp, vp, vp, vp, vp, dims_p, i32, i32, i32, f32, vp, vp, vp]),
        "fsharp_key_state_splits": (i32, [vp, dims_p]),
        "fsharp_attend_key_state": (i32, [vp, vp, vp, vp, vp, dims_p, i32, f32, vp, vp]),
        "fsharp_attend_with_state": (i32, [vp, vp, vp, vp, vp, vp, dims_p, i32, i32, f32, vp, vp, i32, vp]),
        "fsharp_forward_host": (i32, [vp, vp, vp, vp, vp, dims_p, i32, i32, i32, i32, f32, vp]),
        "fsharp_pair_estimate": (i32, [vp, vp, vp, vp, vp, i64, i32, i32, i32, vp, vp, vp]),
        "fsharp_rotate": (i32, [vp, vp, vp, vp, i64, i64, C.POINTER(fsharp_rope), vp, i32, i32, vp,
                                vp]),
        "fsharp_cross_scratch_bytes": (i64, [vp, vp, i32, i32]),
        "fsharp_cross_attend": (i32, [vp, vp, vp, vp, vp, vp, vp, i32, f32, vp, vp, vp, i64]),
        "fsharp_cross_attend_backward": (i32, [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, f32, vp,
                                               vp, vp, vp, i64]),
        "fsharp_set_timing": (i32, [vp, i32]),
        "fsharp_selftest_bounded_wait": (i32, [vp, i32]),
        "fsharp_read_timing": (i32, [vp, i32, C.POINTER(C.c_float), C.POINTER(i32)]),
        "fsharp_kernel_name": (C.c_char_p, [i32]),
        "fsharp_static_scratch_bytes": (C.c_size_t, []),
        "fsharp_featurize_static": (i32, [vp, vp, vp, vp, i32, dims_p, i32, f32, i32, vp, vp, vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def strerror(code: int) -> str:
    return load_library().fsharp_strerror(code).decode()


def stats_doubles(d: int) -> int:
    return load_library().fsharp_stats_doubles(d)


def params_doubles(d: int) -> int:
    return load_library().fsharp_params_doubles(d)


def _check(rc: int, where: str) -> None:
    if rc != 0:
        raise FsharpError(rc, where)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return FSHARP_F32
    if t.dtype == torch.bfloat16:
        return FSHARP_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _strides(t: torch.Tensor):
    """Element strides (batch, head, token) of a [B,H,L,inner] tensor, innermost contiguous."""
    if t.dim() != 4 or (t.shape[3] > 1 and t.stride(3) != 1):
        raise ValueError("expected a [B, H, L, inner] tensor whose last dimension is contiguous")
    return (C.c_int64 * 3)(t.stride(0), t.stride(1), t.stride(2))


_INNER_ONLY = {torch.float32: 3, torch.bfloat16: 7}      # element strides are multiples of 16 bytes: these bits are zero
_NO_STRIDES = (0, 0, 0)
_CROSS_DIMS = struct.Struct("=7i4x25q")                  # fsharp_cross_dims, packed
_ROTATE_DIMS = struct.Struct("=5i4x12q")                 # fsharp_rotate_dims, packed


def _place(t: torch.Tensor):
    """(t, its strides of batch, head and token, its address), or those of a dense copy where the library cannot be told
    t's: a tensor broadcast along every dimension (three zeros mean dense there) or along its tokens, rows or a start that
    are not 16-byte aligned, a last dimension with gaps.  Dimensions of size one get a dense tensor's stride: nothing
    reads it."""
    b, h, l, e = t.stride()
    low, at = _INNER_ONLY[t.dtype], t.data_ptr()
    if e == 1 and b and h and l and not (b | h | l) & low and not at & 15:
        return t, (b, h, l), at
    B, H, L, inner = t.shape
    if B * H * L * inner == 0:
        return t, (H * L * inner, L * inner, inner), at
    own = (b if B > 1 else H * L * inner, h if H > 1 else L * inner, l if L > 1 else inner)
    if (e != 1 and inner > 1) or own[2] == 0 or not any(own) or (own[0] | own[1] | own[2]) & low or at & 15:
        t = t.clone(memory_format=torch.contiguous_format)
        return t, t.stride()[:3], t.data_ptr()
    return t, own, at


def _check_written(name: str, t: torch.Tensor) -> None:
    """Refuses an output that holds one place for several values or whose last dimension has gaps."""
    if t.stride(3) != 1 and t.shape[3] > 1 or any(n > 1 and s == 0 for n, s in zip(t.shape, t.stride())):
        raise ValueError(f"{name}: expected a tensor with a contiguous last dimension and a place for every value")


def _written_place(t: torch.Tensor):
    """An output's strides of batch, head and token; those of dimensions of size one as in a dense tensor."""
    b, h, l, _ = t.stride()
    B, H, L, inner = t.shape
    return (b if B > 1 else H * L * inner, h if H > 1 else L * inner, l if L > 1 else inner)


def _new_like(t: torch.Tensor) -> torch.Tensor:
    """A new tensor of t's shape that the library can write: in t's order of dimensions where the last one is innermost, else dense."""
    g = torch.empty_like(t)                                  # (permuted like a dense tensor, else dense)
    return g if g.stride(3) == 1 else torch.empty_like(t, memory_format=torch.contiguous_format)


def make_dims(B, H, Lq, Lk, d, dv, M, pool=POOL_PER_BH, q=None, k=None, v=None, y=None,
              omega_head_stride=0) -> fsharp_dims:
    dm = fsharp_dims()
    dm.B, dm.H, dm.Lq, dm.Lk, dm.d, dm.dv, dm.M, dm.pool = B, H, Lq, Lk, d, dv, M, pool
    for name, t in (("q_stride", q), ("k_stride", k), ("v_stride", v), ("y_stride", y)):
        if t is not None:
            setattr(dm, name, _strides(t))
    dm.omega_head_stride = omega_head_stride
    return dm


def make_rope(rot, layout="half", base=10000.0, scaling="none", factor=1.0, original=0, slow=1.0, fast=32.0,
              gain=1.0) -> fsharp_rope:
    """Rotary positions of the first `rot` features of a head; the fields as in fsharp.h."""
    r = fsharp_rope()
    r.rot, r.layout, r.scaling = rot, ROT_LAYOUTS[layout], ROPE_SCALINGS[scaling]
    r.base, r.factor, r.original, r.slow, r.fast, r.gain = base, factor, original, slow, fast, gain
    return r


def _on_its_stream(call):
    """Runs a method with the context's stream as torch's current one: the copies of inputs that it makes, its scratch and
    its new outputs are then ordered on the stream that its kernels run on, as the allocator expects."""
    @functools.wraps(call)
    def issue(self, *args, **named):
        at = self._stream
        if at is None or at == torch._C._cuda_getCurrentRawStream(self.device):      # (a Stream object: 2 us more per call)
            return call(self, *args, **named)
        mine = torch.cuda.ExternalStream(at, self.device) if at else torch.cuda.default_stream(self.device)
        with torch.cuda.stream(mine):
            return call(self, *args, **named)
    return issue


class Context:
    """Owns one fsharp_ctx bound to a CUDA device and stream."""

    _stream = None               # the stream's handle

    def __init__(self, device: int = 0, stream: torch.cuda.Stream | None = None):
        self.lib = load_library()
        if not torch.cuda.is_available():
            raise RuntimeError("a CUDA device is required (no CPU implementation exists)")
        self.device = device
        self._h = C.c_void_p()
        sp = stream.cuda_stream if stream is not None else torch.cuda.current_stream(device).cuda_stream
        _check(self.lib.fsharp_create(C.byref(self._h), device, C.c_void_p(sp)), "fsharp_create")
        self._stream = sp

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            self.lib.fsharp_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- plumbing
    def set_stream(self, stream: torch.cuda.Stream):
        _check(self.lib.fsharp_set_stream(self._h, C.c_void_p(stream.cuda_stream)), "fsharp_set_stream")
        self._stream = stream.cuda_stream

    def set_impl(self, impl: int):
        _check(self.lib.fsharp_set_impl(self._h, impl), "fsharp_set_impl")

    def status(self) -> int:
        code = C.c_int(0)
        _check(self.lib.fsharp_status(self._h, C.byref(code)), "fsharp_status")
        return code.value

    def launch_count(self) -> int:
        return self.lib.fsharp_launch_count(self._h)

    def workspace_bytes(self) -> int:
        return self.lib.fsharp_workspace_bytes(self._h)

    def selftest_bounded_wait(self, limit_us: int = 1000):
        _check(self.lib.fsharp_selftest_bounded_wait(self._h, limit_us), "fsharp_selftest_bounded_wait")

    def set_timing(self, on: bool):
        _check(self.lib.fsharp_set_timing(self._h, int(on)), "fsharp_set_timing")

    def read_timing(self) -> dict:
        """{kernel name: (total milliseconds, launches)} since the last read."""
        cap = 64
        ms = (C.c_float * cap)()
        n = (C.c_int * cap)()
        _check(self.lib.fsharp_read_timing(self._h, cap, ms, n), "fsharp_read_timing")
        out = {}
        for i in range(cap):
            if n[i]:
                out[self.lib.fsharp_kernel_name(i).decode()] = (float(ms[i]), int(n[i]))
        return out

    # -- the path
    def fsharp_stats(self, Q, K, pool=POOL_PER_BH, qk_scale=1.0, out=None):
        B, H, Lq, d = Q.shape
        Lk = K.shape[2]
        dm = make_dims(B, H, Lq, Lk, d, d, 16, pool, q=Q, k=K)
        G = B * H if pool == POOL_PER_BH else H
        if out is None:
            out = torch.empty(G, stats_doubles(d), dtype=torch.float64, device=Q.device)
        _check(self.lib.fsharp_stats(self._h, Q.data_ptr(), K.data_ptr(), C.byref(dm), _dtype_code(Q),
                                     qk_scale, out.data_ptr()), "fsharp_stats")
        return out

    def fsharp_fit_params(self, stats, d, variant, ridge=0.0, out=None):
        G = stats.shape[0]
        v = VARIANTS[variant] if isinstance(variant, str) else variant
        if out is None:
            out = torch.empty(G, params_doubles(d), dtype=torch.float64, device=stats.device)
        _check(self.lib.fsharp_fit_params(self._h, stats.data_ptr(), G, d, v, ridge, out.data_ptr()),
               "fsharp_fit_params")
        return out

    def fsharp_featurize(self, X, Omega, params, side, pool=POOL_PER_BH, qk_scale=1.0, stab=STAB_ROW):
        B, H, L, d = X.shape
        M = Omega.shape[-2]
        ohs = Omega.stride(0) if Omega.dim() == 3 else 0
        dm = make_dims(B, H, L, L, d, d, M, pool, q=X, k=X, omega_head_stride=ohs)
        phi = torch.empty(B, H, L, M, dtype=torch.float32, device=X.device)
        ls = None
        if stab == STAB_ROW:
            ls = torch.empty(B, H, L, dtype=torch.float32, device=X.device)
        elif stab == STAB_GROUP:
            ls = torch.empty(B, H, dtype=torch.float32, device=X.device)
        _check(self.lib.fsharp_featurize(self._h, X.data_ptr(), Omega.data_ptr(), params.data_ptr(), side,
                                         C.byref(dm), _dtype_code(X), qk_scale, stab, phi.data_ptr(),
                                         ls.data_ptr() if ls is not None else None), "fsharp_featurize")
        return phi, ls

    def fsharp_attend(self, Q, K, V, Omega, params, causal=False, chunk=0, pool=POOL_PER_BH, qk_scale=1.0,
                      out=None):
        B, H, Lq, d = Q.shape
        Lk, dv = K.shape[2], V.shape[3]
        M = Omega.shape[-2]
        ohs = Omega.stride(0) if Omega.dim() == 3 else 0
        if out is None:
            out = torch.empty(B, H, Lq, dv, dtype=Q.dtype, device=Q.device)
        dm = make_dims(B, H, Lq, Lk, d, dv, M, pool, q=Q, k=K, v=V, y=out, omega_head_stride=ohs)
        _check(self.lib.fsharp_attend(self._h, Q.data_ptr(), K.data_ptr(), V.data_ptr(), Omega.data_ptr(),
                                      params.data_ptr(), C.byref(dm), _dtype_code(Q), int(bool(causal)), chunk,
                                      qk_scale, out.data_ptr()), "fsharp_attend")
        return out

    def fsharp_attend_backward(self, Q, K, V, dY, Omega, params, causal=False, chunk=0, pool=POOL_PER_BH,
                               qk_scale=1.0):
        """(dQ, dK, dV) for the cotangent dY of fsharp_attend's Y; each gradient has its tensor's shape and strides."""
        B, H, Lq, d = Q.shape
        Lk, dv = K.shape[2], V.shape[3]
        M = Omega.shape[-2]
        ohs = Omega.stride(0) if Omega.dim() == 3 else 0
        dQ, dK, dV = (torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device=t.device) for t in (Q, K, V))
        dm = make_dims(B, H, Lq, Lk, d, dv, M, pool, q=Q, k=K, v=V, y=dY, omega_head_stride=ohs)
        _check(self.lib.fsharp_attend_backward(self._h, Q.data_ptr(), K.data_ptr(), V.data_ptr(), dY.data_ptr(),
                                               Omega.data_ptr(), params.data_ptr(), C.byref(dm), _dtype_code(Q),
                                               int(bool(causal)), chunk, qk_scale, dQ.data_ptr(), dK.data_ptr(),
                                               dV.data_ptr()), "fsharp_attend_backward")
        return dQ, dK, dV

    def fsharp_attend_key_state(self, K, V, Omega, params, pool=POOL_PER_BH, qk_scale=1.0):
        """Key-side sums of this call's keys: (state [B*H, ns, 80, 256] fp32, shifts [B*H, ns, 2] fp32)."""
        B, H, Lk, d = K.shape
        dv, M = V.shape[3], Omega.shape[-2]
        ohs = Omega.stride(0) if Omega.dim() == 3 else 0
        dm = make_dims(B, H, Lk, Lk, d, dv, M, pool, q=K, k=K, v=V, omega_head_stride=ohs)
        ns = self.lib.fsharp_key_state_splits(self._h, C.byref(dm))
        _check(min(ns, 0), "fsharp_key_state_splits")
        state = torch.empty(B * H, ns, 80, 256, dtype=torch.float32, device=K.device)
        shifts = torch.empty(B * H, ns, 2, dtype=torch.float32, device=K.device)
        _check(self.lib.fsharp_attend_key_state(self._h, K.data_ptr(), V.data_ptr(), Omega.data_ptr(), params.data_ptr(),
                                                C.byref(dm), _dtype_code(K), qk_scale, state.data_ptr(),
                                                shifts.data_ptr()), "fsharp_attend_key_state")
        return state, shifts

    def fsharp_attend_with_state(self, Q, K, V, Omega, params, states, shifts, causal=False, pool=POOL_PER_BH,
                                 qk_scale=1.0, out=None):
        """Attention of Q over the keys behind `states` (and, causal, over K, V under the mask).  states
        [B*H, n, 80, 256] and shifts [B*H, n, 2] fp32 contiguous, or None (causal only: nothing precedes)."""
        B, H, Lq, d = Q.shape
        M = Omega.shape[-2]
        ohs = Omega.stride(0) if Omega.dim() == 3 else 0
        n = 0 if states is None else states.shape[1]
        if n:
            if not (states.is_contiguous() and shifts.is_contiguous() and states.dtype == torch.float32
                    and shifts.dtype == torch.float32 and tuple(states.shape) == (B * H, n, 80, 256)
                    and tuple(shifts.shape) == (B * H, n, 2)):
                raise ValueError("states / shifts: contiguous fp32 [B*H, n, 80, 256] / [B*H, n, 2]")
        dv = V.shape[3] if V is not None else 64
        if out is None:
            out = torch.empty(B, H, Lq, dv, dtype=Q.dtype, device=Q.device)
        if causal:
            dm = make_dims(B, H, Lq, K.shape[2], d, dv, M, pool, q=Q, k=K, v=V, y=out, omega_head_stride=ohs)
        else:
            dm = make_dims(B, H, Lq, Lq, d, dv, M, pool, q=Q, k=Q, v=out, y=out, omega_head_stride=ohs)
        _check(self.lib.fsharp_attend_with_state(
            self._h, Q.data_ptr(), K.data_ptr() if causal else None, V.data_ptr() if causal else None, Omega.data_ptr(),
            params.data_ptr(), C.byref(dm), _dtype_code(Q), int(bool(causal)), qk_scale,
            states.data_ptr() if n else None, shifts.data_ptr() if n else None, n, out.data_ptr()),
            "fsharp_attend_with_state")
        return out

    def fsharp_kernel_apply(self, X, Y, Cmat, Omega, params, alpha=0.0, pool=POOL_PER_BH, qk_scale=1.0, out=None):
        B, H, Lq, d = X.shape
        Lk, dv = Y.shape[2], Cmat.shape[3]
        M = Omega.shape[-2]
        ohs = Omega.stride(0) if Omega.dim() == 3 else 0
        if out is None:
            out = torch.empty(B, H, Lq, dv, dtype=X.dtype, device=X.device)
        dm = make_dims(B, H, Lq, Lk, d, dv, M, pool, q=X, k=Y, v=Cmat, y=out, omega_head_stride=ohs)
        _check(self.lib.fsharp_kernel_apply(self._h, X.data_ptr(), Y.data_ptr(), Cmat.data_ptr(), Omega.data_ptr(),
                                            params.data_ptr(), float(alpha), C.byref(dm), _dtype_code(X), qk_scale,
                                            out.data_ptr()), "fsharp_kernel_apply")
        return out

    def _mine(self, **named):
        """Refuses tensors that are not on this context's device: the library reads through their pointers unchecked."""
        for name, t in named.items():
            if t is not None and t.get_device() != self.device:
                raise ValueError(f"{name}: expected a tensor on cuda:{self.device}, got {t.device}")

    @_on_its_stream
    def fsharp_rotate(self, Q, K, rope, pos=None, pos0=0, transpose=False, out=None):
        """Rotary positions (make_rope) on Q [B,H,L,d] and K [B,Hk,L,d] (K may be None): (Q', K').  pos: int64 [B,L] or
        [L], None for 0 .. L-1; pos0 is added to it.  transpose: the gradient.  out: a pair of tensors to write, the first
        may be Q and the second K (the other way round is refused); the default is new dense ones, of the context's stream."""
        here = self.device
        if Q.get_device() != here or (K is not None and K.get_device() != here) or (pos is not None and pos.get_device() != here):
            self._mine(Q=Q, K=K, pos=pos)
        dt = _dtype_code(Q)
        B, H, L, d = shape = Q.shape
        Hk, pos_at, pos_stride = 0, None, 0
        if K is not None:
            Bk, Hk, Lk, dk = K.shape
            if Bk != B or Lk != L or dk != d or K.dtype != Q.dtype:
                raise ValueError(f"K: expected {(B, 'Hk', L, d)} of {Q.dtype}, got {tuple(K.shape)} of {K.dtype}")
        if pos is not None:
            if pos.dtype != torch.int64 or tuple(pos.shape) not in ((B, L), (L,)) or (L > 1 and pos.stride(-1) != 1):
                raise ValueError("pos: expected int64 [B, L] or [L] whose last dimension is contiguous")
            pos_at, pos_stride = pos.data_ptr(), pos.stride(0) if pos.dim() == 2 else 0
        if out is None:
            Qo, so = Q.new_empty(shape), (H * L * d, L * d, d)
            Ko, sz = (None, _NO_STRIDES) if K is None else (K.new_empty(K.shape), (Hk * L * d, L * d, d))
        else:
            Qo, Ko = out
            self._mine(out=Qo, out_k=Ko)
            for x, y in ((Q, Qo), (K, Ko)):
                if x is not None:
                    if y is None or y.shape != x.shape or y.dtype != x.dtype:
                        raise ValueError("out: expected the shapes and type of Q and K")
                    _check_written("out", y)
            so, sz = _written_place(Qo), _NO_STRIDES if K is None else _written_place(Ko)
        Q, sq, q_at = _place(Q)
        sk, k_at, ko_at = _NO_STRIDES, None, None
        if K is not None:
            K, sk, k_at = _place(K)
            ko_at = Ko.data_ptr()
        rc = self.lib.fsharp_rotate(self._h, q_at, k_at, pos_at, pos_stride, pos0, rope,
                                    _ROTATE_DIMS.pack(B, L, H, Hk, d, *sq, *sk, *so, *sz), dt, 1 if transpose else 0,
                                    Qo.data_ptr(), ko_at)
        if rc:
            raise FsharpError(rc, "fsharp_rotate")
        return Qo, Ko

    def _cross_check(self, Q, K, V, key_len, key_mask):
        """The sizes (B, H, Hk, Lq, Lk, d, dv), the lengths' and the mask's address and the mask's stride of a cross attention,
        its tensors checked."""
        here, t = self.device, Q.dtype
        if Q.get_device() != here or K.get_device() != here or V.get_device() != here:
            self._mine(Q=Q, K=K, V=V)
        B, H, Lq, d = Q.shape
        Bk, Hk, Lk, dk = K.shape
        Bv, Hv, Lv, dv = V.shape
        if Bk != B or Bv != B or dk != d or Hv != Hk or Lv != Lk or K.dtype != t or V.dtype != t:
            raise ValueError(f"Q {tuple(Q.shape)} {Q.dtype}, K {tuple(K.shape)} {K.dtype}, V {tuple(V.shape)} {V.dtype}: expected "
                             "[B,H,Lq,d], [B,Hk,Lk,d], [B,Hk,Lk,dv] of one type")
        len_at = mask_at = None
        mask_stride = 0
        if key_len is not None:
            self._mine(key_len=key_len)
            if key_len.dtype != torch.int32 or tuple(key_len.shape) != (B,) or not key_len.is_contiguous():
                raise ValueError("key_len: expected a contiguous int32 [B] tensor")
            len_at = key_len.data_ptr()
        if key_mask is not None:
            self._mine(key_mask=key_mask)
            if key_mask.dtype not in (torch.bool, torch.uint8) or tuple(key_mask.shape) not in ((B, Lk), (Lk,)) \
                    or (Lk > 1 and key_mask.stride(-1) != 1):
                raise ValueError("key_mask: expected bool or uint8 [B, Lk] or [Lk] whose last dimension is contiguous")
            mask_at, mask_stride = key_mask.data_ptr(), key_mask.stride(0) if key_mask.dim() == 2 else 0
        return (B, H, Hk, Lq, Lk, d, dv), len_at, mask_at, mask_stride

    def _cross_scratch(self, dims, dtype, backward, device):
        """The call's scratch: a tensor of its own each time, so that the allocator orders its reuse on the stream and a
        captured graph keeps it in its pool."""
        n = self.lib.fsharp_cross_scratch_bytes(self._h, dims, dtype, backward)
        if n <= 0:
            _check(n, "fsharp_cross_scratch_bytes")
            return None, None, 0
        t = torch.empty(n, dtype=torch.uint8, device=device)
        return t, t.data_ptr(), n

    @_on_its_stream
    def fsharp_cross_attend(self, Q, K, V, scale=None, key_len=None, key_mask=None, want_lse=False, out=None):
        """Exact softmax attention of Q [B,H,Lq,d] to K [B,Hk,Lk,d], V [B,Hk,Lk,dv]: Y, or (Y, lse [B,H,Lq] float32) with
        want_lse.  scale: d^-1/2 if None.  key_len: int32 [B].  key_mask: bool or uint8 [B,Lk] or [Lk], true where a key
        is seen."""
        dt = _dtype_code(Q)
        sizes, len_at, mask_at, mask_stride = self._cross_check(Q, K, V, key_len, key_mask)
        B, H, _, Lq, _, d, dv = sizes
        if out is None:
            out, so = Q.new_empty((B, H, Lq, dv)), (H * Lq * dv, Lq * dv, dv)
        else:
            self._mine(out=out)
            if tuple(out.shape) != (B, H, Lq, dv) or out.dtype != Q.dtype:
                raise ValueError(f"out: expected {(B, H, Lq, dv)} of {Q.dtype}")
            _check_written("out", out)
            so = _written_place(out)
        (Q, sq, q_at), (K, sk, k_at), (V, sv, v_at) = _place(Q), _place(K), _place(V)
        lse = Q.new_empty((B, H, Lq), dtype=torch.float32) if want_lse else None
        dims = _CROSS_DIMS.pack(*sizes, *sq, *sk, *sv, *so, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, mask_stride)
        scratch, at, n = self._cross_scratch(dims, dt, 0, Q.device)
        rc = self.lib.fsharp_cross_attend(self._h, q_at, k_at, v_at, len_at, mask_at, dims, dt, d ** -0.5 if scale is None else scale,
                                          out.data_ptr(), lse.data_ptr() if want_lse else None, at, n)
        if rc:
            raise FsharpError(rc, "fsharp_cross_attend")
        return (out, lse) if want_lse else out

    @_on_its_stream
    def fsharp_cross_attend_backward(self, Q, K, V, Y, lse, dY, scale=None, key_len=None, key_mask=None):
        """(dQ, dK, dV) for the cotangent dY of fsharp_cross_attend's Y, with the Y and lse of that call; each gradient is a
        new tensor with its tensor's shape and, where those give every value a place of its own and the last dimension is innermost,
        its order of dimensions; otherwise (keys stored as [B,Hk,d,Lk], say) a dense one."""
        dt = _dtype_code(Q)
        sizes, len_at, mask_at, mask_stride = self._cross_check(Q, K, V, key_len, key_mask)
        self._mine(Y=Y, lse=lse, dY=dY)
        B, H, _, Lq, _, d, dv = sizes
        for name, t in (("Y", Y), ("dY", dY)):
            if tuple(t.shape) != (B, H, Lq, dv) or t.dtype != Q.dtype:
                raise ValueError(f"{name}: expected {(B, H, Lq, dv)} of {Q.dtype}")
        if tuple(lse.shape) != (B, H, Lq) or lse.dtype != torch.float32 or not lse.is_contiguous():
            raise ValueError(f"lse: expected a contiguous float32 tensor of shape {(B, H, Lq)}")
        dQ, dK, dV = _new_like(Q), _new_like(K), _new_like(V)
        (Q, sq, q_at), (K, sk, k_at), (V, sv, v_at), (Y, sy, y_at), (dY, sg, g_at) = (_place(t) for t in (Q, K, V, Y, dY))
        dims = _CROSS_DIMS.pack(*sizes, *sq, *sk, *sv, *sy, *sg, *_written_place(dQ), *_written_place(dK), *_written_place(dV),
                                mask_stride)
        scratch, at, n = self._cross_scratch(dims, dt, 1, Q.device)
        rc = self.lib.fsharp_cross_attend_backward(
            self._h, q_at, k_at, v_at, y_at, lse.data_ptr(), g_at, len_at, mask_at, dims, dt, d ** -0.5 if scale is None else scale,
            dQ.data_ptr(), dK.data_ptr(), dV.data_ptr(), at, n)
        if rc:
            raise FsharpError(rc, "fsharp_cross_attend_backward")
        return dQ, dK, dV

    def fsharp_forward_host(self, Q, K, V, Omega, variant, causal=False, chunk=0, pool=POOL_PER_BH,
                            qk_scale=1.0, out=None):
        """Q, K, V, Omega, out: HOST tensors (dense; pinned memory recommended)."""
        for t in (Q, K, V, Omega):
            if t.is_cuda or not t.is_contiguous():
                raise ValueError("fsharp_forward_host takes dense host tensors")
        B, H, Lq, d = Q.shape
        Lk, dv = K.shape[2], V.shape[3]
        M = Omega.shape[0]
        if out is None:
            out = torch.empty(B, H, Lq, dv, dtype=Q.dtype).pin_memory()
        dm = make_dims(B, H, Lq, Lk, d, dv, M, pool)
        v = VARIANTS[variant] if isinstance(variant, str) else variant
        _check(self.lib.fsharp_forward_host(self._h, Q.data_ptr(), K.data_ptr(), V.data_ptr(), Omega.data_ptr(),
                                            C.byref(dm), _dtype_code(Q), v, int(bool(causal)), chunk, qk_scale,
                                            out.data_ptr()), "fsharp_forward_host")
        return out

    def fsharp_pair_estimate(self, X, Y, Omega, params, want_variance=True, want_pooled=False, est=None):
        """Returns (est [R, npairs], var_cf [npairs] or None) and, with want_pooled, a third item: a float64
        tensor [2] = (pooled empirical, pooled closed-form) relative variance."""
        npairs, d = X.shape
        R, M = Omega.shape[0], Omega.shape[1]
        if est is None:
            est = torch.empty(R, npairs, dtype=torch.float32, device=X.device)
        var = torch.empty(npairs, dtype=torch.float64, device=X.device) if (want_variance or want_pooled) else None
        pooled = torch.empty(2, dtype=torch.float64, device=X.device) if want_pooled else None
        _check(self.lib.fsharp_pair_estimate(self._h, X.data_ptr(), Y.data_ptr(), Omega.data_ptr(),
                                             params.data_ptr(), npairs, d, M, R, est.data_ptr(),
                                             var.data_ptr() if var is not None else None,
                                             pooled.data_ptr() if pooled is not None else None), "fsharp_pair_estimate")
        return (est, var, pooled) if want_pooled else (est, var)


def static_scratch_bytes() -> int:
    return load_library().fsharp_static_scratch_bytes()


def fsharp_featurize_static(X, Omega, params, side, phi, logscale=None, pool=POOL_PER_BH, qk_scale=1.0,
                            stab=STAB_ROW, stream=None, device_status=None) -> int:
    """The feature map without any device allocation by the library: the caller supplies the
    outputs (phi [B,H,L,M] float32, logscale as for fsharp_featurize) and the library's fixed
    in-module scratch is used.  Returns the C return code instead of raising, so a caller can
    test for the size limit (-10)."""
    lib = load_library()
    B, H, L, d = X.shape
    M = Omega.shape[-2]
    ohs = Omega.stride(0) if Omega.dim() == 3 else 0
    dm = make_dims(B, H, L, L, d, d, M, pool, q=X, k=X, omega_head_stride=ohs)

    # the kernels write through these pointers unchecked: refuse anything they would overrun
    def need(t, name, dtype, shape):
        if t.device != X.device or t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous():
            raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {shape} on {X.device}")
    need(phi, "phi", torch.float32, (B, H, L, M))
    if stab == STAB_ROW:
        if logscale is not None:
            need(logscale, "logscale", torch.float32, (B, H, L))
    elif stab == STAB_GROUP:
        if logscale is not None:
            need(logscale, "logscale", torch.float32, (B, H))
    if device_status is not None:
        need(device_status, "device_status", torch.int32, (1,))
    sp = stream.cuda_stream if stream is not None else torch.cuda.current_stream(X.device).cuda_stream
    with torch.cuda.device(X.device):          # the entry point launches on the current device
        return lib.fsharp_featurize_static(
            C.c_void_p(sp), X.data_ptr(), Omega.data_ptr(), params.data_ptr(), side, C.byref(dm), _dtype_code(X),
            qk_scale, stab, phi.data_ptr(), logscale.data_ptr() if logscale is not None else None,
            device_status.data_ptr() if device_status is not None else None)


def unpack_params(blob: torch.Tensor, d: int):
    """Splits one group's parameter blob (a 1-D float64 tensor or array) into named pieces."""
    b = blob.detach().cpu().numpy() if isinstance(blob, torch.Tensor) else blob
    dd = d * d
    t = b[5 * dd:]
    return {"A": b[0:dd].reshape(d, d), "B1": b[dd:2 * dd].reshape(d, d), "B2": b[2 * dd:3 * dd].reshape(d, d),
            "C1": b[3 * dd:4 * dd].reshape(d, d), "C2": b[4 * dd:5 * dd].reshape(d, d),
            "logD": float(t[0]), "objective": float(t[1]), "phi": float(t[2])}


def pack_params(p: dict, d: int):
    """Builds a parameter blob (numpy float64) from matrices A, B1, B2, C1, C2 and logD."""
    import numpy as np
    out = np.zeros(5 * d * d + 8, dtype=np.float64)
    for i, k in enumerate(("A", "B1", "B2", "C1", "C2")):
        out[i * d * d:(i + 1) * d * d] = np.asarray(p[k], dtype=np.float64).reshape(-1)
    t = out[5 * d * d:]
    t[0] = p["logD"]
    t[1] = p.get("objective", 0.0)
    return out
