"""Python binding of ``libqgemm.so``, the gfx950 block-quantised prefill GEMM library.

Argument marshalling only: every step runs in the library's HIP kernels.
PyTorch provides device memory and the current HIP stream. The C entry points
and their contracts are declared in ``include/qgemm.h``; the Python functions
carry the same names without the ``qgemm_`` prefix.

The library must be built (``python -m paper_2607_19438_amd.build``); there is
no fallback path, and a missing library raises ``QGemmError``.

The serving functions' checks and allocations also exist compiled (``csrc/binding.cpp``, built
beside the library): a call with good arguments on the current device goes that way where it
is there and fits the library and torch. It answers ``NotImplemented`` to any other, and the code here says what is wrong.
"""
from __future__ import annotations

import ctypes
import functools
import os
import warnings

import torch  # imported before the library so that both share one HIP runtime

__all__ = ["Q8", "Q4", "QGemmError", "lib", "lib_path", "dense", "moe", "moe_noalloc", "moe_bucket", "moe_grouped",
           "moe_gate_up_swiglu", "moe_down_combine", "swiglu", "moe_combine", "attention_prefill", "probe_mfma_clock", "last_error", "release", "version", "EXPORTS", "ExpertTable",
           "KvPlan", "kv_plan", "rope_frequencies", "rope", "kv4_cache_shape", "kv4_store", "kv4_load", "attention_packed", "attention_kv4",
           "attention_kv4_shared", "beam_select", "KvReorder", "kv_reorder", "kv4_copy", "adapters"]

Q8 = 0
Q4 = 1
_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libqgemm.so")

_vp = ctypes.c_void_p
_i = ctypes.c_int
_l = ctypes.c_int64
_d = ctypes.c_double
_f = ctypes.c_float
# name -> (restype, argtypes); mirrors include/qgemm.h
EXPORTS = {
    "qgemm_dense": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _i, _vp]),
    "qgemm_moe": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _vp]),
    "qgemm_moe_noalloc": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _vp]),
    "qgemm_moe_bucket": (_i, [_vp, _vp, _vp, _i, _i, _vp]),
    "qgemm_moe_grouped": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _vp]),
    "qgemm_moe_gate_up_swiglu": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _vp]),
    "qgemm_moe_down_combine": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _vp]),
    "qgemm_swiglu": (_i, [_vp, _vp, _i, _i, _vp]),
    "qgemm_moe_combine": (_i, [_vp, _vp, _vp, _i, _i, _i, _vp]),
    "qgemm_attention_prefill": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, ctypes.c_float, _i, _vp]),
    "qgemm_kv_plan": (_i, [_vp] * 9 + [_i] * 5 + [_vp]),
    "qgemm_rope_frequencies": (_i, [ctypes.POINTER(_d), ctypes.POINTER(_f), _i, _d, _i, _d, _d, _d, _d]),
    "qgemm_rope": (_i, [_vp, _i, _vp, _vp, _vp, _i, _i, _i, _i, _i, _l, _l, _i, _f, _vp]),
    "qgemm_kv4_store": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _l, _l, _i, _i, _vp]),
    "qgemm_kv4_load": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _vp]),
    "qgemm_attention_packed": (_i, [_vp] * 5 + [_i] * 5 + [_l] * 4 + [_f, _vp]),
    "qgemm_attention_kv4": (_i, [_vp] * 7 + [_l] + [_i] * 8 + [_l, _f, _vp]),
    "qgemm_attention_kv4_workspace": (_i, [_i] * 7 + [ctypes.POINTER(_l)]),
    "qgemm_attention_kv4_shared": (_i, [_vp] * 9 + [_l] + [_i] * 9 + [_l, _f, _vp]),
    "qgemm_attention_kv4_shared_workspace": (_i, [_i] * 8 + [ctypes.POINTER(_l)]),
    "qgemm_beam_select": (_i, [_vp, _i] + [_vp] * 6 + [_l] + [_i] * 4 + [_l, _i, _vp]),
    "qgemm_beam_select_workspace": (_i, [_i] * 4 + [ctypes.POINTER(_l)]),
    "qgemm_kv_reorder": (_i, [_vp] * 13 + [_l] + [_i] * 6 + [_vp]),
    "qgemm_kv_reorder_workspace": (_i, [_i] * 3 + [ctypes.POINTER(_l)]),
    "qgemm_kv4_copy": (_i, [_vp] * 3 + [_i] * 5 + [_vp]),
    "qgemm_adapters": (_i, [_vp] * 8 + [_l] + [_i] * 6 + [_l, _l, _vp]),
    "qgemm_adapters_workspace": (_i, [_i] * 4 + [ctypes.POINTER(_l)]),
    "qgemm_probe_mfma_clock": (_i, [_i, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double), _vp]),
    "qgemm_last_error": (ctypes.c_char_p, []),
    "qgemm_release": (_i, []),
    "qgemm_version": (_i, []),
}


class QGemmError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"qgemm error {code}: {msg}")
        self.code = code


_lib = None
_fast = None      # the compiled way of the serving functions, once the library is loaded


def lib_path() -> str:
    return _LIB_PATH


def lib():
    """Load ``libqgemm.so`` (once) and declare every exported symbol's signature."""
    global _lib, _fast
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise QGemmError(-4, f"{_LIB_PATH} is not built; run `python -m paper_2607_19438_amd.build`")
        way = _compiled_way()
        handle = ctypes.CDLL(_LIB_PATH)
        for name, (res, args) in EXPORTS.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        if way is not None and _header_of(handle) != way.header:
            way = _no_compiled_way("it was built from another header than the library")
        if way is not None:
            names = ("kv_plan", "rope", "kv4_store", "kv4_load", "attention_packed", "attention_kv4", "attention_kv4_workspace",
                     "attention_kv4_shared", "attention_kv4_shared_workspace", "beam_select", "beam_select_workspace", "kv_reorder",
                     "kv_reorder_workspace", "kv4_copy", "adapters", "adapters_workspace")
            way.bind(_raw_stream, *[ctypes.cast(getattr(handle, "qgemm_" + n), ctypes.c_void_p).value for n in names])
        _lib = handle
        _fast = way
    return _lib


def _compiled_way():
    """The serving functions' compiled way, if it is built. Loaded ahead of the library: in the other order each of its
    calls was measured 0.5 us longer (rope 4.6, not 4.1; plan 5.4, not 4.9), in every process."""
    if _raw_stream is None or not os.path.exists(os.path.join(_HERE, "_binding.so")):
        return None
    try:
        from . import _binding
    except ImportError as e:
        return _no_compiled_way(str(e))
    built_for = getattr(_binding, "torch", None)
    return _binding if built_for == torch.__version__ else _no_compiled_way(f"it was built for torch {built_for}, not {torch.__version__}")


def _no_compiled_way(why: str):
    """A binding that is there and does not fit: the library's functions all work without it, the serving ones slower."""
    warnings.warn(f"_binding.so is not used: {why}; run `python -m paper_2607_19438_amd.build`", RuntimeWarning, stacklevel=4)


def _header_of(handle):
    """The stamp of the header that a library was built from."""
    try:
        return (ctypes.c_char * 17).in_dll(handle, "qgemm_header").value.decode()
    except ValueError:
        return None


def _check(rc: int):
    if rc != 0:
        raise QGemmError(rc, lib().qgemm_last_error().decode())


# The current stream's handle without building a torch.cuda.Stream object; with _need's single pass over
# cheap accessors a bucketing call takes 4.2 us of host time instead of 6.7.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(t: torch.Tensor):
    if _raw_stream is not None:
        return _raw_stream(t.get_device())
    return torch.cuda.current_stream(t.device).cuda_stream


def _need(t: torch.Tensor, name: str, dtypes, ndim=None):
    # what is wrong is looked up only when something is
    if isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in dtypes and t.is_contiguous() and (
            ndim is None or t.dim() == ndim):
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be a GPU tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} has dtype {t.dtype}, expected one of {dtypes}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if ndim is not None and t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dimensions")


_W_DTYPES = (torch.int8, torch.uint8)


def _wshape_k(wq: torch.Tensor, fmt: int) -> int:
    return wq.shape[-1] if fmt == Q8 else wq.shape[-1] * 2


def version() -> int:
    return lib().qgemm_version()


def last_error() -> str:
    return lib().qgemm_last_error().decode()


def release():
    _check(lib().qgemm_release())


def dense(x: torch.Tensor, wq: torch.Tensor, scales: torch.Tensor, fmt: int, out: torch.Tensor | None = None):
    """``y[M][N] = x[M][K] . dequant(wq, scales)^T`` in fp32 (``qgemm_dense``)."""
    _need(x, "x", (torch.bfloat16,), 2)
    _need(wq, "wq", _W_DTYPES, 2)
    _need(scales, "scales", (torch.float16,), 2)
    M, K = x.shape
    N = wq.shape[0]
    if _wshape_k(wq, fmt) != K or scales.shape != (N, K // 32):
        raise ValueError("x, wq and scales disagree on N or K")
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=x.device)
    _need(out, "out", (torch.float32,), 2)
    if out.shape != (M, N):
        raise ValueError("out must be [M][N]")
    _check(lib().qgemm_dense(x.data_ptr(), wq.data_ptr(), scales.data_ptr(), out.data_ptr(), M, N, K, fmt,
                             _stream(x)))
    return out


class ExpertTable:
    """Validated per-expert weights with their host pointer arrays, built once and reused.

    ``wq`` / ``scales``: lists of E tensors or stacked ``[E, N, K']`` / ``[E, N, K/32]`` tensors.
    """

    def __init__(self, wq, scales, fmt: int):
        if isinstance(wq, torch.Tensor):
            wq = list(wq.unbind(0))
        if isinstance(scales, torch.Tensor):
            scales = list(scales.unbind(0))
        if len(wq) != len(scales) or not wq:
            raise ValueError("need one weight and one scale tensor per expert")
        for t in wq:
            _need(t, "wq[e]", _W_DTYPES, 2)
        for t in scales:
            _need(t, "scales[e]", (torch.float16,), 2)
        self.E = len(wq)
        self.N = wq[0].shape[0]
        self.K = _wshape_k(wq[0], fmt)
        self.fmt = fmt
        if any(w.shape[0] != self.N or _wshape_k(w, fmt) != self.K for w in wq) or any(
                s.shape != (self.N, self.K // 32) for s in scales):
            raise ValueError("expert weights disagree on N or K")
        self.wq, self.scales = wq, scales          # keep the tensors alive
        self.wp = (ctypes.c_void_p * self.E)(*[t.data_ptr() for t in wq])
        self.sp = (ctypes.c_void_p * self.E)(*[t.data_ptr() for t in scales])


def _expert_tables(wq, scales, E, fmt=None):
    """Host arrays of per-expert device pointers from lists or stacked [E, ...] tensors."""
    if isinstance(wq, ExpertTable):
        if wq.E != E:
            raise ValueError("expert table has the wrong number of experts")
        return wq.wq, wq.scales, wq.wp, wq.sp
    if isinstance(wq, torch.Tensor):
        wq = list(wq.unbind(0))
    if isinstance(scales, torch.Tensor):
        scales = list(scales.unbind(0))
    if len(wq) != E or len(scales) != E:
        raise ValueError("need one weight and one scale tensor per expert")
    for t in wq:
        _need(t, "wq[e]", _W_DTYPES, 2)
    for t in scales:
        _need(t, "scales[e]", (torch.float16,), 2)
    wp = (ctypes.c_void_p * E)(*[t.data_ptr() for t in wq])
    sp = (ctypes.c_void_p * E)(*[t.data_ptr() for t in scales])
    return wq, scales, wp, sp


def moe(x, token_expert_idx, expert_offsets, wq, scales, topk: int, fmt: int, out=None):
    """MoE expert GEMM over token slots (``qgemm_moe``): ``y[T*topk][N]`` fp32 in slot order.

    ``wq`` may be an ExpertTable (then ``scales`` is ignored)."""
    _need(x, "x", (torch.bfloat16,), 2)
    _need(token_expert_idx, "token_expert_idx", (torch.int32,), 1)
    _need(expert_offsets, "expert_offsets", (torch.int32,), 1)
    T, K = x.shape
    E = expert_offsets.shape[0] - 1
    wq, scales, wp, sp = _expert_tables(wq, scales, E)
    N = wq[0].shape[0]
    if token_expert_idx.shape[0] != T * topk:
        raise ValueError("token_expert_idx must have T*topk entries")
    if any(_wshape_k(w, fmt) != K or w.shape[0] != N for w in wq):
        raise ValueError("expert weights disagree with x on K or with each other on N")
    if out is None:
        out = torch.empty((T * topk, N), dtype=torch.float32, device=x.device)
    _need(out, "out", (torch.float32,), 2)
    _check(lib().qgemm_moe(x.data_ptr(), token_expert_idx.data_ptr(), expert_offsets.data_ptr(), wp, sp,
                           out.data_ptr(), T, E, topk, N, K, fmt, _stream(x)))
    return out


def moe_noalloc(x, token_expert_idx, expert_offsets, wq, scales, topk: int, fmt: int, out=None):
    """``qgemm_moe_noalloc``: as ``moe`` with the bucketing buffers in the library's static device
    scratch (no device allocation in the call; ``out`` should be given by callers that cannot
    allocate). ``wq`` may be an ExpertTable."""
    _need(x, "x", (torch.bfloat16,), 2)
    _need(token_expert_idx, "token_expert_idx", (torch.int32,), 1)
    _need(expert_offsets, "expert_offsets", (torch.int32,), 1)
    T, K = x.shape
    E = expert_offsets.shape[0] - 1
    wq, scales, wp, sp = _expert_tables(wq, scales, E)
    N = wq[0].shape[0]
    if token_expert_idx.shape[0] != T * topk:
        raise ValueError("token_expert_idx must have T*topk entries")
    if out is None:
        out = torch.empty((T * topk, N), dtype=torch.float32, device=x.device)
    _need(out, "out", (torch.float32,), 2)
    _check(lib().qgemm_moe_noalloc(x.data_ptr(), token_expert_idx.data_ptr(), expert_offsets.data_ptr(), wp, sp,
                                   out.data_ptr(), T, E, topk, N, K, fmt, _stream(x)))
    return out


def moe_bucket(token_expert_idx, expert_offsets, out=None):
    """Assignments grouped by expert, stable (``qgemm_moe_bucket``)."""
    _need(token_expert_idx, "token_expert_idx", (torch.int32,), 1)
    _need(expert_offsets, "expert_offsets", (torch.int32,), 1)
    n = token_expert_idx.shape[0]
    E = expert_offsets.shape[0] - 1
    if out is None:
        out = torch.empty((n,), dtype=torch.int32, device=token_expert_idx.device)
    _need(out, "out", (torch.int32,), 1)
    _check(lib().qgemm_moe_bucket(token_expert_idx.data_ptr(), expert_offsets.data_ptr(), out.data_ptr(), n, E,
                                  _stream(token_expert_idx)))
    return out


def moe_grouped(x, perm, expert_offsets, wq, scales, topk: int, fmt: int, out=None):
    """Grouped GEMM from an existing bucketing (``qgemm_moe_grouped``); ``wq`` may be an ExpertTable."""
    _need(x, "x", (torch.bfloat16,), 2)
    _need(perm, "perm", (torch.int32,), 1)
    _need(expert_offsets, "expert_offsets", (torch.int32,), 1)
    T, K = x.shape
    E = expert_offsets.shape[0] - 1
    wq, scales, wp, sp = _expert_tables(wq, scales, E)
    N = wq[0].shape[0]
    if out is None:
        out = torch.empty((T * topk, N), dtype=torch.float32, device=x.device)
    _need(out, "out", (torch.float32,), 2)
    _check(lib().qgemm_moe_grouped(x.data_ptr(), perm.data_ptr(), expert_offsets.data_ptr(), wp, sp,
                                   out.data_ptr(), T, E, topk, N, K, fmt, _stream(x)))
    return out


def moe_gate_up_swiglu(x, perm, expert_offsets, wq, scales, topk: int, fmt: int, out=None):
    """Fused gate/up projection + SiLU gate (``qgemm_moe_gate_up_swiglu``): bf16 ``h[T*topk][inter]``.

    Expert weights are ``[2*inter][K]`` (gate rows, then up rows); ``wq`` may be an ExpertTable."""
    _need(x, "x", (torch.bfloat16,), 2)
    _need(perm, "perm", (torch.int32,), 1)
    _need(expert_offsets, "expert_offsets", (torch.int32,), 1)
    T, K = x.shape
    E = expert_offsets.shape[0] - 1
    wq, scales, wp, sp = _expert_tables(wq, scales, E)
    N = wq[0].shape[0]
    if N % 2 != 0:
        raise ValueError("gate/up weights need an even number of rows")
    inter = N // 2
    if out is None:
        out = torch.empty((T * topk, inter), dtype=torch.bfloat16, device=x.device)
    _need(out, "out", (torch.bfloat16,), 2)
    if out.shape != (T * topk, inter):
        raise ValueError("out must be [T*topk][inter]")
    _check(lib().qgemm_moe_gate_up_swiglu(x.data_ptr(), perm.data_ptr(), expert_offsets.data_ptr(), wp, sp,
                                          out.data_ptr(), T, E, topk, inter, K, fmt, _stream(x)))
    return out


def moe_down_combine(h, perm, expert_offsets, wq, scales, route_w, topk: int, fmt: int, y2=None, out=None):
    """Down projection over token slots with the router-weighted combine fused in
    (``qgemm_moe_down_combine``): returns ``(y2 [T*topk][N], out [T][N])``, both fp32.
    ``wq`` may be an ExpertTable."""
    _need(h, "h", (torch.bfloat16,), 2)
    _need(perm, "perm", (torch.int32,), 1)
    _need(expert_offsets, "expert_offsets", (torch.int32,), 1)
    _need(route_w, "route_w", (torch.float32,), 1)
    A, K = h.shape
    if A % topk != 0 or route_w.shape[0] != A:
        raise ValueError("h and route_w need T*topk rows")
    T = A // topk
    E = expert_offsets.shape[0] - 1
    wq, scales, wp, sp = _expert_tables(wq, scales, E)
    N = wq[0].shape[0]
    if any(_wshape_k(w, fmt) != K or w.shape[0] != N for w in wq):
        raise ValueError("expert weights disagree with h on K or with each other on N")
    if y2 is None:
        y2 = torch.empty((A, N), dtype=torch.float32, device=h.device)
    if out is None:
        out = torch.empty((T, N), dtype=torch.float32, device=h.device)
    _need(y2, "y2", (torch.float32,), 2)
    _need(out, "out", (torch.float32,), 2)
    if y2.shape != (A, N) or out.shape != (T, N):
        raise ValueError("y2 must be [T*topk][N] and out [T][N]")
    _check(lib().qgemm_moe_down_combine(h.data_ptr(), perm.data_ptr(), expert_offsets.data_ptr(), wp, sp,
                                        route_w.data_ptr(), y2.data_ptr(), out.data_ptr(), T, E, topk, N, K, fmt,
                                        _stream(h)))
    return y2, out


def swiglu(y1, out=None):
    """``h = bf16(silu(gate) * up)`` over ``y1 = [gate | up]`` (``qgemm_swiglu``)."""
    _need(y1, "y1", (torch.float32,), 2)
    rows, two_inter = y1.shape
    inter = two_inter // 2
    if out is None:
        out = torch.empty((rows, inter), dtype=torch.bfloat16, device=y1.device)
    _need(out, "out", (torch.bfloat16,), 2)
    _check(lib().qgemm_swiglu(y1.data_ptr(), out.data_ptr(), rows, inter, _stream(y1)))
    return out


def moe_combine(y2, route_w, topk: int, out=None):
    """``out[t] = sum_j route_w[t*topk+j] * y2[t*topk+j]`` (``qgemm_moe_combine``)."""
    _need(y2, "y2", (torch.float32,), 2)
    _need(route_w, "route_w", (torch.float32,), 1)
    A, N = y2.shape
    T = A // topk
    if out is None:
        out = torch.empty((T, N), dtype=torch.float32, device=y2.device)
    _need(out, "out", (torch.float32,), 2)
    _check(lib().qgemm_moe_combine(y2.data_ptr(), route_w.data_ptr(), out.data_ptr(), T, topk, N, _stream(y2)))
    return out


def attention_prefill(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, causal: bool = True,
                      scale: float | None = None, out: torch.Tensor | None = None):
    """``qgemm_attention_prefill``: q ``[B][S][H][D]``, k / v ``[B][S][Hkv][D]`` bf16 -> o ``[B][S][H][D]`` bf16."""
    _need(q, "q", (torch.bfloat16,), 4)
    _need(k, "k", (torch.bfloat16,), 4)
    _need(v, "v", (torch.bfloat16,), 4)
    B, S, H, D = q.shape
    if k.shape != v.shape or k.shape[0] != B or k.shape[1] != S or k.shape[3] != D:
        raise ValueError("q, k and v disagree on B, S or D")
    Hkv = k.shape[2]
    if scale is None:
        scale = 1.0 / float(D) ** 0.5
    if out is None:
        out = torch.empty_like(q)
    _need(out, "out", (torch.bfloat16,), 4)
    if out.shape != q.shape:
        raise ValueError("out must have the shape of q")
    _check(lib().qgemm_attention_prefill(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), B, S, H, Hkv, D,
                                         float(scale), int(bool(causal)), _stream(q)))
    return out


# ---------------------------------------------------------------------------
# serving: a step over a ragged batch
# ---------------------------------------------------------------------------

_I32 = (torch.int32,)
_BF16 = (torch.bfloat16,)
_F64 = (torch.float64,)
_ROWS = (torch.float32, torch.bfloat16)


def _need_rows(t: torch.Tensor, name: str, dtypes):
    """A tensor [T][heads][D] whose heads lie end to end; returns its shape and the elements between rows."""
    if isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in dtypes and t.dim() == 3:
        T, h, D = n = t.shape
        s0, s1, s2 = t.stride()
        if (s2 == 1 or D <= 1) and (s1 == D or h <= 1):
            return n, s0 if T > 1 else h * D
        raise ValueError(f"the heads of a row of {name} must be contiguous")
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} has dtype {t.dtype}, expected one of {dtypes}")
    raise ValueError(f"{name} must have 3 dimensions")


_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _device(first: torch.Tensor, *others) -> int:
    """The device that the tensors share."""
    dev = first.get_device()
    for t in others:
        if t.get_device() != dev:
            raise ValueError("the tensors must be on one device")
    return dev


def _sizes(*n):
    """Sizes that the library counts in 32 bits (ctypes would cut them)."""
    if max(n) >= 1 << 31:
        raise ValueError("a size is 2^31 or more")


def _stream_of(dev: int):
    return torch.cuda.current_stream(dev).cuda_stream if _raw_stream is None else _raw_stream(dev)


def _enqueue(fn, dev: int, *args):
    """``fn(*args, stream)`` on the current stream of device ``dev``, which is made current for the call if it is not."""
    if _current_device() == dev:
        rc = fn(*args, _stream_of(dev))
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, _stream_of(dev))
    if rc:
        _check(rc)


class KvPlan:
    """What ``kv_plan`` gives: ``cu_q`` [R+1], ``positions`` [T], ``slots`` [T], ``kv_len`` [R] (with the new
    tokens) and ``used`` [1] (pages taken from the free list), all int32 on the GPU."""

    __slots__ = ("cu_q", "positions", "slots", "kv_len", "used")

    def __init__(self, R: int, T: int, device):
        # one allocation, as the plan of a small step is all latency
        n = torch.empty(2 * R + 2 + 2 * T, dtype=torch.int32, device=device)
        self.cu_q, self.kv_len, self.used, self.positions, self.slots = n.split_with_sizes((R + 1, R, 1, T, T))


def kv_plan(kv_len, q_len, block_table, free_pages, page: int, tokens: int, out: KvPlan | None = None) -> KvPlan:
    """Slots, positions and first rows of a step's tokens, and the pages it adds to ``block_table`` (``qgemm_kv_plan``).

    ``kv_len`` / ``q_len`` [R]: tokens in the cache / new ones; ``block_table`` [R][W] is updated in place from
    ``free_pages``; ``tokens``: rows of the step, those behind the last token have slot -1. ``out``: an earlier
    plan of the same sizes to write into, with no tensor of it among the inputs: where ``kv_len`` is a plan's, ``out`` is
    another plan (two that take turns), else the call is refused."""
    if _fast is not None and out is None:
        r = _fast.kv_plan(kv_len, q_len, block_table, free_pages, page, tokens)
        if r is not NotImplemented:
            plan = KvPlan.__new__(KvPlan)
            plan.cu_q, plan.kv_len, plan.used, plan.positions, plan.slots = r
            return plan
    _need(kv_len, "kv_len", _I32, 1)
    _need(q_len, "q_len", _I32, 1)
    _need(block_table, "block_table", _I32, 2)
    _need(free_pages, "free_pages", _I32, 1)
    R = kv_len.shape[0]
    if q_len.shape[0] != R or block_table.shape[0] != R:
        raise ValueError("kv_len, q_len and block_table disagree on the number of requests")
    if not (0 <= tokens < 1 << 31 and 0 < page < 1 << 31):
        raise ValueError("tokens must be >= 0 and page > 0, both below 2^31")
    _sizes(R, block_table.shape[1], free_pages.shape[0])
    dev = _device(kv_len, q_len, block_table, free_pages)
    if out is None:
        out = KvPlan(R, tokens, kv_len.device)
    else:
        for name, n in (("cu_q", R + 1), ("positions", tokens), ("slots", tokens), ("kv_len", R), ("used", 1)):
            t = getattr(out, name)
            _need(t, "out." + name, _I32, 1)
            if t.shape[0] != n:
                raise ValueError(f"out.{name} must have {n} entries")
        _device(kv_len, out.cu_q, out.positions, out.slots, out.kv_len, out.used)
    _enqueue(lib().qgemm_kv_plan, dev, kv_len.data_ptr(), q_len.data_ptr(), block_table.data_ptr(), free_pages.data_ptr(),
             out.cu_q.data_ptr(), out.positions.data_ptr(), out.slots.data_ptr(), out.kv_len.data_ptr(), out.used.data_ptr(), R,
             block_table.shape[1], free_pages.shape[0], page, tokens)
    return out


_SCALINGS = {"none": 0, "linear": 1, "llama3": 2, "yarn": 3}


def rope_frequencies(rot: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, low: float = 1.0,
                     high: float = 0.0, length: float = 0.0, device=None):
    """``(inv_freq, gain)`` for ``rope`` (``qgemm_rope_frequencies``): float64 [rot/2] on ``device`` (the current GPU
    by default) and the factor of the sine and cosine.

    ``scaling``: "none"; "linear" (``factor``); "llama3" and "yarn" (``factor``, the original context's ``length``, and
    the turns over it up to ``low`` of which a pair is divided by ``factor`` and from ``high`` on kept)."""
    if scaling not in _SCALINGS:
        raise ValueError(f"scaling must be one of {tuple(_SCALINGS)}")
    _sizes(abs(rot))
    f = torch.empty(max(rot // 2, 1), dtype=torch.float64)
    gain = _f(1.0)
    _check(lib().qgemm_rope_frequencies(ctypes.cast(f.data_ptr(), ctypes.POINTER(_d)), ctypes.byref(gain), rot, base,
                                        _SCALINGS[scaling], factor, low, high, length))
    return f.to("cuda" if device is None else device), gain.value


def rope(x: torch.Tensor, positions: torch.Tensor, inv_freq: torch.Tensor, rot_heads: int, interleaved: bool = False,
         gain: float = 1.0, out: torch.Tensor | None = None):
    """Rotary positions on the first ``rot_heads`` heads of rows ``x`` [T][heads][D], fp32 or bf16, and their conversion
    to bf16 (``qgemm_rope``). The first ``2 * len(inv_freq)`` elements of a head are rotated, as pairs half of them
    apart or (``interleaved``) neighbouring. ``out``: bf16, may be a bf16 ``x`` itself."""
    if _fast is not None:
        r = _fast.rope(x, positions, inv_freq, rot_heads, interleaved, gain, out)
        if r is not NotImplemented:
            return r
    (T, heads, D), xs = _need_rows(x, "x", _ROWS)
    _need(positions, "positions", _I32, 1)
    _need(inv_freq, "inv_freq", _F64, 1)
    if positions.shape[0] != T:
        raise ValueError("x and positions disagree on T")
    _sizes(T, heads, D, 2 * inv_freq.shape[0])
    if not 0 <= rot_heads <= heads:
        raise ValueError("rot_heads must lie in [0, heads]")
    if out is None:
        out = torch.empty((T, heads, D), dtype=torch.bfloat16, device=x.device)
        ys = heads * D
    else:
        shape, ys = _need_rows(out, "out", _BF16)
        if shape != (T, heads, D):
            raise ValueError("out must have the shape of x")
    _enqueue(lib().qgemm_rope, _device(x, positions, inv_freq, out), x.data_ptr(), 1 if x.dtype is torch.bfloat16 else 0,
             positions.data_ptr(), inv_freq.data_ptr(), out.data_ptr(), T, heads, rot_heads, D, 2 * inv_freq.shape[0], xs, ys,
             1 if interleaved else 0, float(gain))
    return out


def kv4_cache_shape(pages: int, Hkv: int, D: int, page: int):
    """Shape of the uint8 tensor of a paged 4-bit cache: ``(pages, Hkv, page * (D + D/16))``."""
    return pages, Hkv, page * (D + D // 16)


def _cache_sizes(cache: torch.Tensor, D: int):
    _need(cache, "cache", (torch.uint8,), 3)
    pages, Hkv, record = cache.shape
    if D < 16 or record * 16 % (17 * D):
        raise ValueError(f"the cache's records of {record} bytes hold no whole number of slots of head dimension {D}")
    return pages, Hkv, record * 16 // (17 * D)


def kv4_store(k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, cache: torch.Tensor):
    """Quantises ``k``, ``v`` [T][Hkv][D] bf16 into the cache's ``slots`` [T] (``qgemm_kv4_store``); negative slots are
    skipped. ``cache``: uint8 of ``kv4_cache_shape``."""
    if _fast is not None and _fast.kv4_store(k, v, slots, cache) is None:
        return
    shape, ks = _need_rows(k, "k", _BF16)
    vshape, vs = _need_rows(v, "v", _BF16)
    _need(slots, "slots", _I32, 1)
    T, Hkv, D = shape
    pages, heads, page = _cache_sizes(cache, D)
    if vshape != shape or heads != Hkv or slots.shape[0] != T:
        raise ValueError("k, v, slots and cache disagree on T, Hkv or D")
    _sizes(T, Hkv, D, pages, page)
    _enqueue(lib().qgemm_kv4_store, _device(k, v, slots, cache), k.data_ptr(), v.data_ptr(), slots.data_ptr(), cache.data_ptr(), T, Hkv,
             D, ks, vs, pages, page)


def kv4_load(cache: torch.Tensor, slots: torch.Tensor, D: int, k: torch.Tensor | None = None, v: torch.Tensor | None = None):
    """The keys and values of the cache's ``slots`` [T] as bf16 [T][Hkv][D] each (``qgemm_kv4_load``); rows of negative
    slots are left as they are in ``k`` and ``v``."""
    if _fast is not None and k is None and v is None:
        r = _fast.kv4_load(cache, slots, D)
        if r is not NotImplemented:
            return r
    _need(slots, "slots", _I32, 1)
    pages, Hkv, page = _cache_sizes(cache, D)
    _sizes(slots.shape[0], Hkv, D, pages, page)
    shape = (slots.shape[0], Hkv, D)
    if k is None:
        k = torch.empty(shape, dtype=torch.bfloat16, device=cache.device)
    else:
        _need(k, "k", _BF16, 3)
    if v is None:
        v = torch.empty(shape, dtype=torch.bfloat16, device=cache.device)
    else:
        _need(v, "v", _BF16, 3)
    if k.shape != shape or v.shape != shape:
        raise ValueError("k and v must be [T][Hkv][D]")
    _enqueue(lib().qgemm_kv4_load, _device(cache, slots, k, v), cache.data_ptr(), slots.data_ptr(), k.data_ptr(), v.data_ptr(),
             shape[0], Hkv, D, pages, page)
    return k, v


def attention_packed(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu: torch.Tensor, scale: float | None = None,
                     out: torch.Tensor | None = None):
    """Causal attention over prompts packed end to end, prompt r in rows ``cu[r] .. cu[r+1]-1``
    (``qgemm_attention_packed``): q ``[T][H][D]``, k / v ``[T][Hkv][D]`` bf16, views of one projection row among
    them -> o ``[T][H][D]`` bf16. Rows behind the last prompt are not written."""
    if _fast is not None:
        r = _fast.attention_packed(q, k, v, cu, scale, out)
        if r is not NotImplemented:
            return r
    shape, qs = _need_rows(q, "q", _BF16)
    kshape, ks = _need_rows(k, "k", _BF16)
    vshape, vs = _need_rows(v, "v", _BF16)
    _need(cu, "cu", _I32, 1)
    T, H, D = shape
    if kshape != vshape or kshape[0] != T or kshape[2] != D:
        raise ValueError("q, k and v disagree on T or D")
    R = cu.shape[0] - 1
    _sizes(T, H, D, R, kshape[1])
    if R < 0:
        raise ValueError("cu must have one entry more than there are prompts")
    if out is None:
        out = torch.empty((T, H, D), dtype=torch.bfloat16, device=q.device)
        ys = H * D
    else:
        oshape, ys = _need_rows(out, "out", _BF16)
        if oshape != shape:
            raise ValueError("out must have the shape of q")
    _enqueue(lib().qgemm_attention_packed, _device(q, k, v, cu, out), q.data_ptr(), k.data_ptr(), v.data_ptr(), cu.data_ptr(),
             out.data_ptr(), T, R, H, kshape[1], D, qs, ks, vs, ys, D ** -0.5 if scale is None else float(scale))
    return out


@functools.lru_cache(maxsize=256)
def _kv4_workspace(*sizes) -> int:
    """Bytes of ``attention_kv4``'s workspace, which follow from the sizes alone."""
    n = _l(0)
    _check(lib().qgemm_attention_kv4_workspace(*sizes, ctypes.byref(n)))
    return n.value


def attention_kv4(q: torch.Tensor, cache: torch.Tensor, block_table: torch.Tensor, kv_len: torch.Tensor,
                  cu_q: torch.Tensor | None = None, scale: float | None = None, out: torch.Tensor | None = None):
    """Attention of new tokens over the paged 4-bit cache (``qgemm_attention_kv4``): q ``[T][H][D]`` bf16 -> o
    ``[T][H][D]`` bf16. ``kv_len`` [R]: each request's keys, the new tokens' own (stored before) among them;
    ``cu_q`` [R+1]: first rows of the requests, or None where each has one token. Rows behind the last request
    are not written."""
    if _fast is not None:
        r = _fast.attention_kv4(q, cache, block_table, kv_len, cu_q, scale, out)
        if r is not NotImplemented:
            return r
    (T, H, D), qs = _need_rows(q, "q", _BF16)
    _need(block_table, "block_table", _I32, 2)
    _need(kv_len, "kv_len", _I32, 1)
    pages, Hkv, page = _cache_sizes(cache, D)
    R, W = block_table.shape
    _sizes(T, H, D, R, W, pages, page)
    if kv_len.shape[0] != R or (cu_q is None and T != R):
        raise ValueError("q, block_table and kv_len disagree on the number of requests")
    if cu_q is not None:
        _need(cu_q, "cu_q", _I32, 1)
        if cu_q.shape[0] != R + 1:
            raise ValueError("cu_q must have one entry more than there are requests")
        _device(q, cu_q)
    if out is None:
        out = torch.empty((T, H, D), dtype=torch.bfloat16, device=q.device)
    else:
        _need(out, "out", _BF16, 3)
        if out.shape != q.shape:
            raise ValueError("out must have the shape of q")
    need = _kv4_workspace(T, R, H, Hkv, D, W, page)
    # of the call's own: torch's allocator keeps it from other streams, and inside a capture it is the graph's
    ws = torch.empty(need, dtype=torch.uint8, device=q.device)
    _enqueue(lib().qgemm_attention_kv4, _device(q, cache, block_table, kv_len, out), q.data_ptr(), cache.data_ptr(),
             block_table.data_ptr(), kv_len.data_ptr(), None if cu_q is None else cu_q.data_ptr(), out.data_ptr(),
             ws.data_ptr(), need, T, R, H, Hkv, D, W, pages, page, qs, D ** -0.5 if scale is None else float(scale))
    return out


# ---------------------------------------------------------------------------
# serving: many continuations of a prompt, many tenants
# ---------------------------------------------------------------------------

@functools.lru_cache(maxsize=1024)
def _workspace(name: str, *sizes) -> int:
    """Bytes of a call's workspace, which follow from the sizes alone."""
    n = _l(0)
    _check(getattr(lib(), f"qgemm_{name}_workspace")(*sizes, ctypes.byref(n)))
    return n.value


def attention_kv4_shared(q: torch.Tensor, cache: torch.Tensor, block_table: torch.Tensor, kv_len: torch.Tensor,
                         groups: torch.Tensor, prefix_len: torch.Tensor, cu_q: torch.Tensor | None = None,
                         scale: float | None = None, out: torch.Tensor | None = None):
    """``attention_kv4`` with the keys that the requests of a group share read once (``qgemm_attention_kv4_shared``).

    ``groups`` [G+1]: first requests of the groups; ``prefix_len`` [G]: keys that a group's requests have in common. The other
    arguments are ``attention_kv4``'s, and so are the results, but for the order of summation and the rounding of the softmax
    weights to bf16, which goes by the split of the work."""
    if _fast is not None:
        r = _fast.attention_kv4_shared(q, cache, block_table, kv_len, groups, prefix_len, cu_q, scale, out)
        if r is not NotImplemented:
            return r
    (T, H, D), qs = _need_rows(q, "q", _BF16)
    _need(block_table, "block_table", _I32, 2)
    _need(kv_len, "kv_len", _I32, 1)
    _need(groups, "groups", _I32, 1)
    _need(prefix_len, "prefix_len", _I32, 1)
    pages, Hkv, page = _cache_sizes(cache, D)
    R, W = block_table.shape
    G = prefix_len.shape[0]
    _sizes(T, H, D, R, W, G, pages, page)
    if kv_len.shape[0] != R or (cu_q is None and T != R):
        raise ValueError("q, block_table and kv_len disagree on the number of requests")
    if groups.shape[0] != G + 1:
        raise ValueError("groups must have one entry more than prefix_len")
    if cu_q is not None:
        _need(cu_q, "cu_q", _I32, 1)
        if cu_q.shape[0] != R + 1:
            raise ValueError("cu_q must have one entry more than there are requests")
        _device(q, cu_q)
    if out is None:
        out = torch.empty((T, H, D), dtype=torch.bfloat16, device=q.device)
    else:
        _need(out, "out", _BF16, 3)
        if out.shape != q.shape:
            raise ValueError("out must have the shape of q")
    need = _workspace("attention_kv4_shared", T, R, G, H, Hkv, D, W, page)
    ws = torch.empty(need, dtype=torch.uint8, device=q.device)
    _enqueue(lib().qgemm_attention_kv4_shared, _device(q, cache, block_table, kv_len, groups, prefix_len, out), q.data_ptr(),
             cache.data_ptr(), block_table.data_ptr(), kv_len.data_ptr(), None if cu_q is None else cu_q.data_ptr(), groups.data_ptr(),
             prefix_len.data_ptr(), out.data_ptr(), ws.data_ptr(), need, T, R, G, H, Hkv, D, W, pages, page, qs,
             D ** -0.5 if scale is None else float(scale))
    return out


_FLAGS = (torch.bool, torch.uint8)


def beam_select(logits: torch.Tensor, scores: torch.Tensor, count: int | None = None, finished: torch.Tensor | None = None,
                end: int = 0):
    """The ``count`` (by default as many as beams) best continuations of every request's beams (``qgemm_beam_select``):
    ``(scores, parents, tokens)``, each [R][count], fp32 and int32, best first.

    ``logits`` [R*B][V] fp32 or bf16, rows at any stride; ``scores`` [R][B] fp32, -inf for a beam that is not there;
    ``finished`` [R][B] bool or uint8: beams that go on with ``end`` at their own score. Of a beam the larger logit comes first, then
    the lower token; beams are compared by value, equal ones the lower first. Where candidates are missing the score
    is -inf, the parent -1 and the token ``end``, so that ``tokens == end`` is the next call's ``finished``."""
    if _fast is not None:
        r = _fast.beam_select(logits, scores, count, finished, end)
        if r is not NotImplemented:
            return r
    _need(scores, "scores", (torch.float32,), 2)
    R, B = scores.shape
    if not isinstance(logits, torch.Tensor):
        raise TypeError("logits must be a torch.Tensor")
    if not logits.is_cuda:
        raise ValueError("logits must be a GPU tensor")
    if logits.dtype not in _ROWS:
        raise TypeError(f"logits has dtype {logits.dtype}, expected one of {_ROWS}")
    if logits.dim() != 2 or logits.shape[0] != R * B:
        raise ValueError("logits must be [R*B][V]")
    V = logits.shape[1]
    if V > 1 and R * B and logits.stride(1) != 1:
        raise ValueError("the logits of a row must be contiguous")
    if finished is not None:
        _need(finished, "finished", _FLAGS, 2)
        if finished.shape != scores.shape:
            raise ValueError("finished must have the shape of scores")
        _device(logits, finished)
    K = B if count is None else int(count)
    _sizes(R * B, V, K, abs(int(end)))
    dev = _device(logits, scores)
    need = _workspace("beam_select", R, B, V, K)
    best, parents, tokens = torch.empty(3 * R * K, dtype=torch.int32, device=logits.device).split_with_sizes((R * K,) * 3)
    best = best.view(torch.float32)
    ws = torch.empty(need, dtype=torch.uint8, device=logits.device)
    _enqueue(lib().qgemm_beam_select, dev, logits.data_ptr(), 1 if logits.dtype is torch.bfloat16 else 0, scores.data_ptr(),
             None if finished is None else finished.data_ptr(), best.data_ptr(), parents.data_ptr(), tokens.data_ptr(), ws.data_ptr(), need,
             R, B, V, K, logits.stride(0) if R * B > 1 else V, int(end))
    return best.view(R, K), parents.view(R, K), tokens.view(R, K)


class KvReorder:
    """What ``kv_reorder`` gives: ``block_table`` [R*B][W] and ``kv_len`` [R*B] of the new rows; ``src`` and ``dst`` [R*B], the pages
    to copy (-1: none); ``used`` [1], pages taken from the free list; ``released`` [Q] and ``n_released`` [1], the
    pages that no row holds any more and their number. All int32 on the GPU."""

    __slots__ = ("block_table", "kv_len", "src", "dst", "used", "released", "n_released")

    def __init__(self, rows: int, W: int, Q: int, device):
        n = torch.empty(rows * (W + 3) + Q + 2, dtype=torch.int32, device=device)
        table, self.kv_len, self.src, self.dst, self.released, self.used, self.n_released = n.split_with_sizes((rows * W, rows, rows, rows, Q, 1, 1))
        self.block_table = table.view(rows, W)


def kv_reorder(block_table: torch.Tensor, kv_len: torch.Tensor, parents: torch.Tensor, free_pages: torch.Tensor, page: int,
               keep: torch.Tensor | None = None, released: int | None = None, out: KvReorder | None = None) -> KvReorder:
    """Block tables of the beams after a selection (``qgemm_kv_reorder``).

    ``block_table`` [R*B][W], ``kv_len`` [R*B]: the old rows; ``parents`` [R][B]: the old row, within the request, that each new
    one continues, or -1; ``free_pages``: where second children of a partly filled page get a page of their own;
    ``keep`` [R]: first columns whose pages are never listed as released; ``released``: length of that list (by default that
    of the table, which is enough for all). ``out``: an earlier result of the same sizes to write into, with no tensor
    of it among the inputs."""
    if _fast is not None and out is None:
        r = _fast.kv_reorder(block_table, kv_len, parents, free_pages, page, keep, released)
        if r is not NotImplemented:
            new = KvReorder.__new__(KvReorder)
            new.block_table, new.kv_len, new.src, new.dst, new.used, new.released, new.n_released = r
            return new
    _need(block_table, "block_table", _I32, 2)
    _need(kv_len, "kv_len", _I32, 1)
    _need(parents, "parents", _I32, 2)
    _need(free_pages, "free_pages", _I32, 1)
    rows, W = block_table.shape
    R, B = parents.shape
    if R * B != rows or kv_len.shape[0] != rows:
        raise ValueError("block_table, kv_len and parents disagree on the number of rows")
    Q = rows * W if released is None else int(released)
    _sizes(rows, W, free_pages.shape[0], rows * W, Q)
    if Q < 0 or not 0 < page < 1 << 31:
        raise ValueError("released must be >= 0, and page > 0 and below 2^31")
    dev = _device(block_table, kv_len, parents, free_pages)
    if keep is not None:
        _need(keep, "keep", _I32, 1)
        if keep.shape[0] != R:
            raise ValueError("keep must have one entry for each request")
        _device(block_table, keep)
    if out is None:
        out = KvReorder(rows, W, Q, block_table.device)
    else:
        for name, shape in (("block_table", (rows, W)), ("kv_len", (rows,)), ("src", (rows,)), ("dst", (rows,)), ("used", (1,)),
                            ("released", (Q,)), ("n_released", (1,))):
            t = getattr(out, name)
            _need(t, "out." + name, _I32, len(shape))
            if t.shape != shape:
                raise ValueError(f"out.{name} must have the shape {shape}")
        _device(block_table, *(getattr(out, name) for name in KvReorder.__slots__))
    need = _workspace("kv_reorder", R, B, W)
    ws = torch.empty(need, dtype=torch.uint8, device=block_table.device)
    _enqueue(lib().qgemm_kv_reorder, dev, block_table.data_ptr(), kv_len.data_ptr(), parents.data_ptr(), free_pages.data_ptr(),
             None if keep is None else keep.data_ptr(), out.block_table.data_ptr(), out.kv_len.data_ptr(), out.src.data_ptr(),
             out.dst.data_ptr(), out.used.data_ptr(), out.released.data_ptr(), out.n_released.data_ptr(), ws.data_ptr(), need, R, B, W,
             free_pages.shape[0], Q, page)
    if rows == 0:             # the library leaves a reordering of nothing alone
        out.used.zero_()
        out.n_released.zero_()
        out.released.fill_(-1)
    return out


def kv4_copy(cache: torch.Tensor, src: torch.Tensor, dst: torch.Tensor, D: int | None = None):
    """Whole pages within a cache, page ``src[i]`` to page ``dst[i]`` (``qgemm_kv4_copy``); negative numbers are skipped.
    A page's bytes are copied as they are, so the head dimension ``D`` need not be given."""
    if _fast is not None and _fast.kv4_copy(cache, src, dst, D) is None:
        return
    _need(cache, "cache", (torch.uint8,), 3)
    _need(src, "src", _I32, 1)
    _need(dst, "dst", _I32, 1)
    if src.shape != dst.shape:
        raise ValueError("src and dst must have the same length")
    for d in (128, 64) if D is None else (D,):
        if cache.shape[2] * 16 % (17 * d) == 0 and cache.shape[2] * 16 // (17 * d) >= 16:
            break
    pages, Hkv, page = _cache_sizes(cache, d)
    _sizes(src.shape[0], Hkv, pages, page)
    _enqueue(lib().qgemm_kv4_copy, _device(cache, src, dst), cache.data_ptr(), src.data_ptr(), dst.data_ptr(), src.shape[0], Hkv, d, pages,
             page)


def adapters(y: torch.Tensor, x: torch.Tensor, a: torch.Tensor, b: torch.Tensor, ids: torch.Tensor, gain: torch.Tensor | None = None,
             cu_q: torch.Tensor | None = None):
    """Adds the requests' low-rank adapters to a projection's output: ``y[m] += gain[i] * b[i] @ (a[i] @ x[m])`` with ``i`` the
    entry of ``ids`` [R] for the row's request (``qgemm_adapters``); returns ``y``.

    ``y`` [M][N] fp32 and ``x`` [M][K] bf16, rows at any stride (``x``'s a multiple of 8); ``a`` [n][r][K], ``b`` [n][N][r] bf16;
    ``gain`` [n] fp32; ``cu_q`` [R+1]: first rows of the requests, or None where each has one. Rows of an id outside [0, n)
    are left as they are. Nothing here has a backward pass: a ``y`` that requires a gradient is refused where gradients are
    recorded, and a graph that has saved ``y`` refuses to go back through it afterwards, as after torch's own in-place operations."""
    if _fast is not None:
        done = _fast.adapters(y, x, a, b, ids, gain, cu_q)
        if done is not NotImplemented:
            return done
    for t, name, dtypes in ((y, "y", (torch.float32,)), (x, "x", _BF16)):
        if not isinstance(t, torch.Tensor):
            raise TypeError(f"{name} must be a torch.Tensor")
        if not t.is_cuda:
            raise ValueError(f"{name} must be a GPU tensor")
        if t.dtype not in dtypes:
            raise TypeError(f"{name} has dtype {t.dtype}, expected one of {dtypes}")
        if t.dim() != 2 or (t.numel() and t.shape[1] > 1 and t.stride(1) != 1):
            raise ValueError(f"{name} must have 2 dimensions, the last of them contiguous")
    if y.requires_grad and torch.is_grad_enabled():
        raise ValueError("y requires a gradient, which would lack the adapters' part: call it under torch.no_grad()")
    _need(a, "a", _BF16, 3)
    _need(b, "b", _BF16, 3)
    _need(ids, "ids", _I32, 1)
    M, K = x.shape
    n, r, _ = a.shape
    N, R = y.shape[1], ids.shape[0]
    if y.shape[0] != M or a.shape[2] != K or b.shape != (n, N, r):
        raise ValueError("y, x, a and b disagree on M, N, K, the rank or the number of adapters")
    _sizes(M, N, K, r, n, R)
    dev = _device(y, x, a, b, ids)
    if gain is not None:
        _need(gain, "gain", (torch.float32,), 1)
        if gain.shape[0] != n:
            raise ValueError("gain must have one entry for each adapter")
        _device(y, gain)
    if cu_q is not None:
        _need(cu_q, "cu_q", _I32, 1)
        if cu_q.shape[0] != R + 1:
            raise ValueError("cu_q must have one entry more than there are requests")
        _device(y, cu_q)
    elif M != R:
        raise ValueError("without cu_q every request has one row")
    need = _workspace("adapters", M, N, K, r)
    ws = torch.empty(need, dtype=torch.uint8, device=y.device)
    _enqueue(lib().qgemm_adapters, dev, x.data_ptr(), a.data_ptr(), b.data_ptr(), ids.data_ptr(), None if cu_q is None else cu_q.data_ptr(),
             None if gain is None else gain.data_ptr(), y.data_ptr(), ws.data_ptr(), need, M, N, K, r, n, R, x.stride(0) if M > 1 else K,
             y.stride(0) if M > 1 else N)
    if not y.is_inference():
        torch.autograd.graph.increment_version(y)        # a graph that has saved y must not go back through it
    return y


def probe_mfma_clock(iters: int = 100000):
    """Sustained shader clock (MHz) and bf16 MFMA throughput (TFLOP/s) under full matrix-core load
    (``qgemm_probe_mfma_clock``; synchronises the current stream). A measurement utility."""
    mhz = ctypes.c_double(0.0)
    tf = ctypes.c_double(0.0)
    _check(lib().qgemm_probe_mfma_clock(int(iters), ctypes.byref(mhz), ctypes.byref(tf),
                                        torch.cuda.current_stream().cuda_stream))
    return {"sclk_mhz": mhz.value, "mfma_tflops": tf.value}
