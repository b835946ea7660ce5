"""Thin Python binding of the C ABI in include/liquidgemm.h (argument marshalling only).

The calls of a serving loop -- activation quantisation, GEMM, grouped GEMM -- first go to a native module
(csrc/binding.cpp), which checks, allocates and launches where everything is as it usually is and leaves all else to
the ctypes path below: a token through one 4096 x 4096 projection takes 10.5 us in place of 30.  The module is built against
one torch and one Python; without it, or with another, every call takes the ctypes path, and the first one says so.

Host entry points take and return numpy arrays; device entry points take torch tensors
that live on the GPU (torch is used for device memory and streams, nothing else) and
enqueue on torch's current stream unless `stream` (a raw hipStream_t integer) is given.
Every step of the path runs inside libliquidgemm.so; if the library has not been built
the first call raises -- there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
import sys
import threading
import warnings

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
# LIQUIDGEMM_LIB lets tools load another build of the same library (e.g. an experiment build)
LIB_PATH = os.environ.get("LIQUIDGEMM_LIB") or os.path.join(_PKG, "libliquidgemm.so")
_lib = None
_native = None  # the native module, bound to _lib, or what stands in for it

LQ_OK = 0
LQ_ERR_INVALID, LQ_ERR_ALIGN, LQ_ERR_WORKSPACE, LQ_ERR_HIP = -1, -2, -3, -4


class LiquidGemmError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"liquidgemm error {code}: {message}")
        self.code = code


def lib() -> ctypes.CDLL:
    """Load libliquidgemm.so (built by `python -m paper_2509_01229_amd.build`)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2509_01229_amd.build` "
            "(there is no CPU fallback for the GEMM path)")
    # torch ships its own HIP runtime; load it first so that the library binds to the
    # same runtime that owns the device pointers and streams it is handed.
    import torch  # noqa: F401

    L = ctypes.CDLL(LIB_PATH)
    i, vp, sz = ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t
    L.w4a8_version.restype = i
    L.w4a8_last_error.restype = ctypes.c_char_p
    L.liquidquant_packed_size.restype = i
    L.liquidquant_packed_size.argtypes = [i, i, i, ctypes.POINTER(sz), ctypes.POINTER(sz)]
    L.liquidquant_pack_weights.restype = i
    L.liquidquant_pack_weights.argtypes = [vp, i, i, i, vp, vp, vp]
    L.liquidquant_pack_weights_f16.restype = i
    L.liquidquant_pack_weights_f16.argtypes = [vp, i, i, i, vp, vp, vp]
    L.liquidquant_pack_from_i8.restype = i
    L.liquidquant_pack_from_i8.argtypes = [vp, i, i, i, vp, vp]
    L.liquidquant_unpack_weights.restype = i
    L.liquidquant_unpack_weights.argtypes = [vp, vp, i, i, i, vp, vp, vp]
    L.w4a8_gemm_workspace_size.restype = sz
    L.w4a8_gemm_workspace_size.argtypes = [i, i, i, i]
    L.w4a8_workspace_init.restype = i
    L.w4a8_workspace_init.argtypes = [vp, sz, vp]
    L.w4a8_gemm.restype = i
    L.w4a8_gemm.argtypes = [i, i, i, i, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.w4a8_gemm_static.restype = i
    L.w4a8_gemm_static.argtypes = [i, i, i, i, vp, vp, vp, vp, vp, vp, vp]
    L.w4a8_gemm_i32.restype = i
    L.w4a8_gemm_i32.argtypes = [i, i, i, i, vp, vp, vp, vp, vp, sz, vp]
    L.w4a8_gemm_variant.restype = i
    L.w4a8_gemm_variant.argtypes = [i, i, i, i, i, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.w4a8_variant_count.restype = i
    L.w4a8_variant_name.restype = ctypes.c_char_p
    L.w4a8_variant_name.argtypes = [i]
    L.w4a8_variant_supports.restype = i
    L.w4a8_variant_supports.argtypes = [i, i, i, i, i]
    L.w4a8_select_variant.restype = i
    L.w4a8_select_variant.argtypes = [i, i, i, i]
    L.w4a8_select_plan.restype = i
    L.w4a8_select_plan.argtypes = [i, i, i, i, ctypes.POINTER(ctypes.c_int), ctypes.POINTER(ctypes.c_int)]
    L.w4a8_describe_launch.restype = i
    L.w4a8_describe_launch.argtypes = [i, i, i, i, i, ctypes.c_char_p, sz, ctypes.POINTER(sz)]
    L.w4a8_dequant_dump.restype = i
    L.w4a8_dequant_dump.argtypes = [vp, vp, i, i, i, vp, vp]
    L.w4a8_grouped_gemm.restype = i
    L.w4a8_grouped_gemm.argtypes = [i, ctypes.POINTER(ctypes.c_int), i, i, i, vp, vp, vp, vp, vp, vp, vp, vp]
    L.w4a8_describe_grouped.restype = i
    L.w4a8_describe_grouped.argtypes = [i, ctypes.POINTER(ctypes.c_int), i, i, i, ctypes.c_char_p, sz]
    L.w4a8_quantize_activations.restype = i
    L.w4a8_quantize_activations.argtypes = [i, i, vp, vp, vp, vp, vp]
    L.w8a8_pack_weights.restype = i
    L.w8a8_pack_weights.argtypes = [vp, i, i, vp]
    L.w8a8_gemm.restype = i
    L.w8a8_gemm.argtypes = [i, i, i, vp, vp, vp, vp, vp, vp, vp]
    ll, f, d = ctypes.c_longlong, ctypes.c_float, ctypes.c_double
    L.attn_rope_table.restype = i
    L.attn_rope_table.argtypes = [i, i, d, i, d, i, vp]
    L.attn_qk_norm_rope.restype = i
    L.attn_qk_norm_rope.argtypes = [i] * 5 + [vp, ll, ll] * 2 + [vp, vp, i, i, i, vp, vp, f] + [vp, ll, ll] * 2 + [vp]
    L.kv4_page_bytes.restype = sz
    L.kv4_page_bytes.argtypes = [i, i, i]
    L.kv4_write.restype = i
    L.kv4_write.argtypes = [i] * 4 + [vp, ll, ll] * 2 + [vp, vp, i, i, vp]
    L.kv4_append.restype = i
    L.kv4_append.argtypes = [i] * 5 + [vp, ll, ll] * 3 + [vp, vp, i, i, i, vp, vp, f, vp, ll, ll, vp, vp, i, i, vp]
    L.kv4_read.restype = i
    L.kv4_read.argtypes = [i] * 4 + [vp, i, i, vp, vp, vp, vp]
    L.kv4_attention_workspace_size.restype = sz
    L.kv4_attention_workspace_size.argtypes = [i] * 5
    L.kv4_attention.restype = i
    L.kv4_attention.argtypes = [i] * 6 + [vp, ll, ll, ll, vp, i, i, vp, i, vp, f, vp, vp, sz, vp]
    L.attn_prompt.restype = i
    L.attn_prompt.argtypes = [i] * 7 + [vp, ll, ll] * 3 + [vp, vp, f, i, vp, vp, sz, vp]
    L.attn_prompt_workspace_size.restype = sz
    L.attn_prompt_workspace_size.argtypes = [i] * 6
    L.kv4_attention_chunks_workspace_size.restype = sz
    L.kv4_attention_chunks_workspace_size.argtypes = [i] * 7
    L.kv4_attention_chunks.restype = i
    L.kv4_attention_chunks.argtypes = [i] * 6 + [vp, ll, ll, vp, vp, i, i, vp, i, vp, f, vp, vp, sz, vp]
    L.w4a8_norm_quantize.restype = i
    L.w4a8_norm_quantize.argtypes = [i, i, i, vp, ll, vp, ll, vp, f, vp, vp, vp, vp, vp]
    L.w4a8_swiglu_quantize.restype = i
    L.w4a8_swiglu_quantize.argtypes = [i, i, i, vp, ll, vp, vp, vp]
    L.moe_dispatch.restype = i
    L.moe_dispatch.argtypes = [i] * 5 + [vp, ll] + [vp] * 7
    L.moe_combine.restype = i
    L.moe_combine.argtypes = [i] * 5 + [vp, ll] + [vp] * 4
    L.moe_combine_backward.restype = i
    L.moe_combine_backward.argtypes = [i] * 5 + [vp, ll] * 2 + [vp] * 6
    L.w4a8_calib_stream_read.restype = i
    L.w4a8_calib_stream_read.argtypes = [vp, sz, vp]
    L.w4a8_calib_mfma_i8.restype = i
    L.w4a8_calib_mfma_i8.argtypes = [i, i, ctypes.POINTER(ctypes.c_double), vp]
    _bind(L)
    _lib = L
    return L


class _NoNative:
    """Stands in for the native module where there is none for this torch and Python: declines every call, and says why once."""

    def __init__(self, why):
        self._why = why

    def _decline(self, *args):
        if self._why:
            why, self._why = self._why, None
            warnings.warn(f"no native module for this Python and torch ({why}): calls go through ctypes, 20 us more each; "
                          "build it with `python -m paper_2509_01229_amd.build`", RuntimeWarning, stacklevel=3)

    gemm = quantize = grouped = rope = write = append = read = decode = prompt = _decline
    chunks = norm = swiglu = dispatch = combine = combine_backward = _decline


def native_built_for() -> str:
    """The Python and torch that a native module has to be built against to be used here."""
    import torch

    return f"Python {sys.version_info[0]}.{sys.version_info[1]}, torch {torch.__version__}"


def _bind(L) -> None:
    """Hand the native module, if there is one, the entry points of the loaded library."""
    global _native
    try:
        from . import _binding

        built_for = getattr(_binding, "built_for", "another version of this package")
        if built_for != native_built_for():
            raise ImportError(f"_binding.so is built for {built_for}, this is {native_built_for()}")
    except ImportError as e:
        _native = _NoNative(str(e))
        return
    address = lambda f: ctypes.cast(f, ctypes.c_void_p).value
    _binding.bind(address(L.w4a8_gemm), address(L.w4a8_gemm_workspace_size), address(L.w4a8_quantize_activations),
                  address(L.w4a8_grouped_gemm), address(L.liquidquant_packed_size))
    _binding.bind_attention(address(L.attn_qk_norm_rope), address(L.kv4_write), address(L.kv4_append), address(L.kv4_read),
                            address(L.kv4_attention_workspace_size), address(L.kv4_attention), address(L.attn_prompt_workspace_size),
                            address(L.attn_prompt))
    _binding.bind_layer(address(L.kv4_attention_chunks_workspace_size), address(L.kv4_attention_chunks), address(L.w4a8_norm_quantize),
                        address(L.w4a8_swiglu_quantize), address(L.moe_dispatch), address(L.moe_combine), address(L.moe_combine_backward))
    _native = _binding


def _check(rc: int) -> None:
    if rc != LQ_OK:
        raise LiquidGemmError(rc, lib().w4a8_last_error().decode())


def _result(done):
    """What the native module answered: a result, or an error of the library."""
    if done.__class__ is int:
        _check(done)
    return done


def _np(a):
    return a.ctypes.data_as(ctypes.c_void_p)


# ----------------------------------------------------------------------------- host side
def w4a8_version() -> int:
    return int(lib().w4a8_version())


def liquidquant_packed_size(N: int, K: int, group: int):
    cb, gb = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib().liquidquant_packed_size(N, K, group, ctypes.byref(cb), ctypes.byref(gb)))
    return int(cb.value), int(gb.value)


def _alloc_packed(N, K, group):
    cb, gb = liquidquant_packed_size(N, K, group)
    return np.empty(cb, dtype=np.uint8), np.empty(gb, dtype=np.uint8)


def liquidquant_pack_weights(W, group: int):
    """W: numpy [N,K] float32 (FP16-valued) or float16.  Returns (W_packed, gparams, w_scales)."""
    W = np.ascontiguousarray(W)
    if W.ndim != 2:
        raise ValueError("W must be [N, K]")
    N, K = W.shape
    packed, gparams = _alloc_packed(N, K, group)
    w_scales = np.empty(N, dtype=np.float32)
    if W.dtype == np.float16:
        rc = lib().liquidquant_pack_weights_f16(_np(W.view(np.uint16)), N, K, group, _np(packed),
                                                _np(gparams), _np(w_scales))
    elif W.dtype == np.float32:
        rc = lib().liquidquant_pack_weights(_np(W), N, K, group, _np(packed), _np(gparams), _np(w_scales))
    else:
        raise TypeError("W must be float32 or float16")
    _check(rc)
    return packed, gparams, w_scales


def liquidquant_pack_from_i8(Q_i8, group: int):
    Q = np.ascontiguousarray(Q_i8, dtype=np.int8)
    N, K = Q.shape
    packed, gparams = _alloc_packed(N, K, group)
    _check(lib().liquidquant_pack_from_i8(_np(Q), N, K, group, _np(packed), _np(gparams)))
    return packed, gparams


def w8a8_pack_weights(W_i8):
    """INT8 weights [N,K] (numpy) in the order the W8A8 reference kernel consumes them: uint8 [N*K]."""
    W = np.ascontiguousarray(W_i8, dtype=np.int8)
    if W.ndim != 2:
        raise ValueError("W must be [N, K]")
    N, K = W.shape
    packed = np.empty(N * K, dtype=np.uint8)
    _check(lib().w8a8_pack_weights(_np(W), N, K, _np(packed)))
    return packed


def liquidquant_unpack_weights(W_packed, gparams, N: int, K: int, group: int):
    """Returns (codes [N,K] uint8, s_u8 [N,K/group] uint8, a [N,K/group] uint8)."""
    W_packed = np.ascontiguousarray(W_packed, dtype=np.uint8)
    gparams = np.ascontiguousarray(gparams, dtype=np.uint8)
    cb, gb = liquidquant_packed_size(N, K, group)
    if W_packed.size != cb or gparams.size != gb:
        raise ValueError("packed blob has the wrong size for this shape")
    codes = np.empty((N, K), dtype=np.uint8)
    s_u8 = np.empty((N, K // group), dtype=np.uint8)
    a = np.empty((N, K // group), dtype=np.uint8)
    _check(lib().liquidquant_unpack_weights(_np(W_packed), _np(gparams), N, K, group, _np(codes),
                                            _np(s_u8), _np(a)))
    return codes, s_u8, a


# --------------------------------------------------------------------------- device side
def _dev(t, dtype, shape=None, name="tensor"):
    import torch

    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a torch tensor on the GPU")
    if t.dtype != dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    import torch

    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    return ctypes.c_void_p(int(stream))


def w4a8_gemm_workspace_size(M: int, N: int, K: int, group: int) -> int:
    return int(lib().w4a8_gemm_workspace_size(M, N, K, group))


_ws_cache = {}
_ws_retired = []
_ws_lock = threading.Lock()  # (of two threads that find no buffer, one makes it: neither's may be lost)


def w4a8_workspace_init(workspace, stream=None) -> None:
    """Zero the ticket area at the head of a workspace tensor (uint8, on the GPU)."""
    import torch

    _check(lib().w4a8_workspace_init(_dev(workspace, torch.uint8, name="workspace"), workspace.numel(),
                                     _stream(stream)))


def _ws(workspace, M=0, N=0, K=0, group=64, device=None, stream=None, need=None):
    """Workspace pointer and size.  With workspace=None a zero-initialised buffer of at least the size
    the library asks for (`need`: of another call than a GEMM) is allocated once per (device, stream) and reused: calls on different
    streams may overlap and must not share one (device memory plumbing, nothing else)."""
    import torch

    if workspace is None:
        if device is not None and torch.device(device).type != "cuda":
            raise TypeError("X must be a torch tensor on the GPU")
        if need is None:
            need = w4a8_gemm_workspace_size(M, N, K, group) if M > 0 else 0
        if need == 0:
            return None, 0
        # (the native module looks buffers up by the same key)
        key = (torch.device(device).index, int(stream) if stream is not None else int(torch.cuda.current_stream().cuda_stream))
        with _ws_lock:
            buf = _ws_cache.get(key)
            if buf is None or buf.numel() < need:
                # A raw stream is unknown to torch's allocator, so a superseded buffer is kept
                # alive (earlier launches on that stream may still use it) and the new one is
                # zeroed under a device-wide synchronisation before any stream can see it.
                if buf is not None:
                    _ws_retired.append(buf)
                # A power of two: needs that grow call by call (with a batch, a prompt) meet a wait and
                # leave a buffer behind a few times in all, and less than the one in use.
                buf = torch.zeros(1 << (need - 1).bit_length(), dtype=torch.uint8, device=device)
                torch.cuda.synchronize(device)
                _ws_cache[key] = buf
        workspace = buf
    return _dev(workspace, torch.uint8, name="workspace"), workspace.numel()


def w4a8_gemm(X, act_scales, W_packed, gparams, w_scales, N: int, K: int, group: int, out=None,
              workspace=None, stream=None):
    """Y [M,N] float16 = epilogue(X . dequant(W)^T); all tensors on the GPU."""
    if _native is None:
        lib()
    done = _native.gemm(X, act_scales, W_packed, gparams, w_scales, N, K, group, out, workspace, stream, _ws_cache)
    if done is not None:
        return _result(done)
    import torch

    M = X.shape[0]
    if out is None:
        out = torch.empty((M, N), dtype=torch.float16, device=X.device)
    wsp, wsb = _ws(workspace, M, N, K, group, X.device, stream)
    cb, gb = liquidquant_packed_size(N, K, group)
    _check(lib().w4a8_gemm(M, N, K, group, _dev(X, torch.int8, (M, K), "X"),
                           _dev(act_scales, torch.float32, (M,), "act_scales"),
                           _dev(W_packed, torch.uint8, (cb,), "W_packed"),
                           _dev(gparams, torch.uint8, (gb,), "gparams"),
                           _dev(w_scales, torch.float32, (N,), "w_scales"),
                           _dev(out, torch.float16, (M, N), "out"), wsp, wsb, _stream(stream)))
    return out


def w4a8_gemm_static(X, act_scales, W_packed, gparams, w_scales, N: int, K: int, group: int, out, stream=None):
    """w4a8_gemm on the library's built-in split-K workspace: nothing is allocated, so `out`
    ([M,N] float16 on the GPU) must be given."""
    import torch

    M = X.shape[0]
    cb, gb = liquidquant_packed_size(N, K, group)
    _check(lib().w4a8_gemm_static(M, N, K, group, _dev(X, torch.int8, (M, K), "X"),
                                  _dev(act_scales, torch.float32, (M,), "act_scales"),
                                  _dev(W_packed, torch.uint8, (cb,), "W_packed"),
                                  _dev(gparams, torch.uint8, (gb,), "gparams"),
                                  _dev(w_scales, torch.float32, (N,), "w_scales"),
                                  _dev(out, torch.float16, (M, N), "out"), _stream(stream)))
    return out


def w4a8_gemm_i32(X, W_packed, gparams, N: int, K: int, group: int, out=None, workspace=None,
                  stream=None):
    """Raw INT32 accumulators ACC [M,N] of the same kernels."""
    import torch

    M = X.shape[0]
    if out is None:
        out = torch.empty((M, N), dtype=torch.int32, device=X.device)
    wsp, wsb = _ws(workspace, M, N, K, group, X.device, stream)
    cb, gb = liquidquant_packed_size(N, K, group)
    _check(lib().w4a8_gemm_i32(M, N, K, group, _dev(X, torch.int8, (M, K), "X"),
                               _dev(W_packed, torch.uint8, (cb,), "W_packed"),
                               _dev(gparams, torch.uint8, (gb,), "gparams"),
                               _dev(out, torch.int32, (M, N), "out"), wsp, wsb, _stream(stream)))
    return out


def w4a8_gemm_variant(variant: int, X, act_scales, W_packed, gparams, w_scales, N: int, K: int,
                      group: int, want_y=True, want_acc=True, out_y=None, out_acc=None,
                      workspace=None, stream=None):
    """Run one named kernel variant; returns (Y or None, ACC or None)."""
    import torch

    M = X.shape[0]
    if want_y and out_y is None:
        out_y = torch.empty((M, N), dtype=torch.float16, device=X.device)
    if want_acc and out_acc is None:
        out_acc = torch.empty((M, N), dtype=torch.int32, device=X.device)
    wsp, wsb = _ws(workspace, M, N, K, group, X.device, stream)
    cb, gb = liquidquant_packed_size(N, K, group)
    _check(lib().w4a8_gemm_variant(
        variant, M, N, K, group, _dev(X, torch.int8, (M, K), "X"),
        _dev(act_scales, torch.float32, (M,), "act_scales"),
        _dev(W_packed, torch.uint8, (cb,), "W_packed"), _dev(gparams, torch.uint8, (gb,), "gparams"),
        _dev(w_scales, torch.float32, (N,), "w_scales"),
        _dev(out_y, torch.float16, (M, N), "out_y") if want_y else None,
        _dev(out_acc, torch.int32, (M, N), "out_acc") if want_acc else None, wsp, wsb, _stream(stream)))
    return (out_y if want_y else None), (out_acc if want_acc else None)


def w4a8_variant_count() -> int:
    return int(lib().w4a8_variant_count())


def w4a8_variant_name(variant: int):
    s = lib().w4a8_variant_name(variant)
    return s.decode() if s else None


def w4a8_variant_names():
    return [w4a8_variant_name(i) for i in range(w4a8_variant_count())]


def w4a8_variant_supports(variant: int, M: int, N: int, K: int, group: int) -> bool:
    return bool(lib().w4a8_variant_supports(variant, M, N, K, group))


def w4a8_select_variant(M: int, N: int, K: int, group: int) -> int:
    v = int(lib().w4a8_select_variant(M, N, K, group))
    if v < 0:
        _check(v)
    return v


def w4a8_select_plan(M: int, N: int, K: int, group: int):
    """What w4a8_gemm launches for the shape: [(rows, variant index), ...], one or two launches
    over consecutive rows."""
    rows_first, rest = ctypes.c_int(0), ctypes.c_int(-1)
    v = int(lib().w4a8_select_plan(M, N, K, group, ctypes.byref(rows_first), ctypes.byref(rest)))
    if v < 0:
        _check(v)
    plan = [(int(rows_first.value), v)]
    if rest.value >= 0:
        plan.append((M - int(rows_first.value), int(rest.value)))
    return plan


def w4a8_describe_launch(M: int, N: int, K: int, group: int, variant: int = -1):
    """(name of the kernel that runs, workspace bytes it uses) for the dispatcher or a named variant."""
    text, need = ctypes.create_string_buffer(160), ctypes.c_size_t()
    _check(lib().w4a8_describe_launch(variant, M, N, K, group, text, len(text), ctypes.byref(need)))
    return text.value.decode(), int(need.value)


def w4a8_dequant_dump(W_packed, gparams, N: int, K: int, group: int, out=None, stream=None):
    """Wd [N,K] int8 on the GPU, produced by the kernels' own unpack + dequantisation."""
    import torch

    if out is None:
        out = torch.empty((N, K), dtype=torch.int8, device=W_packed.device)
    cb, gb = liquidquant_packed_size(N, K, group)
    _check(lib().w4a8_dequant_dump(_dev(W_packed, torch.uint8, (cb,), "W_packed"),
                                   _dev(gparams, torch.uint8, (gb,), "gparams"), N, K, group,
                                   _dev(out, torch.int8, (N, K), "out"), _stream(stream)))
    return out


def w8a8_gemm(X, act_scales, W8_packed, w_scales, N: int, K: int, want_y=True, want_acc=False, out_y=None,
              out_acc=None, stream=None):
    """The W8A8 reference GEMM (no dequantisation): returns Y [M,N] float16, raw INT32
    accumulators [M,N], or both (in that order), as asked; out_y / out_acc reuse tensors."""
    import torch

    M = int(X.shape[0])
    dx = _dev(X, torch.int8, (M, K), "X")
    dw = _dev(W8_packed, torch.uint8, (N * K,), "W8_packed")
    want_y, want_acc = want_y or out_y is not None, want_acc or out_acc is not None
    Y = (out_y if out_y is not None else torch.empty((M, N), dtype=torch.float16, device=X.device)) if want_y else None
    ACC = (out_acc if out_acc is not None
           else torch.empty((M, N), dtype=torch.int32, device=X.device)) if want_acc else None
    dsx = _dev(act_scales, torch.float32, (M,), "act_scales") if want_y else None
    dsw = _dev(w_scales, torch.float32, (N,), "w_scales") if want_y else None
    _check(lib().w8a8_gemm(M, N, K, dx, dsx, dw, dsw,
                           _dev(Y, torch.float16, (M, N), "Y") if want_y else None,
                           _dev(ACC, torch.int32, (M, N), "ACC") if want_acc else None, _stream(stream)))
    if want_y and want_acc:
        return Y, ACC
    return Y if want_y else ACC


def w4a8_calib_stream_read(buf, stream=None) -> int:
    """Enqueue one pure read of the whole uint8 device tensor `buf`; returns the bytes read."""
    import torch

    n = buf.numel() // 16 * 16
    _check(lib().w4a8_calib_stream_read(_dev(buf, torch.uint8, name="buf"), n, _stream(stream)))
    return n


def w4a8_calib_mfma_i8(iters: int, random_operands: bool, stream=None) -> float:
    """Enqueue the register-only INT8 MFMA loop; returns the operation count of the launch."""
    ops = ctypes.c_double(0.0)
    _check(lib().w4a8_calib_mfma_i8(iters, 1 if random_operands else 0, ctypes.byref(ops), _stream(stream)))
    return ops.value


def w4a8_quantize_activations(X_f16, smooth=None, out_q=None, out_scales=None, stream=None):
    """Per-token INT8 quantisation of FP16 activations [M,K] on the GPU (after dividing by
    the optional FP32 smooth scales [K]); returns (X_i8 [M,K] int8, act_scales [M] float32)."""
    if _native is None:
        lib()
    done = _native.quantize(X_f16, smooth, out_q, out_scales, stream)
    if done is not None:
        return _result(done)
    import torch

    M, K = X_f16.shape
    if out_q is None:
        out_q = torch.empty((M, K), dtype=torch.int8, device=X_f16.device)
    if out_scales is None:
        out_scales = torch.empty((M,), dtype=torch.float32, device=X_f16.device)
    _check(lib().w4a8_quantize_activations(
        M, K, _dev(X_f16, torch.float16, (M, K), "X_f16"),
        _dev(smooth, torch.float32, (K,), "smooth") if smooth is not None else None,
        _dev(out_q, torch.int8, (M, K), "out_q"), _dev(out_scales, torch.float32, (M,), "out_scales"),
        _stream(stream)))
    return out_q, out_scales


def w4a8_grouped_gemm(row_offsets, X, act_scales, W_packed, gparams, w_scales, N: int, K: int, group: int,
                      want_y=True, want_acc=False, out_y=None, out_acc=None, stream=None):
    """E independent W4A8 GEMMs over disjoint runs of tokens (mixture-of-experts layers).
    row_offsets: E+1 host integers; W_packed / gparams: the experts' blobs back to back on the
    GPU; w_scales: [E, N].  Returns (Y or None, ACC or None)."""
    if want_y and not want_acc:
        if _native is None:
            lib()
        done = _native.grouped(row_offsets, X, act_scales, W_packed, gparams, w_scales, N, K, group, out_y, stream)
        if done is not None:
            return _result(done), None
    import torch

    offs = [int(r) for r in row_offsets]
    E = len(offs) - 1
    M = offs[-1]
    if want_y and out_y is None:
        out_y = torch.empty((M, N), dtype=torch.float16, device=X.device)
    if want_acc and out_acc is None:
        out_acc = torch.empty((M, N), dtype=torch.int32, device=X.device)
    cb, gb = liquidquant_packed_size(N, K, group)
    c_offs = (ctypes.c_int * (E + 1))(*offs)
    _check(lib().w4a8_grouped_gemm(
        E, c_offs, N, K, group, _dev(X, torch.int8, (M, K), "X"),
        _dev(act_scales, torch.float32, (M,), "act_scales"),
        _dev(W_packed, torch.uint8, (E * cb,), "W_packed"), _dev(gparams, torch.uint8, (E * gb,), "gparams"),
        _dev(w_scales, torch.float32, (E, N), "w_scales"),
        _dev(out_y, torch.float16, (M, N), "out_y") if want_y else None,
        _dev(out_acc, torch.int32, (M, N), "out_acc") if want_acc else None, _stream(stream)))
    return (out_y if want_y else None), (out_acc if want_acc else None)


def w4a8_describe_grouped(row_offsets, N: int, K: int, group: int) -> str:
    """The launches of w4a8_grouped_gemm for the given rows, "<kernel>[<experts> experts, <rows> rows]+..." ("..., as <form>]": another form)."""
    offs = [int(r) for r in row_offsets]
    text = ctypes.create_string_buffer(320)
    _check(lib().w4a8_describe_grouped(len(offs) - 1, (ctypes.c_int * len(offs))(*offs), N, K, group, text, len(text)))
    return text.value.decode()


# ------------------------------------------- norm and gated activation, tokens sorted by expert and back
# (As the attention calls: tensors that require a gradient are refused where torch would record one.  moe_combine_backward computes those of
# moe_combine, and moe_combine without weights that of moe_dispatch.)
LQ_F16, LQ_BF16, LQ_I8 = 0, 1, 2


def _on_this_device(**tensors):
    """These calls enqueue on the current device's stream: tensors of another device, or of several, are refused."""
    import torch

    here = torch.cuda.current_device() if any(isinstance(t, torch.Tensor) and t.is_cuda for t in tensors.values()) else None
    for name, t in tensors.items():
        if isinstance(t, torch.Tensor) and t.is_cuda and t.device.index != here:
            raise ValueError(f"{name} is on {t.device}, and the current device is cuda:{here}: call it under torch.cuda.device({name}.device)")


def _countable(t, name):
    """The C calls count in 32 bits."""
    if max(t.shape, default=0) >= 2 ** 31:
        raise ValueError(f"{name} is too large: {tuple(t.shape)}")


def _rows(t, name, dtypes=None, shape=None):
    """A matrix on the GPU whose rows may have a stride of their own: its pointer and that stride."""
    import torch

    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a torch tensor on the GPU")
    dtypes = dtypes or (torch.float16, torch.bfloat16)
    if t.dtype not in dtypes:
        raise TypeError(f"{name} must have dtype {' or '.join(str(d)[6:] for d in dtypes)}, got {t.dtype}")
    if t.dim() != 2 or (shape is not None and tuple(t.shape) != tuple(shape)):
        raise ValueError(f"{name} must have shape {tuple(shape) if shape is not None else '[rows, elements]'}, got {tuple(t.shape)}")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}: the elements of a row must be consecutive")
    _countable(t, name)
    return ctypes.c_void_p(t.data_ptr()), t.stride(0)


def w4a8_norm_quantize(x, weight=None, residual=None, eps=1e-6, want_y=False, out_q=None, out_scales=None, out_h=None, out_y=None, stream=None):
    """The residual's addition, the root-mean-square norm and the INT8 quantisation of rows x [M, K], float16 or bfloat16: h = x + residual
    (rounded to the type), y = h / sqrt(mean(h^2) + eps) * weight (float32 [K], or None for ones), INT8 codes with a scale a row.  out_h may be
    residual or x itself.  Returns (X_i8 [M, K], act_scales [M], h or None without a residual, y rounded to the type or None without want_y or
    out_y)."""
    want_y = want_y or out_y is not None
    if _native is None:
        lib()
    done = _native.norm(x, weight, residual, eps, want_y, out_q, out_scales, out_h, out_y, stream)
    if done is not None:
        return _result(done)
    import torch

    _no_gradients(x=x, weight=weight, residual=residual, out_h=out_h, out_y=out_y)
    _on_this_device(x=x, weight=weight, residual=residual, out_q=out_q, out_scales=out_scales, out_h=out_h, out_y=out_y)
    dx = _rows(x, "x")
    M, K = x.shape
    dr = _rows(residual, "residual", (x.dtype,), (M, K)) if residual is not None else (None, 0)
    if residual is None and out_h is not None:
        raise ValueError("out_h goes with a residual: without one h is x")
    new = lambda given, dtype, shape=(M, K): torch.empty(shape, dtype=dtype, device=x.device) if given is None else given  # noqa: E731
    out_q, out_scales = new(out_q, torch.int8), new(out_scales, torch.float32, (M,))
    out_h = new(out_h, x.dtype) if residual is not None else None
    out_y = new(out_y, x.dtype) if want_y else None
    _check(lib().w4a8_norm_quantize(_dtype_code(x), M, K, *dx, *dr, _dev(weight, torch.float32, (K,), "weight"), eps, _dev(out_h, x.dtype, (M, K), "out_h"),
                                    _dev(out_y, x.dtype, (M, K), "out_y"), _dev(out_q, torch.int8, (M, K), "out_q"),
                                    _dev(out_scales, torch.float32, (M,), "out_scales"), _stream(stream)))
    return out_q, out_scales, out_h, out_y


def w4a8_swiglu_quantize(x, out_q=None, out_scales=None, stream=None):
    """silu(gate) * up of rows x [M, 2K] = [gate | up], float16 or bfloat16 (the product of an MLP's, or the experts', first two matrices), as INT8
    codes with a scale a row.  Returns (X_i8 [M, K], act_scales [M])."""
    if _native is None:
        lib()
    done = _native.swiglu(x, out_q, out_scales, stream)
    if done is not None:
        return _result(done)
    import torch

    _no_gradients(x=x)
    _on_this_device(x=x, out_q=out_q, out_scales=out_scales)
    dx = _rows(x, "x")
    M, K = x.shape[0], x.shape[1] // 2
    if x.shape[1] % 2:
        raise ValueError(f"x must be [rows, 2 * K], got {tuple(x.shape)}")
    out_q = torch.empty((M, K), dtype=torch.int8, device=x.device) if out_q is None else out_q
    out_scales = torch.empty((M,), dtype=torch.float32, device=x.device) if out_scales is None else out_scales
    _check(lib().w4a8_swiglu_quantize(_dtype_code(x), M, K, *dx, _dev(out_q, torch.int8, (M, K), "out_q"),
                                      _dev(out_scales, torch.float32, (M,), "out_scales"), _stream(stream)))
    return out_q, out_scales


def moe_dispatch(X, experts, n_experts: int, act_scales=None, out=None, out_scales=None, stream=None):
    """Each token's row of X [tokens, K] (int8, with act_scales [tokens], or float16 or bfloat16) to a row for each of its experts (int32
    [tokens, each]), sorted by expert, within an expert in the tokens' order.  A pair whose expert is not one of 0 .. n_experts - 1 has no row.  Returns (rows
    [tokens * each, K], row_scales or None, row_offsets int32 [n_experts + 1], places int32 [tokens, each]: the pair's row, or -1); rows
    from row_offsets[n_experts] on are left as they were.  w4a8_grouped_gemm takes row_offsets.tolist() and the rows up to there."""
    if _native is None:
        lib()
    done = _native.dispatch(X, experts, n_experts, act_scales, out, out_scales, stream)
    if done is not None:
        return _result(done)
    import torch

    _no_gradients(X=X, act_scales=act_scales, out=out, out_scales=out_scales)
    _on_this_device(X=X, experts=experts, act_scales=act_scales, out=out, out_scales=out_scales)
    dx = _rows(X, "X", (torch.int8, torch.float16, torch.bfloat16))
    (T, K), code = X.shape, {torch.int8: LQ_I8, torch.float16: LQ_F16, torch.bfloat16: LQ_BF16}[X.dtype]
    if not isinstance(experts, torch.Tensor) or experts.dim() != 2:
        raise ValueError("experts must be [tokens, experts of each]")
    _countable(experts, "experts")
    each = experts.shape[1]
    ids = _dev(experts, torch.int32, (T, each), "experts")
    if not 1 <= n_experts <= 256:
        raise ValueError(f"n_experts must be 1 to 256, got {n_experts}")
    if act_scales is None and out_scales is not None:
        raise ValueError("out_scales goes with act_scales")
    out = torch.empty((T * each, K), dtype=X.dtype, device=X.device) if out is None else out
    if act_scales is not None and out_scales is None:
        out_scales = torch.empty((T * each,), dtype=torch.float32, device=X.device)
    offsets, places = (torch.empty(shape, dtype=torch.int32, device=X.device) for shape in ((n_experts + 1,), (T, each)))
    _check(lib().moe_dispatch(code, T, each, n_experts, K, *dx, _dev(act_scales, torch.float32, (T,), "act_scales"), ids,
                              _dev(out, X.dtype, (T * each, K), "out"), _dev(out_scales, torch.float32, (T * each,), "out_scales"),
                              _dev(offsets, torch.int32), _dev(places, torch.int32), _stream(stream)))
    return out, out_scales, offsets, places


def _places(places, weights):
    import torch

    if not isinstance(places, torch.Tensor) or places.dim() != 2:
        raise ValueError("places must be [tokens, rows of each]")
    _countable(places, "places")
    return (*places.shape, _dev(places, torch.int32, name="places"), _dev(weights, torch.float32, tuple(places.shape), "weights"))


def moe_combine(Y, places, weights=None, out=None, stream=None):
    """The sum of each token's rows of Y [rows, N] (float16 or bfloat16): out[t] = sum_j weights[t, j] * Y[places[t, j]]; weights float32
    [tokens, each], or None for ones; places int32 [tokens, each] (moe_dispatch's; outside the rows: adds nothing).  Returns out [tokens, N].  Without
    weights: the gradient of moe_dispatch's X, from that of its rows."""
    if _native is None:
        lib()
    done = _native.combine(Y, places, weights, out, stream)
    if done is not None:
        return _result(done)
    import torch

    _no_gradients(Y=Y, weights=weights, out=out)
    _on_this_device(Y=Y, places=places, weights=weights, out=out)
    dy = _rows(Y, "Y")
    T, each, dp, dw = _places(places, weights)
    R, N = Y.shape
    out = torch.empty((T, N), dtype=Y.dtype, device=Y.device) if out is None else out
    _check(lib().moe_combine(_dtype_code(Y), T, each, R, N, *dy, dp, dw, _dev(out, Y.dtype, (T, N), "out"), _stream(stream)))
    return out


def moe_combine_backward(grad, Y, places, weights, row_offsets=None, out_Y=None, out_weights=None, stream=None):
    """The gradients of moe_combine's Y and weights from that of its result, grad [tokens, N]: (grad_Y [rows, N], of Y's type, grad_weights
    float32 [tokens, each]).  row_offsets: moe_dispatch's; the rows of grad_Y behind the last expert's are zeroed.  Without it rows that no place names are
    zeros in a new tensor, and left as they were in out_Y."""
    if _native is None:
        lib()
    done = _native.combine_backward(grad, Y, places, weights, row_offsets, out_Y, out_weights, stream)
    if done is not None:
        return _result(done)
    import torch

    _no_gradients(grad=grad, Y=Y, weights=weights, out_Y=out_Y, out_weights=out_weights)
    _on_this_device(grad=grad, Y=Y, places=places, weights=weights, row_offsets=row_offsets, out_Y=out_Y, out_weights=out_weights)
    dy = _rows(Y, "Y")
    if weights is None:
        raise ValueError("weights must be given: without them the gradient of a row is its token's")
    T, each, dp, dw = _places(places, weights)
    R, N = Y.shape
    dg = _rows(grad, "grad", (Y.dtype,), (T, N))
    if row_offsets is not None and (row_offsets.dim() != 1 or not row_offsets.shape[0]):
        raise ValueError(f"row_offsets must be [experts + 1], got {tuple(row_offsets.shape)}")
    used = None if row_offsets is None else ctypes.c_void_p(_dev(row_offsets, torch.int32, name="row_offsets").value + 4 * (row_offsets.shape[0] - 1))
    if out_Y is None:
        out_Y = torch.empty((R, N), dtype=Y.dtype, device=Y.device)
        if used is None:  # (on the call's stream, which writes to it next)
            with torch.cuda.stream(None if stream is None else torch.cuda.ExternalStream(int(stream)) if int(stream) else torch.cuda.default_stream()):
                out_Y.zero_()
    out_weights = torch.empty((T, each), dtype=torch.float32, device=Y.device) if out_weights is None else out_weights
    _check(lib().moe_combine_backward(_dtype_code(Y), T, each, R, N, *dg, *dy, dp, dw, used, _dev(out_Y, Y.dtype, (R, N), "out_Y"),
                                      _dev(out_weights, torch.float32, (T, each), "out_weights"), _stream(stream)))
    return out_Y, out_weights


# ------------------------------------------------------------------------------ attention
# (For inference: tensors that require a gradient are refused where torch would record one.)
_ROPE_SCALING = {None: 0, "linear": 1, "ntk": 2, "yarn": 3}


def attn_rope_table(max_positions: int, rot_dim: int, base: float = 10000.0, scaling=None, factor: float = 1.0,
                    original_positions: int = 0):
    """Cosines and sines of positions 0 .. max_positions - 1, float32 numpy [max_positions, rot_dim]; `scaling`: None, "linear",
    "ntk" or "yarn" stretch the positions by `factor` (yarn: from the `original_positions` of the training)."""
    if scaling not in _ROPE_SCALING:
        raise ValueError(f"scaling must be one of {list(_ROPE_SCALING)}, got {scaling!r}")
    table = np.empty((max(max_positions, 0), max(rot_dim, 0)), dtype=np.float32)
    _check(lib().attn_rope_table(max_positions, rot_dim, base, _ROPE_SCALING[scaling], factor, original_positions, _np(table)))
    return table


def _heads(t, name, dtype=None, shape=None):
    """A [.., heads, head_dim] tensor on the GPU with strides of its own: its pointer and strides (the last one is 1)."""
    import torch

    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a torch tensor on the GPU")
    if t.dtype not in (torch.float16, torch.bfloat16) or (dtype is not None and t.dtype != dtype):
        raise TypeError(f"{name} must have dtype {dtype or 'float16 or bfloat16'}, got {t.dtype}")
    if shape is None and t.dim() != 3:
        raise ValueError(f"{name} must be [tokens, heads, head_dim], got {tuple(t.shape)}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.stride(-1) != 1 and t.shape[-1] != 1:
        raise ValueError(f"{name}: the elements of a head must be consecutive")
    return (ctypes.c_void_p(t.data_ptr()), *t.stride()[:-1])


def _no_gradients(**tensors):
    """The attention calls are for inference: a gradient that is asked for is refused, not left out without a word."""
    import torch

    if torch.is_grad_enabled():
        for name, t in tensors.items():
            if isinstance(t, torch.Tensor) and t.requires_grad:
                raise ValueError(f"{name} requires a gradient, and this call computes none: call it under torch.no_grad(), or with {name}.detach()")


def _dtype_code(t):
    import torch

    return LQ_F16 if t.dtype == torch.float16 else LQ_BF16


def _kv4_shape(cache):
    """(pages, kv heads, page size, head dimension) of a cache tensor made by kv4_cache."""
    import torch

    _dev(cache, torch.uint8, name="cache")
    if cache.dim() == 3:
        for dim in (64, 128):
            page = cache.shape[2] // (dim + 8)
            if page * (dim + 8) == cache.shape[2] and 16 <= page <= 256 and page & (page - 1) == 0:
                return cache.shape[0], cache.shape[1], page, dim
    raise ValueError(f"cache must be [pages, kv_heads, page_size * (head_dim + 8)] as kv4_cache makes it, got {tuple(cache.shape)}")


def kv4_cache(num_pages: int, page_size: int, n_kv_heads: int, head_dim: int, device="cuda"):
    """An empty 4-bit cache of keys and values: uint8 [num_pages, n_kv_heads, page_size * (head_dim + 8)], zeroed."""
    import torch

    nbytes = int(lib().kv4_page_bytes(page_size, n_kv_heads, head_dim))
    if nbytes == 0 or not 1 <= num_pages <= (2**31 - 1) // page_size:
        raise ValueError(f"no cache of {num_pages} pages of {page_size} tokens, {n_kv_heads} heads of {head_dim}: page_size is a power of two "
                         "from 16 to 256, head_dim 64 or 128, num_pages * page_size below 2^31")
    return torch.zeros((num_pages, n_kv_heads, nbytes // n_kv_heads), dtype=torch.uint8, device=device)


def _norms(q_norm, k_norm, dim):
    import torch

    return _dev(q_norm, torch.float32, (dim,), "q_norm"), _dev(k_norm, torch.float32, (dim,), "k_norm")


def _rotation(positions, table, tokens):
    import torch

    if table.dim() != 2:
        raise ValueError(f"table must be [positions, rot_dim], got {tuple(table.shape)}")
    return _dev(positions, torch.int32, (tokens,), "positions"), _dev(table, torch.float32, name="table"), table.shape[0], table.shape[1]


def attn_qk_norm_rope(q, k, positions, table, interleaved=False, q_norm=None, k_norm=None, eps=1e-6, out_q=None, out_k=None, stream=None):
    """Norm of each head (where there are weights, float32 [head_dim]) and rotation of queries [tokens, heads, head_dim] and keys
    [tokens, kv_heads, head_dim], float16 or bfloat16, at `positions` (int32 [tokens]) of `table` (attn_rope_table's, on the GPU).
    out_q, out_k may be q and k themselves.  Returns (out_q, out_k)."""
    if _native is None:
        lib()
    done = _native.rope(q, k, positions, table, interleaved, q_norm, k_norm, eps, out_q, out_k, stream)
    if done is not None:
        return _result(done)
    import torch

    _no_gradients(q=q, k=k, table=table, q_norm=q_norm, k_norm=k_norm, out_q=out_q, out_k=out_k)
    dq, dk = _heads(q, "q"), _heads(k, "k", q.dtype)
    (T, Hq, D), Hkv = q.shape, k.shape[1]
    if tuple(k.shape) != (T, Hkv, D):
        raise ValueError(f"k must have shape {(T, Hkv, D)}, got {tuple(k.shape)}")
    out_q = torch.empty((T, Hq, D), dtype=q.dtype, device=q.device) if out_q is None else out_q
    out_k = torch.empty((T, Hkv, D), dtype=q.dtype, device=q.device) if out_k is None else out_k
    _check(lib().attn_qk_norm_rope(_dtype_code(q), T, Hq, Hkv, D, *dq, *dk, *_rotation(positions, table, T), int(bool(interleaved)),
                                   *_norms(q_norm, k_norm, D), eps, *_heads(out_q, "out_q", q.dtype, (T, Hq, D)),
                                   *_heads(out_k, "out_k", q.dtype, (T, Hkv, D)), _stream(stream)))
    return out_q, out_k


def kv4_write(k, v, slots, cache, stream=None):
    """Quantises keys and values [tokens, kv_heads, head_dim] into the cache's slots (int32 [tokens]: page * page_size + place;
    outside the cache: left out).  Returns the cache."""
    if _native is None:
        lib()
    done = _native.write(k, v, slots, cache, stream)
    if done is not None:
        return _result(done)
    import torch

    _no_gradients(k=k, v=v)
    dk, (T, Hkv, D) = _heads(k, "k"), k.shape
    dv = _heads(v, "v", k.dtype, (T, Hkv, D))
    pages, heads, page, dim = _kv4_shape(cache)
    if (heads, dim) != (Hkv, D):
        raise ValueError(f"the cache holds {heads} heads of {dim}, k has {Hkv} of {D}")
    _check(lib().kv4_write(_dtype_code(k), T, Hkv, D, *dk, *dv, _dev(slots, torch.int32, (T,), "slots"),
                           _dev(cache, torch.uint8, name="cache"), pages, page, _stream(stream)))
    return cache


def kv4_append(q, k, v, positions, table, slots, cache, interleaved=False, q_norm=None, k_norm=None, eps=1e-6, out_q=None, stream=None):
    """attn_qk_norm_rope and kv4_write in one launch: returns the turned queries; keys and values are in the cache."""
    if _native is None:
        lib()
    done = _native.append(q, k, v, positions, table, slots, cache, interleaved, q_norm, k_norm, eps, out_q, stream)
    if done is not None:
        return _result(done)
    import torch

    _no_gradients(q=q, k=k, v=v, table=table, q_norm=q_norm, k_norm=k_norm, out_q=out_q)
    dq, dk = _heads(q, "q"), _heads(k, "k", q.dtype)
    (T, Hq, D), Hkv = q.shape, k.shape[1]
    if tuple(k.shape) != (T, Hkv, D):
        raise ValueError(f"k must have shape {(T, Hkv, D)}, got {tuple(k.shape)}")
    dv = _heads(v, "v", q.dtype, (T, Hkv, D))
    pages, heads, page, dim = _kv4_shape(cache)
    if (heads, dim) != (Hkv, D):
        raise ValueError(f"the cache holds {heads} heads of {dim}, k has {Hkv} of {D}")
    out_q = torch.empty((T, Hq, D), dtype=q.dtype, device=q.device) if out_q is None else out_q
    _check(lib().kv4_append(_dtype_code(q), T, Hq, Hkv, D, *dq, *dk, *dv, *_rotation(positions, table, T), int(bool(interleaved)),
                            *_norms(q_norm, k_norm, D), eps, *_heads(out_q, "out_q", q.dtype, (T, Hq, D)),
                            _dev(slots, torch.int32, (T,), "slots"), _dev(cache, torch.uint8, name="cache"), pages, page, _stream(stream)))
    return out_q


def kv4_read(cache, slots, dtype=None, stream=None):
    """Keys and values [tokens, kv_heads, head_dim] that the slots hold (zeros outside the cache), float16 or `dtype`."""
    import torch

    dtype = dtype or torch.float16
    if dtype not in (torch.float16, torch.bfloat16):
        raise TypeError(f"dtype must be float16 or bfloat16, got {dtype}")
    if _native is None:
        lib()
    done = _native.read(cache, slots, dtype is torch.bfloat16, stream)
    if done is not None:
        return _result(done)
    pages, Hkv, page, D = _kv4_shape(cache)
    T = slots.shape[0]
    k, v = (torch.empty((T, Hkv, D), dtype=dtype, device=cache.device) for _ in range(2))
    _check(lib().kv4_read(_dtype_code(k), T, Hkv, D, _dev(cache, torch.uint8, name="cache"), pages, page,
                          _dev(slots, torch.int32, (T,), "slots"), _heads(k, "k")[0], _heads(v, "v")[0], _stream(stream)))
    return k, v


def kv4_attention(q, cache, block_table, context, scale=None, out=None, workspace=None, stream=None):
    """Attention of the newest tokens q [sequences, new, heads, head_dim] (or [sequences, heads, head_dim]: one each) over the
    cache: `block_table` int32 [sequences, width] names each sequence's pages, `context` int32 [sequences] its tokens, the new ones among
    them; new token i sees the first context - new + 1 + i.  scale: 1 / sqrt(head_dim) unless given.  Returns out, shaped as q."""
    if _native is None:
        lib()
    done = _native.decode(q, cache, block_table, context, scale, out, workspace, stream, _ws_cache)
    if done is not None:
        return _result(done)
    import torch

    _no_gradients(q=q, out=out)
    pages, Hkv, page, D = _kv4_shape(cache)
    one = q.dim() == 3
    if q.dim() not in (3, 4) or q.shape[-1] != D:
        raise ValueError(f"q must be [sequences, new tokens, heads, {D}] or [sequences, heads, {D}], got {tuple(q.shape)}")
    B, n, Hq = (q.shape[0], 1, q.shape[1]) if one else q.shape[:3]
    dq = _heads(q, "q", shape=q.shape)
    if one:
        dq = (dq[0], dq[1], 0, dq[2])
    if block_table.dim() != 2:
        raise ValueError(f"block_table must be [sequences, width], got {tuple(block_table.shape)}")
    out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if out is None else out
    need = int(lib().kv4_attention_workspace_size(B, n, Hq, Hkv, D))
    wsp, wsb = _ws(workspace, device=q.device, stream=stream, need=need)
    _check(lib().kv4_attention(_dtype_code(q), B, n, Hq, Hkv, D, *dq, _dev(cache, torch.uint8, name="cache"), pages, page,
                               _dev(block_table, torch.int32, (B, block_table.shape[1]), "block_table"), block_table.shape[1],
                               _dev(context, torch.int32, (B,), "context"), D ** -0.5 if scale is None else scale,
                               _dev(out, q.dtype, q.shape, "out"), wsp, wsb, _stream(stream)))
    return out


def kv4_attention_chunks(q, cache, block_table, context, starts_q, scale=None, out=None, workspace=None, stream=None):
    """Attention of new tokens over the cache that holds them already, packed sequences with any number of them each: q [tokens, heads,
    head_dim], sequence s has those from starts_q[s] to starts_q[s + 1] - 1 (int32 [sequences + 1] on the GPU); cache, block_table and context as in
    kv4_attention.  New token i of a sequence's n sees the first context - n + 1 + i.  scale: 1 / sqrt(head_dim) unless given.  Returns out, shaped as q;
    rows that belong to no sequence are left as they were.  From 65 sequences on long contexts are not cut into parts that run side by side
    (kv4_attention cuts them for any number of sequences): one of 32768 among many short ones then takes 250 us by itself."""
    if _native is None:
        lib()
    done = _native.chunks(q, cache, block_table, context, starts_q, scale, out, workspace, stream, _ws_cache)
    if done is not None:
        return _result(done)
    import torch

    _no_gradients(q=q, out=out)
    _on_this_device(q=q, cache=cache, block_table=block_table, context=context, starts_q=starts_q, out=out, workspace=workspace)
    pages, Hkv, page, D = _kv4_shape(cache)
    dq, (T, Hq, _) = _heads(q, "q"), q.shape
    if q.shape[2] != D:
        raise ValueError(f"q must be [tokens, heads, {D}], got {tuple(q.shape)}")
    if starts_q.dim() != 1 or starts_q.shape[0] < 1:
        raise ValueError(f"starts_q must be [sequences + 1], got {tuple(starts_q.shape)}")
    S = starts_q.shape[0] - 1
    if block_table.dim() != 2:
        raise ValueError(f"block_table must be [sequences, width], got {tuple(block_table.shape)}")
    for name, t in (("q", q), ("cache", cache), ("starts_q", starts_q), ("block_table", block_table)):
        _countable(t, name)
    width = block_table.shape[1]
    out = torch.empty((T, Hq, D), dtype=q.dtype, device=q.device) if out is None else out
    need = int(lib().kv4_attention_chunks_workspace_size(S, T, Hq, Hkv, D, page, width))
    wsp, wsb = _ws(workspace, device=q.device, stream=stream, need=need)
    _check(lib().kv4_attention_chunks(_dtype_code(q), S, T, Hq, Hkv, D, *dq, _dev(starts_q, torch.int32, (S + 1,), "starts_q"),
                                      _dev(cache, torch.uint8, name="cache"), pages, page, _dev(block_table, torch.int32, (S, width), "block_table"), width,
                                      _dev(context, torch.int32, (S,), "context"), D ** -0.5 if scale is None else scale,
                                      _dev(out, q.dtype, (T, Hq, D), "out"), wsp, wsb, _stream(stream)))
    return out


def attn_prompt(q, k, v, starts_q, starts_k=None, scale=None, causal=True, out=None, workspace=None, stream=None):
    """Attention over packed sequences: q [queries, heads, head_dim], k and v [keys, kv_heads, head_dim]; sequence s has the
    queries starts_q[s] .. starts_q[s + 1] - 1 and the keys starts_k[s] .. (int32 on the GPU; starts_k: starts_q unless given).  causal: query
    i sees the keys up to i + (keys - queries) of its sequence.  scale: 1 / sqrt(head_dim) unless given.  Returns out, shaped as q."""
    if _native is None:
        lib()
    done = _native.prompt(q, k, v, starts_q, starts_q if starts_k is None else starts_k, scale, causal, out, workspace, stream, _ws_cache)
    if done is not None:
        return _result(done)
    import torch

    _no_gradients(q=q, k=k, v=v, out=out)
    dq, dk = _heads(q, "q"), _heads(k, "k", q.dtype)
    (Tq, Hq, D), (Tk, Hkv, _) = q.shape, k.shape
    if k.shape[2] != D:
        raise ValueError(f"k must have heads of {D}, got {tuple(k.shape)}")
    dv = _heads(v, "v", q.dtype, (Tk, Hkv, D))
    starts_k = starts_q if starts_k is None else starts_k
    if starts_q.dim() != 1 or starts_q.shape[0] < 1:
        raise ValueError(f"starts_q must be [sequences + 1], got {tuple(starts_q.shape)}")
    S = starts_q.shape[0] - 1
    out = torch.empty((Tq, Hq, D), dtype=q.dtype, device=q.device) if out is None else out
    need = int(lib().attn_prompt_workspace_size(S, Tq, Tk, Hq, Hkv, D))
    wsp, wsb = _ws(workspace, device=q.device, stream=stream, need=need)
    _check(lib().attn_prompt(_dtype_code(q), S, Tq, Tk, Hq, Hkv, D, *dq, *dk, *dv, _dev(starts_q, torch.int32, (S + 1,), "starts_q"),
                             _dev(starts_k, torch.int32, (S + 1,), "starts_k"), D ** -0.5 if scale is None else scale, int(bool(causal)),
                             _dev(out, q.dtype, (Tq, Hq, D), "out"), wsp, wsb, _stream(stream)))
    return out
