"""Thin Python binding of libfxp (include/fxp.h): argument marshalling only.

Every function takes torch CUDA tensors, allocates the outputs with torch, hands raw
device pointers and the current torch stream to the C ABI and raises FxpError on a
non-zero status.  All arithmetic runs in the HIP kernels; there is no CPU or PyTorch
fallback: if libfxp.so cannot be loaded, or a tensor is not on the GPU, the call fails.
"""
import ctypes
import math
import os
from fractions import Fraction

import torch

from . import build as _build

STOCHASTIC, NEAREST = 0, 1
OP_SCALE, OP_GEMM, OP_LINEAR_FWD, OP_LINEAR_BWD, OP_BMM_FWD, OP_BMM_BWD = 0, 1, 2, 3, 4, 5
TAG_X, TAG_W, TAG_DY = 0, 1, 2
ABSMAX_WORDS = 256      # uint32 words of an abs-max area (FXP_ABSMAX_WORDS)


class FxpError(RuntimeError):
    pass


class _Saved(ctypes.Structure):
    _fields_ = [("Xq", ctypes.c_void_p), ("XqT", ctypes.c_void_p), ("Wq", ctypes.c_void_p), ("WqT", ctypes.c_void_p),
                ("eX", ctypes.c_void_p), ("eW", ctypes.c_void_p)]


class _MapDesc(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("e_max", ctypes.c_void_p),
                ("q", ctypes.c_void_p), ("qT", ctypes.c_void_p), ("stream_id", ctypes.c_uint64)]


class _SgdTensor(ctypes.Structure):
    _fields_ = [("w", ctypes.c_void_p), ("g", ctypes.c_void_p), ("v", ctypes.c_void_p), ("tmp", ctypes.c_void_p),
                ("n", ctypes.c_size_t)]


class _ConvShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("N", "H", "W", "C", "Cout", "KH", "KW", "stride", "pad")]


class _ConvSaved(ctypes.Structure):
    _fields_ = [("Xq", ctypes.c_void_p), ("Wq", ctypes.c_void_p), ("WqT", ctypes.c_void_p), ("WqF", ctypes.c_void_p),
                ("eX", ctypes.c_void_p), ("eW", ctypes.c_void_p)]


class _KvCache(ctypes.Structure):
    _fields_ = [("kq", ctypes.c_void_p), ("vq", ctypes.c_void_p), ("ek", ctypes.c_void_p), ("ev", ctypes.c_void_p),
                ("pages", ctypes.c_int64), ("heads", ctypes.c_int64), ("dim", ctypes.c_int64), ("bits", ctypes.c_int)]


class _KvStep(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int64) for n in ("requests", "blocks", "tokens", "pages")] +
                [(n, ctypes.c_void_p) for n in ("lens", "free_pages", "n_free", "block_table", "lens_after", "n_free_after", "first",
                                                "slots", "positions", "runs", "refused")])


class _Rotation(ctypes.Structure):
    _fields_ = [("turns", ctypes.c_void_p), ("rot", ctypes.c_int64), ("interleaved", ctypes.c_int), ("amplitude", ctypes.c_double)]


class _Mx4(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64)]


class _Mx4Layer(ctypes.Structure):
    _fields_ = [(n, _Mx4) for n in ("X", "XT", "W", "WT", "dY", "dYT")]


_lib = None


def lib():
    """Load libfxp.so (building it first only when no built library exists)."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.LIB
    if not os.path.exists(path):
        path = _build.build()
    L = ctypes.CDLL(path)
    c = ctypes
    vp, i32, i64, u64, sz, ci = c.c_void_p, c.c_int32, c.c_int64, c.c_uint64, c.c_size_t, c.c_int
    L.fxp_strerror.restype = c.c_char_p
    L.fxp_strerror.argtypes = [ci]
    L.fxp_version.restype = ci
    L.fxp_workspace_bytes.restype = sz
    L.fxp_workspace_bytes.argtypes = [ci, i64, i64, i64]
    L.fxp_scale.argtypes = [vp, sz, vp, vp, sz, vp]
    L.fxp_map.argtypes = [vp, i64, i64, vp, vp, vp, u64, u64, ci, ci, vp]
    L.fxp_scale_map.argtypes = [vp, i64, i64, vp, vp, vp, u64, u64, ci, ci, vp, sz, vp]
    L.fxp_gemm.argtypes = [ci, ci, i64, i64, i64, vp, i64, vp, i64, vp, i64, vp, sz, vp]
    L.fxp_unmap.argtypes = [vp, sz, vp, ci, vp, ci, vp, vp]
    L.fxp_unmap_i8.argtypes = [vp, sz, vp, ci, vp, vp]
    L.fxp_gemm_unmap.argtypes = [ci, ci, i64, i64, i64, vp, i64, vp, i64, vp, ci, vp, ci, vp, i64, vp, sz, vp]
    L.fxp_gemm_unmap_absmax.argtypes = [ci, ci, i64, i64, i64, vp, i64, vp, i64, vp, ci, vp, ci, vp, i64, vp, vp, sz, vp]
    L.fxp_map_absmax.argtypes = [vp, i64, i64, vp, vp, vp, vp, u64, u64, ci, ci, vp]
    L.fxp_linear_fwd.argtypes = [vp, vp, i64, i64, i64, vp, c.POINTER(_Saved), u64, u64, ci, ci, vp, sz, vp]
    L.fxp_linear_bwd.argtypes = [vp, c.POINTER(_Saved), i64, i64, i64, vp, vp, vp, vp, vp, u64, u64, ci, ci, vp, sz, vp]
    L.fxp_linear_fwd_guess.argtypes = L.fxp_linear_fwd.argtypes
    L.fxp_linear_bwd_guess.argtypes = L.fxp_linear_bwd.argtypes
    L.fxp_linear_fwd_guess.restype = ci
    L.fxp_linear_bwd_guess.restype = ci
    L.fxp_linear_fwd_static.argtypes = [vp, vp, i64, i64, i64, vp, c.POINTER(_Saved), u64, u64, ci, ci, vp]
    L.fxp_linear_fwd_static.restype = ci
    L.fxp_static_scratch_bytes.restype = sz
    L.fxp_static_scratch_bytes.argtypes = []
    L.fxp_clock_probe.argtypes = [vp, c.c_uint32, vp]
    L.fxp_clock_probe.restype = ci
    L.fxp_timeline_begin.argtypes = [ci]
    L.fxp_timeline_begin.restype = ci
    L.fxp_timeline_end.argtypes = [vp, vp, ci, vp]
    L.fxp_timeline_end.restype = ci
    L.fxp_conv2d_workspace_bytes.restype = sz
    L.fxp_conv2d_workspace_bytes.argtypes = [c.POINTER(_ConvShape), ci]
    L.fxp_conv2d_fwd.argtypes = [vp, vp, c.POINTER(_ConvShape), vp, c.POINTER(_ConvSaved), u64, u64, ci, ci, vp, sz, vp]
    L.fxp_conv2d_bwd.argtypes = [vp, c.POINTER(_ConvSaved), c.POINTER(_ConvShape), vp, vp, vp, vp, vp, u64, u64, ci, ci,
                                 vp, sz, vp]
    L.fxp_conv2d_fwd.restype = ci
    L.fxp_conv2d_bwd.restype = ci
    L.fxp_gemm_batched.argtypes = [i64, i64, i64, vp, i64, i64, vp, i64, i64, vp, i64, i64, i64, vp]
    L.fxp_gemm_unmap_batched.argtypes = [i64, i64, i64, vp, i64, i64, vp, i64, i64, vp, ci, vp, ci, vp, i64, i64, i64, vp]
    L.fxp_bmm_fwd.argtypes = [vp, vp, i64, i64, i64, i64, ci, vp, c.POINTER(_Saved), u64, u64, ci, ci, vp, sz, vp]
    L.fxp_bmm_bwd.argtypes = [vp, c.POINTER(_Saved), i64, i64, i64, i64, ci, vp, vp, vp, vp, vp, u64, u64, ci, ci, vp, sz,
                              vp]
    L.fxp_bmm_fwd_guess.argtypes = L.fxp_bmm_fwd.argtypes
    L.fxp_bmm_bwd_guess.argtypes = L.fxp_bmm_bwd.argtypes
    L.fxp_bmm_fwd_guess.restype = ci
    L.fxp_bmm_bwd_guess.restype = ci
    L.fxp_map2.argtypes = [c.POINTER(_MapDesc), c.POINTER(_MapDesc), u64, ci, ci, vp]
    L.fxp_scale_map2.argtypes = [c.POINTER(_MapDesc), c.POINTER(_MapDesc), u64, ci, ci, vp, sz, vp]
    L.fxp_map2.restype = ci
    L.fxp_scale_map2.restype = ci
    L.fxp_sgd16_multi_workspace_bytes.restype = sz
    L.fxp_sgd16_multi_workspace_bytes.argtypes = [c.POINTER(_SgdTensor), sz]
    L.fxp_sgd16_step_multi.argtypes = [c.POINTER(_SgdTensor), sz, c.c_float, c.c_float, c.c_float, u64, u64, ci, vp, sz, vp]
    L.fxp_sgd16_step_multi.restype = ci
    L.fxp_sgd16_workspace_bytes.restype = sz
    L.fxp_sgd16_workspace_bytes.argtypes = []
    L.fxp_axpy16.argtypes = [vp, vp, c.c_float, sz, vp, vp, u64, u64, ci, vp, sz, vp]
    L.fxp_sgd16_step.argtypes = [vp, vp, vp, sz, c.c_float, c.c_float, c.c_float, vp, u64, u64, ci, vp, sz, vp]
    L.fxp_axpy16.restype = ci
    L.fxp_sgd16_step.restype = ci
    cache, step = c.POINTER(_KvCache), c.POINTER(_KvStep)
    L.fxp_kv_max_runs.argtypes = [i64, i64]
    L.fxp_kv_max_runs.restype = i64
    L.fxp_kv_tables.argtypes = [step, vp, vp, sz, vp]
    L.fxp_kv_append.argtypes = [cache, ci, vp, i64, i64, vp, i64, i64, i64, vp, i64, vp]
    L.fxp_kv_load.argtypes = [cache, ci, vp, vp, i64, vp, i64, vp]
    L.fxp_kv_attention_workspace_bytes.argtypes = [i64, i64, i64, i64, i64]
    L.fxp_kv_attention_workspace_bytes.restype = sz
    L.fxp_kv_attention.argtypes = [cache, step, ci, vp, i64, i64, i64, c.c_float, i64, vp, i64, i64, vp, vp, sz, vp]
    L.fxp_w4_packed_bytes.argtypes = [i64, i64]
    L.fxp_w4_packed_bytes.restype = sz
    L.fxp_w4_scale_bytes.argtypes = [i64, i64, ci]
    L.fxp_w4_scale_bytes.restype = sz
    L.fxp_w4_workspace_bytes.argtypes = [ci, i64, i64, ci]
    L.fxp_w4_workspace_bytes.restype = sz
    L.fxp_w4_pack.argtypes = [ci, vp, i64, i64, i64, ci, vp, vp, vp]
    L.fxp_w4_linear.argtypes = [ci, vp, i64, i64, i64, i64, vp, vp, ci, vp, i64, vp, sz, vp]
    turn = c.POINTER(_Rotation)
    L.fxp_rotary.argtypes = [turn, ci, ci, i64, i64, i64, i64, vp, i64, i64, i64, vp, i64, vp, i64, i64, i64, vp]
    L.fxp_rotary.restype = ci
    L.fxp_kv_append_rotary.argtypes = [cache, step, turn, ci, vp, i64, i64, vp, i64, i64, vp, i64, i64, i64, vp, i64, i64, vp]
    L.fxp_kv_append_rotary.restype = ci
    mx = c.POINTER(_Mx4)
    L.fxp_mx4_data_bytes.argtypes = [i64, i64]
    L.fxp_mx4_data_bytes.restype = sz
    L.fxp_mx4_scale_bytes.argtypes = [i64, i64]
    L.fxp_mx4_scale_bytes.restype = sz
    L.fxp_mx4_map.argtypes = [ci, vp, i64, i64, i64, mx, mx, u64, u64, ci, vp]
    L.fxp_mx4_map.restype = ci
    L.fxp_mx4_unmap.argtypes = [mx, ci, vp, i64, vp]
    L.fxp_mx4_unmap.restype = ci
    L.fxp_mx4_gemm.argtypes = [mx, mx, ci, vp, i64, vp, sz, vp]
    L.fxp_mx4_linear.argtypes = [ci, vp, i64, i64, mx, vp, i64, vp, sz, vp]
    L.fxp_mx4_linear_fwd.argtypes = [ci, vp, vp, i64, i64, i64, vp, c.POINTER(_Mx4Layer), u64, u64, ci, vp, sz, vp]
    L.fxp_mx4_linear_bwd.argtypes = [ci, vp, c.POINTER(_Mx4Layer), i64, i64, i64, vp, vp, u64, u64, ci, vp, sz, vp]
    for name in ("fxp_mx4_gemm", "fxp_mx4_linear", "fxp_mx4_linear_fwd", "fxp_mx4_linear_bwd"):
        getattr(L, name).restype = ci
    for name in ("fxp_mx4_gemm_workspace_bytes", "fxp_mx4_linear_workspace_bytes", "fxp_mx4_layer_workspace_bytes"):
        getattr(L, name).argtypes = [i64, i64, i64]
        getattr(L, name).restype = sz
    for name in ("fxp_kv_tables", "fxp_kv_append", "fxp_kv_load", "fxp_kv_attention", "fxp_w4_pack", "fxp_w4_linear"):
        getattr(L, name).restype = ci
    for name in ("fxp_scale", "fxp_map", "fxp_scale_map", "fxp_gemm", "fxp_unmap", "fxp_unmap_i8", "fxp_gemm_unmap",
                 "fxp_gemm_unmap_absmax", "fxp_map_absmax",
                 "fxp_linear_fwd", "fxp_linear_bwd", "fxp_gemm_batched", "fxp_gemm_unmap_batched", "fxp_bmm_fwd",
                 "fxp_bmm_bwd"):
        getattr(L, name).restype = ci
    _lib = L
    return L


def _check(rc, what):
    if rc != 0:
        raise FxpError(f"{what}: {lib().fxp_strerror(rc).decode()} ({rc})")


def _dev(t, dtype, what):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise FxpError(f"{what} must be a CUDA tensor: libfxp has no CPU path")
    if t.dtype != dtype or not t.is_contiguous():
        raise FxpError(f"{what} must be a contiguous {dtype} tensor")
    return t


def _p(t):
    return None if t is None else t.data_ptr()


def _stream():
    # the handle of torch.cuda.current_stream() without the Stream object around it, which costs several microseconds a call -
    # as much as the launches of a small layer (256^3 step, of the host: 25.6 us, without it 19.3)
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def workspace_bytes(op, M, N=0, K=0):
    return int(lib().fxp_workspace_bytes(op, M, N, K))


def _ws(op, M, N=0, K=0, device=None):
    return torch.empty(max(256, workspace_bytes(op, M, N, K)), dtype=torch.uint8, device=device)


def scale(x, ws=None):
    """e_max of a tensor as a 1-element int32 device tensor (no synchronisation)."""
    x = _dev(x, torch.float32, "x")
    e = torch.empty(1, dtype=torch.int32, device=x.device)
    ws = ws if ws is not None else _ws(OP_SCALE, x.numel(), device=x.device)
    _check(lib().fxp_scale(_p(x), x.numel(), _p(e), _p(ws), ws.numel(), _stream()), "fxp_scale")
    return e


def _map_outputs(x, want_q, want_qT):
    rows, cols = x.shape
    q = torch.empty((rows, cols), dtype=torch.int8, device=x.device) if want_q else None
    qT = torch.empty((cols, rows), dtype=torch.int8, device=x.device) if want_qT else None
    return q, qT


def map(x, e_max, seed=0, stream_id=0, rounding=STOCHASTIC, bits=8, want_q=True, want_qT=False):
    """(q, qT) int8 tensors of x[rows, cols] under the device scale e_max."""
    x = _dev(x, torch.float32, "x")
    e_max = _dev(e_max, torch.int32, "e_max")
    assert x.dim() == 2
    q, qT = _map_outputs(x, want_q, want_qT)
    _check(lib().fxp_map(_p(x), x.shape[0], x.shape[1], _p(e_max), _p(q), _p(qT), seed, stream_id, rounding, bits,
                         _stream()), "fxp_map")
    return q, qT


def scale_map(x, seed=0, stream_id=0, rounding=STOCHASTIC, bits=8, want_q=True, want_qT=False, ws=None):
    """(e_max, q, qT): scale and map in one call."""
    x = _dev(x, torch.float32, "x")
    assert x.dim() == 2
    e = torch.empty(1, dtype=torch.int32, device=x.device)
    q, qT = _map_outputs(x, want_q, want_qT)
    ws = ws if ws is not None else _ws(OP_SCALE, x.numel(), device=x.device)
    _check(lib().fxp_scale_map(_p(x), x.shape[0], x.shape[1], _p(e), _p(q), _p(qT), seed, stream_id, rounding, bits,
                               _p(ws), ws.numel(), _stream()), "fxp_scale_map")
    return e, q, qT


def _gemm_dims(A, B, transA, transB):
    M, K = (A.shape[1], A.shape[0]) if transA else A.shape
    Kb, N = (B.shape[1], B.shape[0]) if transB else B.shape
    if K != Kb:
        raise FxpError("contraction lengths differ")
    return M, N, K


def gemm(A, B, transA=False, transB=False, ws=None):
    """int32 C[M,N] = op(A) op(B) for int8 operands."""
    A, B = _dev(A, torch.int8, "A"), _dev(B, torch.int8, "B")
    M, N, K = _gemm_dims(A, B, transA, transB)
    C = torch.empty((M, N), dtype=torch.int32, device=A.device)
    ws = ws if ws is not None else _ws(OP_GEMM, M, N, K, device=A.device)
    _check(lib().fxp_gemm(int(transA), int(transB), M, N, K, _p(A), A.shape[1], _p(B), B.shape[1], _p(C), N, _p(ws),
                          ws.numel(), _stream()), "fxp_gemm")
    return C


def unmap(acc, eA, eB=None, bitsA=8, bitsB=8, out=None):
    acc = _dev(acc, torch.int32, "acc")
    out = out if out is not None else torch.empty(acc.shape, dtype=torch.float32, device=acc.device)
    _check(lib().fxp_unmap(_p(acc), acc.numel(), _p(eA), bitsA, _p(eB), bitsB, _p(out), _stream()), "fxp_unmap")
    return out


def unmap_i8(q, eA, bits=8):
    q = _dev(q, torch.int8, "q")
    out = torch.empty(q.shape, dtype=torch.float32, device=q.device)
    _check(lib().fxp_unmap_i8(_p(q), q.numel(), _p(eA), bits, _p(out), _stream()), "fxp_unmap_i8")
    return out


def gemm_unmap(A, B, eA, eB, transA=False, transB=False, bitsA=8, bitsB=8, ws=None):
    """fp32 C = unmap(op(A) op(B)) with the inverse mapping fused into the GEMM."""
    A, B = _dev(A, torch.int8, "A"), _dev(B, torch.int8, "B")
    M, N, K = _gemm_dims(A, B, transA, transB)
    C = torch.empty((M, N), dtype=torch.float32, device=A.device)
    ws = ws if ws is not None else _ws(OP_GEMM, M, N, K, device=A.device)
    _check(lib().fxp_gemm_unmap(int(transA), int(transB), M, N, K, _p(A), A.shape[1], _p(B), B.shape[1], _p(eA), bitsA,
                                _p(eB), bitsB, _p(C), N, _p(ws), ws.numel(), _stream()), "fxp_gemm_unmap")
    return C


def gemm_unmap_absmax(A, B, eA, eB, absmax, transA=False, transB=False, bitsA=8, bitsB=8, ws=None):
    """gemm_unmap that also raises the abs-max area `absmax` (ABSMAX_WORDS int32 words, bits of max |C|) for map_absmax."""
    A, B = _dev(A, torch.int8, "A"), _dev(B, torch.int8, "B")
    M, N, K = _gemm_dims(A, B, transA, transB)
    C = torch.empty((M, N), dtype=torch.float32, device=A.device)
    ws = ws if ws is not None else _ws(OP_GEMM, M, N, K, device=A.device)
    _check(lib().fxp_gemm_unmap_absmax(int(transA), int(transB), M, N, K, _p(A), A.shape[1], _p(B), B.shape[1], _p(eA), bitsA,
                                   _p(eB), bitsB, _p(C), N, _p(absmax), _p(ws), ws.numel(), _stream()),
           "fxp_gemm_unmap_absmax")
    return C


def map_absmax(x, absmax, seed=0, stream_id=0, rounding=STOCHASTIC, bits=8, want_q=True, want_qT=False):
    """(e_max, q, qT) of x with the scale taken from the abs-max area `absmax` (its maximum = bits of max |x|)."""
    x = _dev(x, torch.float32, "x")
    assert x.dim() == 2
    e = torch.empty(1, dtype=torch.int32, device=x.device)
    q, qT = _map_outputs(x, want_q, want_qT)
    _check(lib().fxp_map_absmax(_p(x), x.shape[0], x.shape[1], _p(absmax), _p(e), _p(q), _p(qT), seed, stream_id, rounding,
                            bits, _stream()), "fxp_map_absmax")
    return e, q, qT


class LayerBuffers:
    """Caller-owned device buffers of one layer shape, allocated once and reused."""

    def __init__(self, M, K, N, device="cuda"):
        i8 = dict(dtype=torch.int8, device=device)
        self.M, self.K, self.N = M, K, N
        self.Xq, self.XqT = torch.empty((M, K), **i8), torch.empty((K, M), **i8)
        self.Wq, self.WqT = torch.empty((K, N), **i8), torch.empty((N, K), **i8)
        self.dYq, self.dYqT = torch.empty((M, N), **i8), torch.empty((N, M), **i8)
        self.e = torch.zeros(3, dtype=torch.int32, device=device)       # eX, eW, e_dY
        self.Y = torch.empty((M, N), dtype=torch.float32, device=device)
        self.dX = torch.empty((M, K), dtype=torch.float32, device=device)
        self.dW = torch.empty((K, N), dtype=torch.float32, device=device)
        nbytes = max(workspace_bytes(OP_LINEAR_FWD, M, N, K), workspace_bytes(OP_LINEAR_BWD, M, N, K), 256)
        self.ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.saved = _Saved(_p(self.Xq), _p(self.XqT), _p(self.Wq), _p(self.WqT), self.e[0:1].data_ptr(),
                            self.e[1:2].data_ptr())

    @property
    def eX(self):
        return self.e[0:1]

    @property
    def eW(self):
        return self.e[1:2]

    @property
    def e_dY(self):
        return self.e[2:3]


def linear_fwd(X, W, buf, seed=0, step=0, rounding=STOCHASTIC, bits=8, guess=False):
    """Y = unmap(map(X) map(W)); fills buf.Xq/XqT/Wq/WqT/eX/eW and returns buf.Y.  guess: the scales buf.e holds
    from the previous call are taken as guesses (fxp_linear_fwd_guess)."""
    X, W = _dev(X, torch.float32, "X"), _dev(W, torch.float32, "W")
    M, K = X.shape
    if W.shape[0] != K or (M, K, W.shape[1]) != (buf.M, buf.K, buf.N):
        raise FxpError("shapes do not match the layer buffers")
    fn = lib().fxp_linear_fwd_guess if guess else lib().fxp_linear_fwd
    _check(fn(_p(X), _p(W), M, K, buf.N, _p(buf.Y), ctypes.byref(buf.saved), seed, step, rounding,
                                bits, _p(buf.ws), buf.ws.numel(), _stream()), "fxp_linear_fwd")
    return buf.Y


def linear_fwd_static(X, W, buf, seed=0, step=0, rounding=STOCHASTIC, bits=8):
    """linear_fwd through the entry point that takes no workspace (its scratch is a device array inside the library)."""
    X, W = _dev(X, torch.float32, "X"), _dev(W, torch.float32, "W")
    M, K = X.shape
    if W.shape[0] != K or (M, K, W.shape[1]) != (buf.M, buf.K, buf.N):
        raise FxpError("shapes do not match the layer buffers")
    _check(lib().fxp_linear_fwd_static(_p(X), _p(W), M, K, buf.N, _p(buf.Y), ctypes.byref(buf.saved), seed, step, rounding,
                                       bits, _stream()), "fxp_linear_fwd_static")
    return buf.Y


def linear_bwd(dY, buf, seed=0, step=0, rounding=STOCHASTIC, bits=8, need_dX=True, need_dW=True, guess=False):
    """(dX, dW) from the upstream gradient and the operands the forward call saved."""
    dY = _dev(dY, torch.float32, "dY")
    if tuple(dY.shape) != (buf.M, buf.N):
        raise FxpError("shapes do not match the layer buffers")
    dX = buf.dX if need_dX else None
    dW = buf.dW if need_dW else None
    fn = lib().fxp_linear_bwd_guess if guess else lib().fxp_linear_bwd
    _check(fn(_p(dY), ctypes.byref(buf.saved), buf.M, buf.K, buf.N, _p(dX), _p(dW), _p(buf.dYq),
                                _p(buf.dYqT), buf.e.data_ptr() + 8, seed, step, rounding, bits, _p(buf.ws),
                                buf.ws.numel(), _stream()), "fxp_linear_bwd")
    return dX, dW


def gemm_batched(A, B, eA=None, eB=None, bitsA=8, bitsB=8):
    """C_b = A_b[M,K] B_b[N,K]^T for dense int8 A[batch,M,K], B[batch,N,K]: int32, or fp32 through the fused
    inverse mapping when the scales eA (and eB) are given."""
    A, B = _dev(A, torch.int8, "A"), _dev(B, torch.int8, "B")
    if A.dim() != 3 or B.dim() != 3 or A.shape[0] != B.shape[0] or A.shape[2] != B.shape[2]:
        raise FxpError("gemm_batched wants A[batch,M,K] and B[batch,N,K]")
    batch, M, K = A.shape
    N = B.shape[1]
    if eA is None:
        C = torch.empty((batch, M, N), dtype=torch.int32, device=A.device)
        _check(lib().fxp_gemm_batched(M, N, K, _p(A), K, M * K, _p(B), K, N * K, _p(C), N, M * N, batch, _stream()),
               "fxp_gemm_batched")
    else:
        C = torch.empty((batch, M, N), dtype=torch.float32, device=A.device)
        _check(lib().fxp_gemm_unmap_batched(M, N, K, _p(A), K, M * K, _p(B), K, N * K, _p(eA), bitsA, _p(eB), bitsB, _p(C),
                                            N, M * N, batch, _stream()), "fxp_gemm_unmap_batched")
    return C


class BmmBuffers:
    """Caller-owned device buffers of one batched product layer (attention matmul), allocated once."""

    def __init__(self, batch, M, K, N, transB=False, device="cuda"):
        i8 = dict(dtype=torch.int8, device=device)
        f32 = dict(dtype=torch.float32, device=device)
        self.batch, self.M, self.K, self.N, self.transB = batch, M, K, N, bool(transB)
        b_shape = (batch, N, K) if transB else (batch, K, N)
        self.Aq, self.AqT = torch.empty((batch, M, K), **i8), torch.empty((K, batch * M), **i8)
        self.Bq, self.BqT = torch.empty(b_shape, **i8), torch.empty((b_shape[2], batch * b_shape[1]), **i8)
        self.dYq, self.dYqT = torch.empty((batch, M, N), **i8), torch.empty((N, batch * M), **i8)
        self.e = torch.zeros(3, dtype=torch.int32, device=device)       # eA, eB, e_dY
        self.Y = torch.empty((batch, M, N), **f32)
        self.dA = torch.empty((batch, M, K), **f32)
        self.dB = torch.empty(b_shape, **f32)
        nbytes = max(workspace_bytes(OP_BMM_FWD, M, N, K), workspace_bytes(OP_BMM_BWD, M, N, K), 256)
        self.ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.saved = _Saved(_p(self.Aq), _p(self.AqT), _p(self.Bq), _p(self.BqT), self.e[0:1].data_ptr(),
                            self.e[1:2].data_ptr())


def bmm_fwd(A, Bm, buf, seed=0, step=0, rounding=STOCHASTIC, bits=8, guess=False):
    """Y_b = unmap(map(A)_b op(map(Bm)_b)); fills buf.Aq/AqT/Bq/BqT/e[0:2] and returns buf.Y."""
    A, Bm = _dev(A, torch.float32, "A"), _dev(Bm, torch.float32, "Bm")
    if tuple(A.shape) != tuple(buf.Aq.shape) or tuple(Bm.shape) != tuple(buf.Bq.shape):
        raise FxpError("shapes do not match the layer buffers")
    _check((lib().fxp_bmm_fwd_guess if guess else lib().fxp_bmm_fwd)(_p(A), _p(Bm), buf.batch, buf.M, buf.K, buf.N, int(buf.transB), _p(buf.Y),
                             ctypes.byref(buf.saved), seed, step, rounding, bits, _p(buf.ws), buf.ws.numel(), _stream()),
           "fxp_bmm_fwd")
    return buf.Y


def bmm_bwd(dY, buf, seed=0, step=0, rounding=STOCHASTIC, bits=8, need_dA=True, need_dB=True, guess=False):
    """(dA, dBm) from the upstream gradient and the operands the forward call saved."""
    dY = _dev(dY, torch.float32, "dY")
    if tuple(dY.shape) != (buf.batch, buf.M, buf.N):
        raise FxpError("shapes do not match the layer buffers")
    dA = buf.dA if need_dA else None
    dB = buf.dB if need_dB else None
    _check((lib().fxp_bmm_bwd_guess if guess else lib().fxp_bmm_bwd)(_p(dY), ctypes.byref(buf.saved), buf.batch, buf.M, buf.K, buf.N, int(buf.transB), _p(dA),
                             _p(dB), _p(buf.dYq), _p(buf.dYqT), buf.e.data_ptr() + 8, seed, step, rounding, bits,
                             _p(buf.ws), buf.ws.numel(), _stream()), "fxp_bmm_bwd")
    return dA, dB


class ConvBuffers:
    """Caller-owned device buffers of one convolution layer (channels-last), allocated once."""

    def __init__(self, N, H, W, C, Cout, KH, KW, stride=1, pad=0, device="cuda"):
        self.shape = _ConvShape(N, H, W, C, Cout, KH, KW, stride, pad)
        self.Ho, self.Wo = (H + 2 * pad - KH) // stride + 1, (W + 2 * pad - KW) // stride + 1
        M, K = N * self.Ho * self.Wo, KH * KW * C
        i8 = dict(dtype=torch.int8, device=device)
        f32 = dict(dtype=torch.float32, device=device)
        self.Xq = torch.empty((N, H, W, C), **i8)
        self.Wq, self.WqT = torch.empty((Cout, K), **i8), torch.empty((K, Cout), **i8)
        self.WqF = torch.empty((C, KH * KW * Cout), **i8)
        self.dYq, self.dYqT = torch.empty((M, Cout), **i8), torch.empty((Cout, M), **i8)
        self.e = torch.zeros(3, dtype=torch.int32, device=device)          # eX, eW, e_dY
        self.Y = torch.empty((N, self.Ho, self.Wo, Cout), **f32)
        self.dX = torch.empty((N, H, W, C), **f32)
        self.dW = torch.empty((Cout, KH, KW, C), **f32)
        nbytes = max(int(lib().fxp_conv2d_workspace_bytes(ctypes.byref(self.shape), 0)),
                     int(lib().fxp_conv2d_workspace_bytes(ctypes.byref(self.shape), 1)), 256)
        self.ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.saved = _ConvSaved(_p(self.Xq), _p(self.Wq), _p(self.WqT), _p(self.WqF), self.e[0:1].data_ptr(),
                                self.e[1:2].data_ptr())


def conv2d_fwd(X, W, buf, seed=0, step=0, rounding=STOCHASTIC, bits=8):
    """Y[N,Ho,Wo,Cout] of the integer convolution layer; X[N,H,W,C], W[Cout,KH,KW,C] fp32."""
    X, W = _dev(X, torch.float32, "X"), _dev(W, torch.float32, "W")
    sh = buf.shape
    if tuple(X.shape) != (sh.N, sh.H, sh.W, sh.C) or tuple(W.shape) != (sh.Cout, sh.KH, sh.KW, sh.C):
        raise FxpError("shapes do not match the convolution buffers")
    _check(lib().fxp_conv2d_fwd(_p(X), _p(W), ctypes.byref(sh), _p(buf.Y), ctypes.byref(buf.saved), seed, step, rounding,
                                bits, _p(buf.ws), buf.ws.numel(), _stream()), "fxp_conv2d_fwd")
    return buf.Y


def conv2d_bwd(dY, buf, seed=0, step=0, rounding=STOCHASTIC, bits=8, need_dX=True, need_dW=True):
    dY = _dev(dY, torch.float32, "dY")
    sh = buf.shape
    if tuple(dY.shape) != (sh.N, buf.Ho, buf.Wo, sh.Cout):
        raise FxpError("shapes do not match the convolution buffers")
    dX = buf.dX if need_dX else None
    dW = buf.dW if need_dW else None
    _check(lib().fxp_conv2d_bwd(_p(dY), ctypes.byref(buf.saved), ctypes.byref(sh), _p(dX), _p(dW), _p(buf.dYq),
                                _p(buf.dYqT), buf.e.data_ptr() + 8, seed, step, rounding, bits, _p(buf.ws),
                                buf.ws.numel(), _stream()), "fxp_conv2d_bwd")
    return dX, dW


def axpy16(x, y, a, out=None, seed=0, step=0, rounding=STOCHASTIC, ws=None):
    """z = x_hat + SR(a_hat * y_hat) in 16-bit fixed point; returns (z, e) with e = int32[3] scales of x, y, a."""
    x, y = _dev(x, torch.float32, "x"), _dev(y, torch.float32, "y")
    if x.shape != y.shape:
        raise FxpError("x and y differ in shape")
    z = out if out is not None else torch.empty_like(x)
    _dev(z, torch.float32, "out")
    e = torch.zeros(3, dtype=torch.int32, device=x.device)
    ws = ws if ws is not None else torch.empty(2 * workspace_bytes(OP_SCALE, 1), dtype=torch.uint8, device=x.device)
    _check(lib().fxp_axpy16(_p(x), _p(y), float(a), x.numel(), _p(z), _p(e), seed, step, rounding, _p(ws), ws.numel(),
                            _stream()), "fxp_axpy16")
    return z, e


class SgdBuffers:
    """Scratch of the int16 SGD step for tensors of up to n elements."""

    def __init__(self, n, device="cuda"):
        self.tmp = torch.empty(n, dtype=torch.float32, device=device)
        self.ws = torch.empty(int(lib().fxp_sgd16_workspace_bytes()), dtype=torch.uint8, device=device)


def sgd16_step(w, g, v, buf, lr, momentum=0.0, weight_decay=0.0, seed=0, step=0, rounding=STOCHASTIC):
    """In-place SGD step on w (and the momentum buffer v, which may be None when momentum == 0)."""
    w, g = _dev(w, torch.float32, "w"), _dev(g, torch.float32, "g")
    if v is not None:
        _dev(v, torch.float32, "v")
    if g.numel() != w.numel() or (v is not None and v.numel() != w.numel()) or buf.tmp.numel() < w.numel():
        raise FxpError("w, g, v and the scratch differ in size")
    _check(lib().fxp_sgd16_step(_p(w), _p(g), _p(v), w.numel(), float(lr), float(momentum), float(weight_decay),
                                _p(buf.tmp), seed, step, rounding, _p(buf.ws), buf.ws.numel(), _stream()),
           "fxp_sgd16_step")
    return w, v


def _desc(x, e, q, qT, stream_id):
    x = _dev(x, torch.float32, "x")
    if x.dim() != 2:
        raise FxpError("x must be a matrix")
    return _MapDesc(_p(x), x.shape[0], x.shape[1], _p(e), _p(q), _p(qT), stream_id)


def map2(xa, ea, xb, eb, seed=0, stream_ids=(0, 1), rounding=STOCHASTIC, bits=8):
    """fxp.map of two tensors (given scales) in one launch; returns ((qa, qaT), (qb, qbT))."""
    outs = [(torch.empty(x.shape, dtype=torch.int8, device=x.device),
             torch.empty((x.shape[1], x.shape[0]), dtype=torch.int8, device=x.device)) for x in (xa, xb)]
    da = _desc(xa, ea, outs[0][0], outs[0][1], stream_ids[0])
    db = _desc(xb, eb, outs[1][0], outs[1][1], stream_ids[1])
    _check(lib().fxp_map2(ctypes.byref(da), ctypes.byref(db), seed, rounding, bits, _stream()), "fxp_map2")
    return outs


def scale_map2(xa, xb, seed=0, stream_ids=(0, 1), rounding=STOCHASTIC, bits=8):
    """fxp.scale_map of two tensors in two launches; returns (e[2], (qa, qaT), (qb, qbT))."""
    e = torch.zeros(2, dtype=torch.int32, device=xa.device)
    outs = [(torch.empty(x.shape, dtype=torch.int8, device=x.device),
             torch.empty((x.shape[1], x.shape[0]), dtype=torch.int8, device=x.device)) for x in (xa, xb)]
    da = _desc(xa, e[0:1], outs[0][0], outs[0][1], stream_ids[0])
    db = _desc(xb, e[1:2], outs[1][0], outs[1][1], stream_ids[1])
    ws = torch.empty(2 * workspace_bytes(OP_SCALE, 1), dtype=torch.uint8, device=xa.device)
    _check(lib().fxp_scale_map2(ctypes.byref(da), ctypes.byref(db), seed, rounding, bits, _p(ws), ws.numel(), _stream()),
           "fxp_scale_map2")
    return e, outs[0], outs[1]


class SgdMultiBuffers:
    """Descriptor table and scratch for the multi-tensor int16 SGD step over fixed lists of parameter tensors."""

    def __init__(self, ws, gs, vs=None, weight_decay=True):
        k = len(ws)
        for t in list(ws) + list(gs) + [v for v in (vs or []) if v is not None]:
            _dev(t, torch.float32, "parameter tensors")
        self.tmps = [torch.empty_like(w) for w in ws] if weight_decay else [None] * k
        self.keep = (list(ws), list(gs), list(vs) if vs is not None else None)      # the table holds raw pointers
        self.table = (_SgdTensor * k)(*[
            _SgdTensor(_p(ws[t]), _p(gs[t]), _p(vs[t]) if vs is not None else None, _p(self.tmps[t]), ws[t].numel())
            for t in range(k)])
        self.count = k
        nbytes = int(lib().fxp_sgd16_multi_workspace_bytes(self.table, k))
        self.ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=ws[0].device)


def sgd16_step_multi(buf, lr, momentum=0.0, weight_decay=0.0, seed=0, step=0, rounding=STOCHASTIC):
    """In-place SGD step on every tensor of buf (own scales per tensor), a handful of launches in all."""
    _check(lib().fxp_sgd16_step_multi(buf.table, buf.count, float(lr), float(momentum), float(weight_decay), seed, step,
                                      rounding, _p(buf.ws), buf.ws.numel(), _stream()), "fxp_sgd16_step_multi")


# ---- serving: a paged cache of mapped keys and values, attention over it, products with 4-bit weights ----
# None of these calls records gradients.

KV_PAGE = 64            # tokens of a page (FXP_KV_PAGE)
KV_TICKET_BYTES = 2048  # of the workspace of fxp_kv_attention, zero between calls (FXP_KV_TICKET_BYTES)
_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def _on_current(t, what):
    """t is a tensor on the current device, whose stream the calls use."""
    at = t.get_device() if isinstance(t, torch.Tensor) else -1
    if at < 0:
        raise FxpError(f"{what} must be a CUDA tensor: libfxp has no CPU path")
    if at != torch._C._cuda_getDevice():
        raise FxpError(f"{what} is on another device than the current one")


def _served(t, what, dims):
    """The type code of a float tensor of `dims` dimensions on the current device whose last dimension is contiguous."""
    _on_current(t, what)
    code = _TYPES.get(t.dtype)
    if code is None or t.dim() != dims or not (t.is_contiguous() or t.stride(-1) == 1 or t.shape[-1] == 1):
        raise FxpError(f"{what} must be a {dims}-dimensional float32, bfloat16 or float16 tensor with a contiguous last dimension")
    return code


def _index(t, what, shape=None, dtype=torch.int32):
    _on_current(t, what)
    if t.dtype != dtype or not t.is_contiguous():
        raise FxpError(f"{what} must be a contiguous {dtype} tensor")
    if shape is not None and t.shape != shape:
        raise FxpError(f"{what} must have the shape {tuple(shape)}")
    return t


def _here(owner, what):
    """`owner` (a cache, tables, buffers, weights) is on the current device; .index is its device's."""
    if owner.index != torch._C._cuda_getDevice():
        raise FxpError(f"{what} is on another device than the current one")


def _row_stride(t, what):
    """Elements from one row of a matrix to the next; rows may not overlap."""
    rows, cols = t.shape
    if rows <= 1:
        return cols
    if t.stride(0) < cols:
        raise FxpError(f"the rows of {what} overlap")
    return t.stride(0)


def _rows_overlap(t):
    """Whether rows (the last dimension) of a tensor share elements."""
    reach = t.shape[-1]                   # elements that the rows so far span
    for stride, n in sorted((t.stride(i), t.shape[i]) for i in range(t.dim() - 1)):
        if n > 1:
            if stride < reach:
                return True
            reach += stride * (n - 1)
    return False


def _span(t):
    """Addresses of a tensor's first byte and of the one behind its last."""
    at, reach = t.data_ptr(), 1
    for stride, n in zip(t.stride(), t.shape):
        reach += stride * (n - 1)
    return at, at + reach * t.element_size()


def _same_rows(a, b):
    """Whether two tensors of one shape are the same elements in the same places."""
    return a.data_ptr() == b.data_ptr() and all(n <= 1 or x == y for n, x, y in zip(a.shape, a.stride(), b.stride()))


def _between(lead, low, high):
    """Whether a sum of i * stride with -n < i < n, one for each (stride, n) of `lead`, smallest strides first, lies between `low` and `high` (both
    excluded)."""
    if not lead:
        return low < 0 < high
    *rest, (stride, n) = lead
    reach = sum(s * (m - 1) for s, m in rest)
    if stride == 0:
        return _between(rest, low, high)
    # where rows do not overlap, the others together reach no further than one stride: few i are left
    first, last = max((low - reach) // stride + 1, 1 - n), min((high + reach - 1) // stride, n - 1)
    return any(_between(rest, low - i * stride, high - i * stride) for i in range(first, last + 1))


def _share(a, b):
    """Whether rows (contiguous last dimensions) of two tensors of one type and of as many rows share elements.  Exact where their strides are
    alike, as those of parts of one buffer are; otherwise whether the tensors' spans meet."""
    (a0, a1), (b0, b1) = _span(a), _span(b)
    if a1 <= b0 or b1 <= a0 or not a.numel() or not b.numel():
        return False
    lead = [(n, stride, other) for n, stride, other in zip(a.shape[:-1], a.stride(), b.stride()) if n > 1]
    if any(stride != other for _, stride, other in lead):
        return True
    # rows of a and of b lie at the same strides: does the distance of two of them leave them short of each other's ends?
    delta = (b0 - a0) // a.element_size()
    return _between(sorted((stride, n) for n, stride, _ in lead), delta - a.shape[-1], delta + b.shape[-1])


class KvCache:
    """Caller-owned cache of one layer: int8 keys [pages, heads, 64, dim], values [pages, heads, 4, dim, 16], scales [pages, heads]."""

    def __init__(self, pages, heads, dim, bits=8, device="cuda"):
        i8, i32 = dict(dtype=torch.int8, device=device), dict(dtype=torch.int32, device=device)
        self._set(torch.empty((pages, heads, KV_PAGE, dim), **i8), torch.empty((pages, heads, KV_PAGE // 16, dim, 16), **i8),
                  torch.ones((pages, heads), **i32), torch.ones((pages, heads), **i32), bits)

    @classmethod
    def of(cls, kq, vq, ek, ev, bits=8):
        """The cache that four tensors of these shapes are."""
        self = cls.__new__(cls)
        self._set(kq, vq, ek, ev, bits)
        return self

    def _set(self, kq, vq, ek, ev, bits):
        if kq.dim() != 4 or kq.shape[2] != KV_PAGE:
            raise FxpError(f"kq must be [pages, heads, {KV_PAGE}, dim]")
        pages, heads, _, dim = kq.shape
        _index(kq, "kq", dtype=torch.int8)
        _index(vq, "vq", (pages, heads, KV_PAGE // 16, dim, 16), torch.int8)
        _index(ek, "ek", (pages, heads))
        _index(ev, "ev", (pages, heads))
        if dim % 16 or dim > 256 or not 2 <= bits <= 8:
            raise FxpError("dim must be a multiple of 16, at most 256, and bits in 2..8")
        self.kq, self.vq, self.ek, self.ev, self.bits = kq, vq, ek, ev, bits
        self.pages, self.heads, self.dim, self.device, self.index = pages, heads, dim, kq.device, kq.get_device()
        self.c = _KvCache(_p(kq), _p(vq), _p(ek), _p(ev), pages, heads, dim, bits)
        self.ref = ctypes.byref(self.c)


class KvTables:
    """Caller-owned tables of up to `requests` requests of `blocks` pages and of a step of up to `tokens` new tokens; all layers of
    a model share them.  The caller frees a finished request by pushing its pages on `free` (free[n_free] and up), raising
    n_free and setting its length to 0; tokens that are taken back (guesses that were rejected) likewise: the pages behind the first
    ceil(length / 64) of its row are pushed and the length lowered - a page that is left in the row is not found again, because a request's
    pages are counted by its length.  Rows of a step's q that belong to a refused request have no tokens of their own in the cache; what
    kv_attention makes of them is to be dropped.  in_place: a step moves lens and n_free on (lens_after is lens); otherwise it leaves them and
    writes lens_after and n_free_after."""

    def __init__(self, requests, blocks, tokens, pages, in_place=True, device="cuda"):
        i32 = dict(dtype=torch.int32, device=device)
        self.requests, self.blocks, self.tokens, self.pages = requests, blocks, tokens, pages
        self.block_table = torch.full((requests, blocks), -1, **i32)
        self.lens = torch.zeros(requests, **i32)
        self.free = torch.arange(pages - 1, -1, -1, **i32)          # page 0 is taken first
        self.n_free = torch.full((1,), pages, **i32)
        self.lens_after = self.lens if in_place else torch.zeros(requests, **i32)
        self.n_free_after = self.n_free if in_place else torch.zeros(1, **i32)
        self.first = torch.zeros(requests + 1, **i32)
        self.slots = torch.full((tokens,), -1, dtype=torch.int64, device=device)
        self.positions = torch.full((tokens,), -1, **i32)
        self.runs = torch.zeros((int(lib().fxp_kv_max_runs(requests, tokens)), 4), **i32)
        self.runs[:, 2] = -1
        self.refused = torch.zeros(requests, **i32)
        self.ws = torch.zeros(256, dtype=torch.uint8, device=device)
        self.index = self.ws.get_device()
        self.c = _KvStep(requests, blocks, tokens, pages, _p(self.lens), _p(self.free), _p(self.n_free), _p(self.block_table), _p(self.lens_after),
                         _p(self.n_free_after), _p(self.first), _p(self.slots), _p(self.positions), _p(self.runs), _p(self.refused))
        self.ref = ctypes.byref(self.c)


def kv_tables(n_new, tab):
    """Room for n_new[b] more tokens of each request, and the step's tables (tab.first, slots, positions, runs, refused); returns tab.  A
    request that finds no room in its row, on the stack or among tab.tokens rows is refused and keeps its length."""
    _index(n_new, "n_new", (tab.requests,))
    _here(tab, "tab")
    _check(lib().fxp_kv_tables(tab.ref, n_new.data_ptr(), tab.ws.data_ptr(), 256, _stream()), "fxp_kv_tables")
    return tab


def _runs(runs):
    runs = _index(runs, "runs")
    if runs.dim() != 2 or runs.shape[1] != 4:
        raise FxpError("runs must be [n, 4]")
    return runs


def kv_append(k, v, cache, runs):
    """Maps the new tokens k, v [tokens, heads, dim] (any strides of the first two) into the cache; runs: KvTables.runs."""
    code = _served(k, "k", 3)
    if _served(v, "v", 3) != code or k.shape != v.shape or k.shape[1:] != (cache.heads, cache.dim):
        raise FxpError("k and v must be [tokens, heads, dim] of the cache and of one type")
    _here(cache, "cache")
    runs = _runs(runs)
    _check(lib().fxp_kv_append(cache.ref, code, k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(), v.stride(0), v.stride(1), k.shape[0],
                               runs.data_ptr(), runs.shape[0], _stream()), "fxp_kv_append")


def kv_load(cache, runs, tokens, dtype=torch.float32, out=None):
    """(k, v) [tokens, heads, dim]: the values that the cached tokens of `runs` stand for; out: the two tensors to fill."""
    runs = _runs(runs)
    _here(cache, "cache")
    shape = (tokens, cache.heads, cache.dim)
    if out is None:
        code = _TYPES.get(dtype)
        if code is None:
            raise FxpError("dtype must be float32, bfloat16 or float16")
        k, v = cache.kq.new_empty(shape, dtype=dtype), cache.kq.new_empty(shape, dtype=dtype)
    else:
        k, v = out
        code = _served(k, "k", 3)
        for t, name in ((k, "k"), (v, "v")):
            if _served(t, name, 3) != code or t.shape != shape or not t.is_contiguous():
                raise FxpError("the outputs must be contiguous [tokens, heads, dim] tensors of one type")
        if _share(k, v):
            raise FxpError("the outputs share elements")
    _check(lib().fxp_kv_load(cache.ref, code, k.data_ptr(), v.data_ptr(), tokens, runs.data_ptr(), runs.shape[0], _stream()), "fxp_kv_load")
    return k, v


class AttentionBuffers:
    """Scratch of kv_attention for up to `requests` requests with `tokens` rows in all; one call at a time."""

    def __init__(self, requests, tokens, q_heads, cache):
        self.nbytes = int(lib().fxp_kv_attention_workspace_bytes(requests, tokens, q_heads, cache.heads, cache.dim))
        if self.nbytes == 0:
            raise FxpError("bad sizes: q_heads must be a multiple of the cache's heads")
        self.ws = torch.empty(self.nbytes, dtype=torch.uint8, device=cache.device)
        self.ws[:KV_TICKET_BYTES].zero_()
        self.index = self.ws.get_device()


def kv_attention(q, cache, tab, buf=None, scale=None, window=0, out=None, lse=None):
    """Attention of the step's rows q [tokens, q_heads, dim] over the cache: causal, over the last `window` tokens where it is > 0.
    scale: dim ** -0.5 by default; out: may be q itself, and shares no elements with it otherwise; lse: [tokens, q_heads] fp32 to fill with
    the logarithms of the softmax's sums.  Rows of bfloat16 and float16 are held in 15 bits under their largest element, and so are the
    softmax's weights of 64 tokens; of float32 in 23: for rows with single elements far above the rest, whose rest matters, pass float32."""
    code = _served(q, "q", 3)
    tokens, q_heads, dim = q.shape
    if tokens != tab.tokens or dim != cache.dim:
        raise FxpError("q must be [tokens, q_heads, dim] of the tables and the cache")
    _here(cache, "cache")
    _here(tab, "tab")
    if out is None:
        out = q.new_empty((tokens, q_heads, dim))
    elif _served(out, "out", 3) != code or out.shape != q.shape or _rows_overlap(out):
        raise FxpError("out must have the shape and type of q, and rows that do not overlap")
    elif not _same_rows(out, q) and _share(q, out):
        raise FxpError("out shares elements with q, and is not q")
    if lse is not None:
        _index(lse, "lse", (tokens, q_heads), torch.float32)
    if buf is None:
        buf = AttentionBuffers(tab.requests, tokens, q_heads, cache)
    _here(buf, "buf")
    _check(lib().fxp_kv_attention(cache.ref, tab.ref, code, q.data_ptr(), q.stride(0), q.stride(1), q_heads, dim ** -0.5 if scale is None else scale,
                                  window, out.data_ptr(), out.stride(0), out.stride(1), _p(lse), buf.ws.data_ptr(), buf.nbytes, _stream()),
           "fxp_kv_attention")
    return out


class W4Weights:
    """A weight matrix [K, N] as packed 4-bit mantissas and scales (the layout of include/fxp.h)."""

    def __init__(self, packed, scales, K, N, group=64):
        if int(lib().fxp_w4_scale_bytes(K, N, group)) == 0:
            raise FxpError("group must be 32, 64 or 128, and K and N in range")
        _index(packed, "packed", dtype=torch.uint8)
        _index(scales, "scales", dtype=torch.uint8)
        if packed.numel() != lib().fxp_w4_packed_bytes(K, N) or scales.numel() != lib().fxp_w4_scale_bytes(K, N, group):
            raise FxpError("packed or scales have another size than K, N and group ask for")
        self.packed, self.scales, self.K, self.N, self.group = packed, scales, K, N, group
        self.pointers, self.index = (packed.data_ptr(), scales.data_ptr()), packed.get_device()


def pack4(W, group=64):
    """W4Weights of a float matrix W [K, N]: mantissas -7..7 rounded to nearest, a scale for each `group` inputs of an output."""
    code = _served(W, "W", 2)
    K, N = W.shape
    nbytes = int(lib().fxp_w4_packed_bytes(K, N)), int(lib().fxp_w4_scale_bytes(K, N, group))
    packed, scales = (torch.empty(max(n, 1), dtype=torch.uint8, device=W.device) for n in nbytes)
    _check(lib().fxp_w4_pack(code, _p(W), _row_stride(W, "W"), K, N, group, _p(packed), _p(scales), _stream()), "fxp_w4_pack")
    return W4Weights(packed, scales, K, N, group)


def linear4(x, w, out=None, ws=None):
    """y [M, N] = x [M, K] W of x's type, W the 4-bit weights w; made for a few rows.  out: may not share elements with x.  bfloat16 and
    float16 x is held in 15 bits under the largest of its `group` elements, float32 in 23."""
    code = _served(x, "x", 2)
    M, K = x.shape
    if K != w.K:
        raise FxpError("x must be [M, K] of the weights")
    _here(w, "w")
    ldy = w.N
    if out is None:
        out = x.new_empty((M, ldy))
    elif _served(out, "out", 2) != code or out.shape != (M, ldy):
        raise FxpError("out must be [M, N] of x's type")
    else:
        ldy = _row_stride(out, "out")
        if _share(x, out):
            raise FxpError("out shares elements with x")
    if ws is not None:
        _index(ws, "ws", dtype=torch.uint8)
    elif M > 2:
        ws = x.new_empty(int(lib().fxp_w4_workspace_bytes(code, M, K, w.group)), dtype=torch.uint8)
    packed, scales = w.pointers
    _check(lib().fxp_w4_linear(code, x.data_ptr(), _row_stride(x, "x"), M, K, w.N, packed, scales, w.group, out.data_ptr(), ldy, _p(ws),
                               ws.numel() if ws is not None else 0, _stream()), "fxp_w4_linear")
    return out


# ---- rotary positions ----
# None of these calls records gradients: rotary_bwd is the gradient of rotary.

# 1 / (2 pi) to 190 bits and more
_TURN = Fraction("0.1591549430918953357688837633725143620344596457404564487476673440588967976")


class Rotary:
    """How heads are turned: pair i of dim / 2 by position * f_i radians, f_i = base ** (-2 i / dim).  Pairs are neighbouring elements (interleaved)
    or elements dim / 2 apart; a head's elements from `dim` on stay.  scaling, for contexts longer than a model was trained with: "linear" (f / factor), "base"
    (base * factor ** (dim / (dim - 2)): the slowest pair becomes `factor` times slower) or "parts" (f where a pair makes `high` turns or more over the
    `original` tokens, f / factor where it makes `low` or fewer, in between in proportion).  amplitude: what turned elements are multiplied by.
    frequencies: f itself, in place of all that.  Made once a model: exact fractions and a copy to the device, under a millisecond for 64 pairs; rotary,
    rotary_bwd and kv_append_rotary take as many positions and tensors with it as there are."""

    def __init__(self, dim, base=10000.0, interleaved=False, scaling=None, factor=1.0, original=0, low=1.0, high=32.0, amplitude=1.0, frequencies=None,
                 device="cuda"):
        if dim < 2 or dim % 2 or dim > 1024:
            raise FxpError("dim must be even, 2 to 1024")
        if not base > 0 or not factor > 0 or not 2.0 ** -126 <= amplitude < 1e30:
            raise FxpError("base, factor and amplitude must be positive, amplitude from 2^-126 to 1e30")
        if frequencies is None:
            if scaling == "base" and dim > 2:
                base = base * factor ** (dim / (dim - 2))
            frequencies = [base ** (-2 * i / dim) for i in range(dim // 2)]
            if scaling == "linear":
                frequencies = [f / factor for f in frequencies]
            elif scaling == "parts":
                if not original > 0 or not low < high:
                    raise FxpError("parts need original > 0 and low < high")
                share = [min(1.0, max(0.0, (original * f / (2 * math.pi) - low) / (high - low))) for f in frequencies]
                frequencies = [f * (s + (1 - s) / factor) for f, s in zip(frequencies, share)]
            elif scaling not in (None, "base"):
                raise FxpError("scaling must be None, 'linear', 'base' or 'parts'")
        frequencies = [float(f) for f in frequencies]
        if len(frequencies) != dim // 2 or not all(math.isfinite(f) for f in frequencies):
            raise FxpError("frequencies must be dim / 2 finite numbers")
        turns = [round(Fraction(f) * _TURN * 2 ** 64) % 2 ** 64 for f in frequencies]
        self.dim, self.interleaved, self.amplitude, self.frequencies = dim, bool(interleaved), float(amplitude), frequencies
        self.turns = torch.tensor([t - 2 ** 64 if t >= 2 ** 63 else t for t in turns], dtype=torch.int64).to(device)
        if not self.turns.is_cuda:
            raise FxpError("the table must be on a GPU: libfxp has no CPU path")
        self.index = self.turns.get_device()
        self.c = _Rotation(_p(self.turns), dim, int(self.interleaved), self.amplitude)
        self.ref = ctypes.byref(self.c)


def _rotary(x, positions, rope, out, backward):
    if not isinstance(x, torch.Tensor) or x.dim() not in (3, 4):
        raise FxpError("x must be [tokens, heads, dim] or [batch, tokens, heads, dim]")
    code = _served(x, "x", x.dim())
    *batch, tokens, heads, dim = x.shape
    _here(rope, "rope")
    _index(positions, "positions")
    if positions.shape != (tokens,) and positions.shape != (*batch, tokens):
        raise FxpError("positions must be [tokens] or [batch, tokens]")
    if rope.dim > dim:
        raise FxpError("the rotated part is larger than a head")
    if out is None:
        out = x.new_empty(x.shape)
        backward |= 0x100                 # FXP_ROTARY_ZERO: no row of it holds what was in the memory before
    elif _served(out, "out", x.dim()) != code or out.shape != x.shape or _rows_overlap(out):
        raise FxpError("out must have the shape and type of x, and rows that do not overlap")
    elif not _same_rows(out, x) and _share(x, out):
        raise FxpError("out shares elements with x, and is not x")
    xs, ys = x.stride(), out.stride()
    xb, yb = (xs[0], ys[0]) if batch else (0, 0)
    _check(lib().fxp_rotary(rope.ref, backward, code, batch[0] if batch else 1, tokens, heads, dim, x.data_ptr(), xb, xs[-3], xs[-2], positions.data_ptr(),
                            tokens if positions.dim() == 2 else 0, out.data_ptr(), yb, ys[-3], ys[-2], _stream()), "fxp_rotary")
    return out


def rotary(x, positions, rope, out=None):
    """x [tokens, heads, dim] or [batch, tokens, heads, dim] (any strides but the last) turned by rope's angles at `positions`, int32 [tokens] or
    [batch, tokens]; rows at negative positions are left as they are in out (zeros, without one).  out: may be x itself, and shares no elements with
    it otherwise."""
    return _rotary(x, positions, rope, out, 0)


def rotary_bwd(dy, positions, rope, out=None):
    """The gradient of rotary for its x, from the upstream gradient dy; arguments as there."""
    return _rotary(dy, positions, rope, out, 1)


def _meet(a, b):
    """Whether tensors [tokens, heads, dim] of one type share elements; exact where a token's heads lie together and tokens are as far apart in both, and
    where both have as many heads, tokens and heads as far apart in both."""
    (a0, a1), (b0, b1) = _span(a), _span(b)
    if a1 <= b0 or b1 <= a0 or not a.numel() or not b.numel():
        return False
    step = a.stride(0)
    reach = [(t.shape[1] - 1) * t.stride(1) + t.shape[2] for t in (a, b)]
    if a.shape[0] > 1 and b.shape[0] > 1 and step == b.stride(0) and max(reach) <= step:
        at = (b0 - a0) // a.element_size() % step       # of a token of b behind one of a
        if at >= reach[0] and at + reach[1] <= step:
            return False
    return a.shape[:2] != b.shape[:2] or _share(a, b)


def kv_append_rotary(k, v, cache, tab, rope, q=None, out=None):
    """kv_append of the step's tokens with the keys turned by `rope` on the way (tab.runs, tab.positions); keys are mapped as they come out of the
    rotation, without a rounding between.  q [tokens, q_heads, dim]: the step's queries, which the same launch turns into out (q itself, or a tensor
    that shares no elements with q, k and v); returns out, or None without q.  Rows of out whose tokens are not written to the cache - of refused
    requests, behind the last one - are left as they are (not set, without out)."""
    code = _served(k, "k", 3)
    if _served(v, "v", 3) != code or k.shape != v.shape or k.shape != (tab.tokens, cache.heads, cache.dim):
        raise FxpError("k and v must be [tokens, heads, dim] of the tables and the cache, and of one type")
    _here(cache, "cache")
    _here(tab, "tab")
    _here(rope, "rope")
    if rope.dim > cache.dim:
        raise FxpError("the rotated part is larger than a head")
    if q is None:
        if out is not None:
            raise FxpError("out goes with q")
        queries = (None, 0, 0, 0, None, 0, 0)
    else:
        if _served(q, "q", 3) != code or q.shape[0] != tab.tokens or q.shape[2] != cache.dim or q.shape[1] < 1 or q.shape[1] % cache.heads:
            raise FxpError("q must be [tokens, q_heads, dim] of k's type, q_heads a multiple of the cache's heads")
        if out is None:
            out = q.new_empty(q.shape)
        else:
            if _served(out, "out", 3) != code or out.shape != q.shape or _rows_overlap(out):
                raise FxpError("out must have the shape and type of q, and rows that do not overlap")
            if not _same_rows(out, q) and _share(q, out):
                raise FxpError("out shares elements with q, and is not q")
            if _meet(out, k) or _meet(out, v):
                raise FxpError("out shares elements with k or v")
        queries = (q.data_ptr(), q.stride(0), q.stride(1), q.shape[1], out.data_ptr(), out.stride(0), out.stride(1))
    _check(lib().fxp_kv_append_rotary(cache.ref, tab.ref, rope.ref, code, k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(), v.stride(0), v.stride(1),
                                      *queries, _stream()), "fxp_kv_append_rotary")
    return out


# ---- products in microscaled 4-bit floating point ----
# None of these calls records gradients: mx4_linear_bwd is the gradient of mx4_linear_fwd.

MX4_PANEL = 256         # columns of a panel of a mapped matrix


def _check_mx4(rc, what):
    if rc == -10:                         # FXP_ERR_VALUE: of these calls' arguments only shared memory has it
        raise FxpError(f"{what}: operands share memory")
    _check(rc, what)


class Mx4:
    """A matrix [rows, cols] in 4-bit floats with a scale for each 32 elements of a row (the layout of include/fxp.h), for products that contract over cols:
    data uint8 [panels, rows, 128], scales uint8 [panels, rows, 8]."""

    def __init__(self, rows, cols, device="cuda"):
        if min(rows, cols) < 0 or max(rows, cols) > 2 ** 24 - 2 ** 16:
            raise FxpError("rows and cols must be between 0 and 2^24 - 2^16")
        self._own(rows, cols, torch.empty(_mx4_bytes(rows, cols), dtype=torch.uint8, device=device))

    @classmethod
    def of(cls, data, scales, rows, cols):
        """The matrix that two tensors of these shapes are; codes and scales behind the last column have to be zeros."""
        self = cls.__new__(cls)
        panels = -(-cols // MX4_PANEL)
        _index(data, "data", (panels, rows, 128), torch.uint8)
        _index(scales, "scales", (panels, rows, 8), torch.uint8)
        self._set(rows, cols, data.data_ptr(), scales.data_ptr(), data.get_device())
        self._data, self._scales = data, scales
        return self

    def _own(self, rows, cols, buf):
        """Codes and scales in one buffer; the tensors of them are made when they are asked for."""
        at = buf.data_ptr()
        self._set(rows, cols, at, at + -(-cols // MX4_PANEL) * rows * 128, buf.get_device())
        self._buf, self._data, self._scales = buf, None, None
        if self.index < 0:
            raise FxpError("a mapped matrix must be on a GPU: libfxp has no CPU path")
        return self

    def _set(self, rows, cols, data, scales, index):
        self.rows, self.cols, self.index = rows, cols, index
        self.c = _Mx4(data, scales, rows, cols)
        self.ref = ctypes.byref(self.c)

    def _split(self):
        panels = -(-self.cols // MX4_PANEL)
        n = panels * self.rows * 128
        self._data, self._scales = self._buf[:n].view(panels, self.rows, 128), self._buf[n:].view(panels, self.rows, 8)

    @property
    def data(self):
        if self._data is None:
            self._split()
        return self._data

    @property
    def scales(self):
        if self._scales is None:
            self._split()
        return self._scales


def _mx4_bytes(rows, cols):
    return -(-cols // MX4_PANEL) * rows * 136


def _mx4_like(x, rows, cols):
    if rows > 2 ** 24 - 2 ** 16 or cols > 2 ** 24 - 2 ** 16:
        raise FxpError("rows and cols must be at most 2^24 - 2^16")
    return Mx4.__new__(Mx4)._own(rows, cols, x.new_empty(_mx4_bytes(rows, cols), dtype=torch.uint8))


def mx4_map(x, rounding=STOCHASTIC, seed=0, stream_id=0, want_q=True, want_qT=False, out=None):
    """(q, qT): x [rows, cols] mapped with blocks along its rows, for products that contract over cols, and x transposed with blocks along its columns, for
    products that contract over rows; None where not wanted.  rounding: NEAREST (ties to even) or STOCHASTIC (Philox words as in map).  out: the pair of
    Mx4 to fill, None where not wanted; they share no memory with x or each other."""
    code = _served(x, "x", 2)
    rows, cols = x.shape
    if out is None:
        q, qT = _mx4_like(x, rows, cols) if want_q else None, _mx4_like(x, cols, rows) if want_qT else None
    else:
        q, qT = out
        for t, shape in ((q, (rows, cols)), (qT, (cols, rows))):
            if t is not None:
                _here(t, "out")
                if (t.rows, t.cols) != shape:
                    raise FxpError("out must be the mapped matrix of x's shape, and of the transposed one")
    if q is None and qT is None:
        raise FxpError("neither copy is wanted")
    _check_mx4(lib().fxp_mx4_map(code, x.data_ptr(), _row_stride(x, "x"), rows, cols, q.ref if q else None, qT.ref if qT else None, seed, stream_id, rounding, _stream()),
               "fxp_mx4_map")
    return q, qT


def mx4_unmap(q, dtype=torch.float32, out=None):
    """The values [rows, cols] that q stands for, in `dtype` or out's type; out shares no memory with q."""
    _here(q, "q")
    if out is None:
        if dtype not in _TYPES:
            raise FxpError("dtype must be float32, bfloat16 or float16")
        out = torch.empty((q.rows, q.cols), dtype=dtype, device=q.index)
    code = _served(out, "out", 2)
    if out.shape != (q.rows, q.cols):
        raise FxpError("out must be [rows, cols] of q")
    _check_mx4(lib().fxp_mx4_unmap(q.ref, code, out.data_ptr(), _row_stride(out, "out"), _stream()), "fxp_mx4_unmap")
    return out


def mx4_gemm(A, B, dtype=torch.float32, out=None, ws=None):
    """C [A.rows, B.rows] = A B^T of two mapped matrices, in `dtype` or out's type; out shares no memory with them."""
    _here(A, "A")
    _here(B, "B")
    if A.cols != B.cols:
        raise FxpError("contraction lengths differ")
    if out is None:
        if dtype not in _TYPES:
            raise FxpError("dtype must be float32, bfloat16 or float16")
        out = torch.empty((A.rows, B.rows), dtype=dtype, device=A.index)
    code = _served(out, "out", 2)
    if out.shape != (A.rows, B.rows):
        raise FxpError("out must be [A.rows, B.rows]")
    if ws is not None:
        _index(ws, "ws", dtype=torch.uint8)
    else:
        nbytes = int(lib().fxp_mx4_gemm_workspace_bytes(A.rows, B.rows, A.cols))
        ws = out.new_empty(nbytes, dtype=torch.uint8) if nbytes else None
    _check_mx4(lib().fxp_mx4_gemm(A.ref, B.ref, code, out.data_ptr(), _row_stride(out, "out"), _p(ws), ws.numel() if ws is not None else 0, _stream()), "fxp_mx4_gemm")
    return out


def mx4_linear(x, w, out=None, ws=None):
    """y [M, N] = x [M, K] W of x's type; w: W transposed and mapped, [N, K] (mx4_map(W, want_q=False, want_qT=True)[1] of W [K, N]).  x is mapped to nearest on the way.  Any M,
    one token to many.  out: may not share elements with x, or memory with w."""
    code = _served(x, "x", 2)
    M, K = x.shape
    if K != w.cols:
        raise FxpError("x must be [M, K] of the weights")
    _here(w, "w")
    ldy = w.rows
    if out is None:
        out = x.new_empty((M, ldy))
    elif _served(out, "out", 2) != code or out.shape != (M, ldy):
        raise FxpError("out must be [M, N] of x's type")
    else:
        ldy = _row_stride(out, "out")
        if _share(x, out):
            raise FxpError("out shares elements with x")
    if ws is not None:
        _index(ws, "ws", dtype=torch.uint8)
    elif M > 4:
        ws = x.new_empty(int(lib().fxp_mx4_linear_workspace_bytes(M, w.rows, K)), dtype=torch.uint8)
    _check_mx4(lib().fxp_mx4_linear(code, x.data_ptr(), _row_stride(x, "x"), M, w.ref, out.data_ptr(), ldy, _p(ws), ws.numel() if ws is not None else 0, _stream()),
               "fxp_mx4_linear")
    return out


class Mx4LayerBuffers:
    """Caller-owned device buffers of one layer in 4-bit floats, allocated once and reused."""

    def __init__(self, M, K, N, dtype=torch.float32, device="cuda"):
        if dtype not in _TYPES:
            raise FxpError("dtype must be float32, bfloat16 or float16")
        self.M, self.K, self.N, self.dtype = M, K, N, dtype
        shapes = dict(X=(M, K), XT=(K, M), W=(K, N), WT=(N, K), dY=(M, N), dYT=(N, M))
        for name, shape in shapes.items():
            setattr(self, name, Mx4(*shape, device=device))
        like = dict(dtype=dtype, device=device)
        self.y, self.dx, self.dw = torch.empty((M, N), **like), torch.empty((M, K), **like), torch.empty((K, N), **like)
        self.ws = torch.empty(int(lib().fxp_mx4_layer_workspace_bytes(M, K, N)), dtype=torch.uint8, device=device)
        self.index = self.ws.get_device()
        self.c = _Mx4Layer(*[getattr(self, name).c for name in shapes])
        self.ref = ctypes.byref(self.c)


def _layer_operand(t, shape, buf, what):
    _on_current(t, what)
    if t.dtype != buf.dtype or t.shape != shape or not t.is_contiguous():
        raise FxpError(f"{what} must be a contiguous {buf.dtype} tensor of the layer's shape")


def mx4_linear_fwd(X, W, buf, seed=0, step=0, rounding=STOCHASTIC):
    """Y = X W in 4-bit floats, X [M, K], W [K, N] of the buffers' type; fills buf.X, XT, W, WT and returns buf.y."""
    _here(buf, "buf")
    _layer_operand(X, (buf.M, buf.K), buf, "X")
    _layer_operand(W, (buf.K, buf.N), buf, "W")
    _check_mx4(lib().fxp_mx4_linear_fwd(_TYPES[buf.dtype], X.data_ptr(), W.data_ptr(), buf.M, buf.K, buf.N, buf.y.data_ptr(), buf.ref, seed, step, rounding,
                                       buf.ws.data_ptr(), buf.ws.numel(), _stream()), "fxp_mx4_linear_fwd")
    return buf.y


def mx4_linear_bwd(dY, buf, seed=0, step=0, rounding=STOCHASTIC, need_dX=True, need_dW=True):
    """(dX, dW) from the upstream gradient and the operands the forward call left in buf."""
    _here(buf, "buf")
    _layer_operand(dY, (buf.M, buf.N), buf, "dY")
    dX, dW = buf.dx if need_dX else None, buf.dw if need_dW else None
    _check_mx4(lib().fxp_mx4_linear_bwd(_TYPES[buf.dtype], dY.data_ptr(), buf.ref, buf.M, buf.K, buf.N, _p(dX), _p(dW), seed, step, rounding, buf.ws.data_ptr(),
                                       buf.ws.numel(), _stream()), "fxp_mx4_linear_bwd")
    return dX, dW
