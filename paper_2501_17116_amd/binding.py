"""ctypes binding of libfp4mi.so: argument marshalling only.

Every function here has the name and the meaning of the C entry point it calls
(include/fp4_linear.h); torch supplies device memory and the current HIP stream,
nothing else.  There is no fallback: if the library is missing or a call fails, an
exception is raised.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
import threading
from typing import NamedTuple, Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfp4mi.so")

FP4_F32, FP4_BF16 = 0, 1
FP4_AXIS_ROW, FP4_AXIS_COL, FP4_AXIS_TENSOR = 0, 1, 2
FP4_OCC_TENSOR, FP4_OCC_TOKEN = 0, 1
FP4_OP_QUANTIZE, FP4_OP_OCC, FP4_OP_FWD, FP4_OP_DGRAD, FP4_OP_WGRAD, FP4_OP_SPMM, FP4_OP_PREPARE, FP4_OP_FWD_MIXED, FP4_OP_BWD = range(9)
FP4_OP_MX_FWD, FP4_OP_MX_DGRAD, FP4_OP_MX_WGRAD, FP4_OP_MX_BWD = range(9, 13)
FP4_OP_HP_NORM_BWD, FP4_OP_HP_EMBED_BWD, FP4_OP_HP_HEAD_FWD, FP4_OP_HP_HEAD_BWD = range(13, 17)
FP4_FMT_E2M1, FP4_FMT_E4M3 = 0, 1

_lib = None


class Fp4Error(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s failed: %s (%d)" % (where, status_string(status), status))


class fp4_fwd_ctx(C.Structure):
    _fields_ = [("gamma_W", C.c_void_p), ("thresholds", C.c_void_p), ("row_ptr", C.c_void_p),
                ("col_idx", C.c_void_p), ("val", C.c_void_p), ("capacity", C.c_int64),
                ("nnz", C.c_void_p), ("scope", C.c_int32)]


class fp4_weight_cache(C.Structure):
    _fields_ = [("qWt", C.c_void_p), ("gamma_W", C.c_void_p), ("qWk", C.c_void_p), ("gamma_Wk", C.c_void_p)]


class fp4_mx(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("lines", C.c_int64), ("length", C.c_int64), ("bits", C.c_int32)]


class hp_norm(C.Structure):
    _fields_ = [("w_before", C.c_void_p), ("w_after", C.c_void_p), ("gate", C.c_void_p), ("ld_gate", C.c_int64), ("scale", C.c_float),
                ("eps", C.c_float)]


def lib() -> C.CDLL:
    """The native library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("native library %s not built: run `python -c 'import __graft_entry__ as g; "
                               "g.build()'` (needs hipcc)" % LIB_PATH)
        L = C.CDLL(LIB_PATH)
        vp, i64, f32, f64, sz, i32 = C.c_void_p, C.c_int64, C.c_float, C.c_double, C.c_size_t, C.c_int
        L.fp4_status_string.restype = C.c_char_p
        L.fp4_status_string.argtypes = [i32]
        L.fp4_workspace_bytes.restype = sz
        L.fp4_workspace_bytes.argtypes = [i32, i64, i64, i64, i32]
        L.fp4_occ_capacity.restype = i64
        L.fp4_occ_capacity.argtypes = [i64, i64, f64]
        L.fp4_quantize.argtypes = [vp, i32, i64, i64, i64, i32, vp, vp, vp, sz, vp]
        L.fp4_quantize_noalloc.argtypes = [vp, i32, i64, i64, i64, i32, vp, vp, vp]
        L.fp4_quantize_noalloc.restype = i32
        L.occ_clamp_residual.argtypes = [vp, i32, i64, i64, i64, f64, vp, vp, vp, vp, vp, vp, vp, i64, vp,
                                         vp, sz, vp]
        L.occ_clamp_residual_token.argtypes = L.occ_clamp_residual.argtypes
        L.occ_clamp_residual_token.restype = i32
        L.fp4_occ_capacity_token.restype = i64
        L.fp4_occ_capacity_token.argtypes = [i64, i64, f64]
        L.fp4_linear_fwd.argtypes = [vp, vp, i32, i64, i64, i64, f64, vp, C.POINTER(fp4_fwd_ctx), vp, sz, vp]
        L.fp4_linear_bwd_dgrad.argtypes = [vp, vp, i32, i64, i64, i64, vp, vp, sz, vp]
        L.fp4_linear_bwd_wgrad.argtypes = [vp, vp, vp, i32, i64, i64, i64, C.POINTER(fp4_fwd_ctx), f32, f32,
                                           vp, vp, sz, vp]
        L.fp4_prepare_weights.argtypes = [vp, i32, i64, i64, C.POINTER(fp4_weight_cache), vp, sz, vp]
        L.fp4_linear_fwd_cached.argtypes = [vp, vp, C.POINTER(fp4_weight_cache), i32, i64, i64, i64, f64, vp,
                                            C.POINTER(fp4_fwd_ctx), vp, sz, vp]
        L.fp4_linear_bwd_dgrad_cached.argtypes = [vp, C.POINTER(fp4_weight_cache), i32, i64, i64, i64, vp, vp, sz, vp]
        for name in ("fp4_prepare_weights", "fp4_linear_fwd_cached", "fp4_linear_bwd_dgrad_cached"):
            getattr(L, name).restype = i32
        L.fp4_linear_bwd.argtypes = [vp, vp, vp, C.POINTER(fp4_weight_cache), i32, i64, i64, i64, C.POINTER(fp4_fwd_ctx),
                                     f32, f32, vp, vp, vp, sz, vp]
        L.fp4_linear_bwd.restype = i32
        L.fp8_quantize.argtypes = [vp, i32, i64, i64, i64, i32, vp, vp, vp, sz, vp]
        L.fp4_gemm_mixed.argtypes = [vp, i32, vp, vp, i32, vp, i64, i64, i64, vp, vp, i32, i64, vp]
        L.fp4_linear_fwd_mixed.argtypes = [vp, vp, i32, i64, i64, i64, i32, i32, f64, vp, C.POINTER(fp4_fwd_ctx), vp, sz, vp]
        L.fp4_linear_fwd_granularity.argtypes = [vp, vp, i32, i64, i64, i64, i32, i32, f64, vp, C.POINTER(fp4_fwd_ctx), vp, sz,
                                                 vp]
        L.fp4_linear_fwd_granularity.restype = i32
        mx = C.POINTER(fp4_mx)
        L.mx_pitch.restype = i64
        L.mx_pitch.argtypes = [i64]
        L.mx_quantize.argtypes = [vp, i32, i64, i64, i64, mx, mx, vp]
        L.mx_dequantize.argtypes = [mx, i32, vp, i32, i64, vp]
        L.mx_gemm.argtypes = [mx, mx, vp, vp, i32, i64, vp]
        L.mx_linear_fwd.argtypes = [vp, i32, i64, i64, i64, i64, i32, mx, vp, i64, mx, vp, sz, vp]
        L.mx_linear_bwd_dgrad.argtypes = [vp, i32, i64, i64, i64, i64, mx, vp, i64, vp, sz, vp]
        L.mx_linear_bwd_wgrad.argtypes = [vp, i32, i64, i64, i64, i64, mx, i32, i32, vp, i64, vp, sz, vp]
        L.mx_linear_bwd.argtypes = [vp, i32, i64, i64, i64, i64, mx, mx, i32, vp, i64, i32, vp, i64, vp, sz, vp]
        L.mx_gemm_by_tile.argtypes = [mx, mx, vp, vp, i32, i64, i32, vp]
        L.mx_gemm_tile.argtypes = [i64, i64, i64, i32, i32, i32, vp]
        for name in ("mx_gemm_by_tile", "mx_gemm_tile", "mx_quantize", "mx_dequantize", "mx_gemm", "mx_linear_fwd", "mx_linear_bwd_dgrad", "mx_linear_bwd_wgrad", "mx_linear_bwd"):
            getattr(L, name).restype = i32
        hp = C.POINTER(hp_norm)
        L.hp_norm_fwd.argtypes = [hp, i32, i64, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp]
        L.hp_norm_bwd.argtypes = [hp, i32, i64, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, i64, vp, i64, vp, i64, vp, vp, i32, vp, sz, vp]
        L.hp_embed_fwd.argtypes = [vp, i32, i64, i64, i64, vp, i64, f32, vp, i64, vp]
        L.hp_embed_bwd.argtypes = [vp, i32, i64, i64, i64, vp, i64, f32, i32, vp, i64, vp, sz, vp]
        L.hp_head_fwd.argtypes = [vp, vp, vp, i32, i64, i64, i64, i64, i64, vp, vp, vp, sz, vp]
        L.hp_head_bwd.argtypes = [vp, vp, vp, vp, vp, i32, i64, i64, i64, i64, i64, vp, i64, vp, i32, i64, i32, vp, sz, vp]
        for name in ("hp_norm_fwd", "hp_norm_bwd", "hp_embed_fwd", "hp_embed_bwd", "hp_head_fwd", "hp_head_bwd"):
            getattr(L, name).restype = i32
        L.fp8_host_round_codes.argtypes = [vp, i64, vp]
        for name in ("fp8_quantize", "fp4_gemm_mixed", "fp4_linear_fwd_mixed", "fp8_host_round_codes"):
            getattr(L, name).restype = i32
        L.fp4_gemm.argtypes = [vp, vp, vp, vp, i64, i64, i64, vp, vp, i32, i64, vp]
        L.fp4_unpack.argtypes = [vp, i64, i64, vp, vp]
        L.fp4_dge_apply.argtypes = [vp, vp, i32, vp, i64, i64, f32, f32, vp, vp]
        L.fp4_residual_spmm.argtypes = [vp, vp, vp, i64, i64, vp, i32, i64, vp, vp, sz, vp]
        L.fp4_residual_spmm_general.argtypes = L.fp4_residual_spmm.argtypes
        L.fp4_residual_spmm_bounded.argtypes = [vp, vp, vp, i64, i64, i64, vp, i32, i64, vp, vp, sz, vp]
        L.fp4_residual_spmm_gathers.argtypes = [i64, i64, i64, i32, i64]
        L.fp4_residual_spmm_gathers.restype = i32
        L.fp4_quantize_cols_folds.argtypes = [i64, i64]
        L.fp4_quantize_cols_folds.restype = i32
        L.fp4_select_route.argtypes = [i64, i64, i64, i32]
        L.fp4_select_route.restype = i32
        L.fp4_select_beside.argtypes = [i64, i64, i64, i32, i32]
        L.fp4_select_beside.restype = i32
        L.fp4_transpose_beside.argtypes = [i64, i64, i64, i32]
        L.fp4_transpose_beside.restype = i32
        L.fp4_count_beside.argtypes = [i64, i64, i64, i32, i32, i64, i32]
        L.fp4_count_beside.restype = i32
        L.fp4_residual_transpose_positions.argtypes = [i64, i64]
        L.fp4_residual_transpose_positions.restype = i32
        L.fp4_residual_transpose.argtypes = [vp, vp, vp, vp, i64, i64, i64, i32, vp, vp, vp, vp, sz, vp]
        L.fp4_residual_transpose.restype = i32
        L.fp4_host_round_codes.argtypes = [vp, i64, vp]
        L.fp4_device_round_codes.argtypes = [vp, i64, vp, vp]
        L.fp4_device_round_sweep.argtypes = [vp, vp]
        L.fp4_probe_mfma.argtypes = [vp, i64, i32, i32, vp, vp]
        L.fp4_probe_mfma.restype = i32
        L.fp4_probe_copy.argtypes = [vp, vp, i64, vp]
        L.fp4_probe_copy.restype = i32
        L.fp4_gemm_tiling.argtypes = [i64, i64, i64, i32, i32, i32, i32, i32, vp, vp]
        L.fp4_gemm_tiling.restype = i32
        L.fp4_gemm_splits.argtypes = [i64, i64, i64, i32, i32]
        L.fp4_gemm_splits.restype = i32
        L.fp4_trace_begin.argtypes = [i32]
        L.fp4_trace_begin.restype = i32
        L.fp4_trace_end.argtypes = [vp, vp, i32]
        L.fp4_trace_end.restype = i32
        for name in ("fp4_quantize", "occ_clamp_residual", "fp4_linear_fwd", "fp4_linear_bwd_dgrad",
                     "fp4_linear_bwd_wgrad", "fp4_gemm", "fp4_unpack", "fp4_dge_apply", "fp4_residual_spmm",
                     "fp4_host_round_codes", "fp4_device_round_codes", "fp4_device_round_sweep"):
            getattr(L, name).restype = i32
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().fp4_status_string(int(status)).decode()


def _check(status: int, where: str):
    if status != 0:
        raise Fp4Error(status, where)


_DTYPES = {torch.float32: FP4_F32, torch.bfloat16: FP4_BF16}


def _dt(t: torch.Tensor) -> int:
    dt = _DTYPES.get(t.dtype)
    if dt is None:
        raise TypeError("dtype must be float32 or bfloat16, got %s" % t.dtype)
    return dt


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice()))


def _current(index: int) -> int:
    """index, if that is the current device: launches go there, and another one's addresses mean nothing to them."""
    if index != torch._C._cuda_getDevice():
        raise ValueError("tensors and workspaces must live on the current device, cuda:%d; this one is on cuda:%d" % (torch._C._cuda_getDevice(), index))
    return index


def _dev_check(*ts):
    current = None
    for t in ts:
        if t is not None:
            if not t.is_cuda:
                raise ValueError("tensors must live on the GPU")
            if t.device.index != current:
                current = _current(t.device.index)
            if not t.is_contiguous():
                raise ValueError("tensors must be contiguous")


def workspace_bytes(op: int, M: int, K: int, N: int, dt: int) -> int:
    return int(lib().fp4_workspace_bytes(op, M, K, N, dt))


def occ_capacity(rows: int, cols: int, alpha: float) -> int:
    return int(lib().fp4_occ_capacity(rows, cols, float(alpha)))


class Workspace:
    """A growable device byte buffer handed to the entry points as their workspace.

    One Workspace serves calls that stream order serializes (the ABI's workspace rule): use one
    per stream and thread, since a call is several launches and two threads' launches mix on a
    stream, and one per captured graph that is replayed beside other calls.  Growing keeps the
    outgrown buffers alive until release(), because kernels enqueued earlier may still be running
    in them, captured graphs may replay in them, and torch's allocator knows nothing of streams
    other than the one a tensor was allocated on.  A buffer that takes another's place is at least
    half as large again, so that all of them together stay below 4.5 times what was asked for,
    whatever the steps it comes in."""

    def __init__(self, device="cuda"):
        self.device = device
        self.buf = torch.empty(0, dtype=torch.uint8, device=device)
        self._outgrown = []

    def get(self, nbytes: int) -> torch.Tensor:
        buf = self._sized(nbytes)
        if buf.is_cuda:
            _current(buf.device.index)
        return buf

    def _sized(self, nbytes: int) -> torch.Tensor:
        had = self.buf.numel()
        if had < nbytes:
            try:
                buf = torch.empty(max(nbytes, had + had // 2), dtype=torch.uint8, device=self.device)
            except torch.OutOfMemoryError:
                buf = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            if had:
                self._outgrown.append(self.buf)
            self.buf = buf
        return self.buf

    def release(self) -> None:
        """Drop outgrown buffers; call after the streams that used them have been synchronized."""
        self._outgrown.clear()


_thread = threading.get_ident
_default_ws = {}   # (device index, stream handle, thread) -> Workspace: never shared between streams or threads


def _default_workspace(device_index: int, stream: int) -> Workspace:
    """The calling thread's for its stream.  (A thread that has ended leaves its own to the next one of its number, whose calls come later.)"""
    key = (device_index, stream, _thread())
    ws = _default_ws.get(key)
    if ws is None:
        ws = _default_ws[key] = Workspace(torch.device("cuda", device_index))
    return ws


_releasing = threading.Lock()


def release_outgrown() -> None:
    """Give back what the workspaces that calls take by themselves (ws=None) have outgrown, after waiting for the devices it is on.  Graphs that
    were captured with such a workspace must not be replayed afterwards; those with a Workspace of their own are not concerned."""
    with _releasing:
        old = [(key[0], ws, len(ws._outgrown)) for key, ws in _default_ws.copy().items() if ws._outgrown]
        for device in sorted({device for device, _, _ in old}):
            torch.cuda.synchronize(device)
        for _, ws, n in old:
            del ws._outgrown[:n]     # what other threads have outgrown meanwhile stands behind


def _ws(nbytes: int, ws: Optional[Workspace]) -> torch.Tensor:
    if ws is None:
        return _default_workspace(torch.cuda.current_device(), torch.cuda.current_stream().cuda_stream)._sized(nbytes)
    return ws.get(nbytes)


class FwdCtx:
    """Device buffers the forward pass fills for the weight-gradient pass."""

    def __init__(self, M: int, K: int, N: int, alpha: float, device="cuda", scope: int = FP4_OCC_TENSOR):
        cap = occ_capacity(M, K, alpha) if alpha < 1.0 else 0
        self.alpha = float(alpha)
        self.scope = scope
        self.gamma_W = torch.empty(N, dtype=torch.float32, device=device)
        self.thresholds = torch.empty(2 * M if scope == FP4_OCC_TOKEN else 2, dtype=torch.float32, device=device)
        self.row_ptr = torch.empty(M + 1, dtype=torch.int64, device=device)
        self.col_idx = torch.empty(max(cap, 1), dtype=torch.int32, device=device)
        self.val = torch.empty(max(cap, 1), dtype=torch.float32, device=device)
        self.nnz = torch.zeros(1, dtype=torch.int64, device=device)
        self.capacity = cap
        self.c = fp4_fwd_ctx(self.gamma_W.data_ptr(), self.thresholds.data_ptr(), self.row_ptr.data_ptr(),
                             self.col_idx.data_ptr(), self.val.data_ptr(), cap, self.nnz.data_ptr(), scope)


def fp4_quantize(x: torch.Tensor, axis: int, ws: Optional[Workspace] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    _dev_check(x)
    rows, cols = x.shape
    if axis == FP4_AXIS_ROW:
        codes = torch.empty((rows, cols // 2), dtype=torch.uint8, device=x.device)
        gamma = torch.empty(rows, dtype=torch.float32, device=x.device)
    elif axis == FP4_AXIS_TENSOR:   # one scale for the whole tensor, codes laid out as for ROW
        codes = torch.empty((rows, cols // 2), dtype=torch.uint8, device=x.device)
        gamma = torch.empty(1, dtype=torch.float32, device=x.device)
    else:
        codes = torch.empty((cols, rows // 2), dtype=torch.uint8, device=x.device)
        gamma = torch.empty(cols, dtype=torch.float32, device=x.device)
    nb = workspace_bytes(FP4_OP_QUANTIZE, rows, cols, 0, _dt(x))
    w = _ws(nb, ws)
    _check(lib().fp4_quantize(_ptr(x), _dt(x), rows, cols, cols, axis, _ptr(codes), _ptr(gamma), _ptr(w),
                              w.numel(), _stream()), "fp4_quantize")
    return codes, gamma


def fp4_quantize_noalloc(x: torch.Tensor, axis: int, codes: torch.Tensor, gamma: torch.Tensor) -> None:
    """fp4_quantize without a workspace, into outputs the caller brings (nothing is allocated)."""
    _dev_check(x, codes, gamma)
    rows, cols = x.shape
    _check(lib().fp4_quantize_noalloc(_ptr(x), _dt(x), rows, cols, cols, axis, _ptr(codes), _ptr(gamma),
                                      _stream()), "fp4_quantize_noalloc")


def occ_clamp_residual(x: torch.Tensor, alpha: float, want_codes: bool = True, want_clamped: bool = False,
                       capacity: Optional[int] = None, ws: Optional[Workspace] = None,
                       scope: int = FP4_OCC_TENSOR) -> dict:
    _dev_check(x)
    rows, cols = x.shape
    token = scope == FP4_OCC_TOKEN
    if capacity is not None:
        cap = capacity
    elif token:
        cap = int(lib().fp4_occ_capacity_token(rows, cols, float(alpha)))
    else:
        cap = occ_capacity(rows, cols, alpha)
    dev = x.device
    out = {
        "thresholds": torch.empty(2 * rows if token else 2, dtype=torch.float32, device=dev),
        "codes": torch.empty((rows, cols // 2), dtype=torch.uint8, device=dev) if want_codes else None,
        "gamma": torch.empty(rows, dtype=torch.float32, device=dev) if want_codes else None,
        "x_clamped": torch.empty_like(x) if want_clamped else None,
        "row_ptr": torch.empty(rows + 1, dtype=torch.int64, device=dev),
        "col_idx": torch.empty(max(cap, 1), dtype=torch.int32, device=dev),
        "val": torch.empty(max(cap, 1), dtype=torch.float32, device=dev),
        "nnz": torch.zeros(1, dtype=torch.int64, device=dev),
    }
    nb = workspace_bytes(FP4_OP_OCC, rows, cols, 0, _dt(x))
    w = _ws(nb, ws)
    fn = lib().occ_clamp_residual_token if token else lib().occ_clamp_residual
    _check(fn(_ptr(x), _dt(x), rows, cols, cols, float(alpha), _ptr(out["thresholds"]),
                                    _ptr(out["codes"]), _ptr(out["gamma"]), _ptr(out["x_clamped"]),
                                    _ptr(out["row_ptr"]), _ptr(out["col_idx"]), _ptr(out["val"]), cap,
                                    _ptr(out["nnz"]), _ptr(w), w.numel(), _stream()), "occ_clamp_residual")
    return out


def fp4_linear_fwd(A: torch.Tensor, W: torch.Tensor, alpha: float, ctx: Optional[FwdCtx] = None,
                   Y: Optional[torch.Tensor] = None, ws: Optional[Workspace] = None, scope: int = FP4_OCC_TENSOR):
    """scope only matters when no ctx is passed (a ctx carries its own)."""
    _dev_check(A, W, Y)
    M, K = A.shape
    K2, N = W.shape
    if K2 != K or A.dtype != W.dtype:
        raise ValueError("A [M,K] and W [K,N] must agree in K and dtype")
    if ctx is None:
        ctx = FwdCtx(M, K, N, alpha, A.device, scope)
    if Y is None:
        Y = torch.empty((M, N), dtype=A.dtype, device=A.device)
    nb = workspace_bytes(FP4_OP_FWD, M, K, N, _dt(A))
    w = _ws(nb, ws)
    _check(lib().fp4_linear_fwd(_ptr(A), _ptr(W), _dt(A), M, K, N, float(alpha), _ptr(Y), C.byref(ctx.c),
                                _ptr(w), w.numel(), _stream()), "fp4_linear_fwd")
    return Y, ctx


class WeightCache:
    """Device buffers for W's two quantizations (forward's per-output-channel, dgrad's per-input-channel)."""

    def __init__(self, K: int, N: int, device="cuda"):
        self.K, self.N = K, N
        self.qWt = torch.empty((N, K // 2), dtype=torch.uint8, device=device)
        self.gamma_W = torch.empty(N, dtype=torch.float32, device=device)
        self.qWk = torch.empty((K, N // 2), dtype=torch.uint8, device=device)
        self.gamma_Wk = torch.empty(K, dtype=torch.float32, device=device)
        self.c = fp4_weight_cache(self.qWt.data_ptr(), self.gamma_W.data_ptr(), self.qWk.data_ptr(),
                                  self.gamma_Wk.data_ptr())


def fp4_prepare_weights(W: torch.Tensor, wq: Optional[WeightCache] = None, ws: Optional[Workspace] = None) -> WeightCache:
    _dev_check(W)
    K, N = W.shape
    if wq is None:
        wq = WeightCache(K, N, W.device)
    w = _ws(workspace_bytes(FP4_OP_PREPARE, 0, K, N, _dt(W)), ws)
    _check(lib().fp4_prepare_weights(_ptr(W), _dt(W), K, N, C.byref(wq.c), _ptr(w), w.numel(), _stream()),
           "fp4_prepare_weights")
    return wq


def fp4_linear_fwd_cached(A: torch.Tensor, W: torch.Tensor, wq: WeightCache, alpha: float,
                          ctx: Optional[FwdCtx] = None, Y: Optional[torch.Tensor] = None,
                          ws: Optional[Workspace] = None):
    _dev_check(A, W, Y)
    M, K = A.shape
    K2, N = W.shape
    if K2 != K or A.dtype != W.dtype or (wq.K, wq.N) != (K, N):
        raise ValueError("A [M,K], W [K,N] and the weight cache must agree")
    if ctx is None:
        ctx = FwdCtx(M, K, N, alpha, A.device)
    if Y is None:
        Y = torch.empty((M, N), dtype=A.dtype, device=A.device)
    w = _ws(workspace_bytes(FP4_OP_FWD, M, K, N, _dt(A)), ws)
    _check(lib().fp4_linear_fwd_cached(_ptr(A), _ptr(W), C.byref(wq.c), _dt(A), M, K, N, float(alpha), _ptr(Y),
                                       C.byref(ctx.c), _ptr(w), w.numel(), _stream()), "fp4_linear_fwd_cached")
    return Y, ctx


def fp4_linear_bwd_dgrad_cached(dY: torch.Tensor, wq: WeightCache, dA: Optional[torch.Tensor] = None,
                                ws: Optional[Workspace] = None) -> torch.Tensor:
    _dev_check(dY, dA)
    M, N = dY.shape
    K = wq.K
    if wq.N != N:
        raise ValueError("dY [M,N] and the weight cache must agree in N")
    if dA is None:
        dA = torch.empty((M, K), dtype=dY.dtype, device=dY.device)
    w = _ws(workspace_bytes(FP4_OP_DGRAD, M, K, N, _dt(dY)), ws)
    _check(lib().fp4_linear_bwd_dgrad_cached(_ptr(dY), C.byref(wq.c), _dt(dY), M, K, N, _ptr(dA), _ptr(w),
                                             w.numel(), _stream()), "fp4_linear_bwd_dgrad_cached")
    return dA


def fp4_linear_bwd_dgrad(dY: torch.Tensor, W: torch.Tensor, dA: Optional[torch.Tensor] = None,
                         ws: Optional[Workspace] = None) -> torch.Tensor:
    _dev_check(dY, W, dA)
    M, N = dY.shape
    K, N2 = W.shape
    if N2 != N or dY.dtype != W.dtype:
        raise ValueError("dY [M,N] and W [K,N] must agree in N and dtype")
    if dA is None:
        dA = torch.empty((M, K), dtype=dY.dtype, device=dY.device)
    nb = workspace_bytes(FP4_OP_DGRAD, M, K, N, _dt(dY))
    w = _ws(nb, ws)
    _check(lib().fp4_linear_bwd_dgrad(_ptr(dY), _ptr(W), _dt(dY), M, K, N, _ptr(dA), _ptr(w), w.numel(),
                                      _stream()), "fp4_linear_bwd_dgrad")
    return dA


def fp4_linear_bwd_wgrad(A: torch.Tensor, dY: torch.Tensor, W: torch.Tensor, ctx: FwdCtx, dge_k: float = 5.0,
                         dge_cap: float = 3.0, dW: Optional[torch.Tensor] = None,
                         ws: Optional[Workspace] = None) -> torch.Tensor:
    _dev_check(A, dY, W, dW)
    M, K = A.shape
    _, N = W.shape
    if dY.shape != (M, N) or W.shape != (K, N) or not (A.dtype == dY.dtype == W.dtype):
        raise ValueError("shape / dtype mismatch")
    if dW is None:
        dW = torch.empty((K, N), dtype=torch.float32, device=A.device)
    nb = workspace_bytes(FP4_OP_WGRAD, M, K, N, _dt(A))
    w = _ws(nb, ws)
    _check(lib().fp4_linear_bwd_wgrad(_ptr(A), _ptr(dY), _ptr(W), _dt(A), M, K, N, C.byref(ctx.c),
                                      float(dge_k), float(dge_cap), _ptr(dW), _ptr(w), w.numel(), _stream()),
           "fp4_linear_bwd_wgrad")
    return dW


def fp4_linear_bwd(dY: torch.Tensor, A: torch.Tensor, W: torch.Tensor, ctx: FwdCtx, dge_k: float = 5.0, dge_cap: float = 3.0,
                   wq: Optional["WeightCache"] = None, dA: Optional[torch.Tensor] = None, dW: Optional[torch.Tensor] = None,
                   ws: Optional[Workspace] = None):
    """Both gradients in one call (dY read once for both of its quantizations).  Returns (dA, dW)."""
    _dev_check(dY, A, W, dA, dW)
    M, K = A.shape
    _, N = W.shape
    if dY.shape != (M, N) or W.shape != (K, N) or not (A.dtype == dY.dtype == W.dtype):
        raise ValueError("shape / dtype mismatch")
    if dA is None:
        dA = torch.empty((M, K), dtype=dY.dtype, device=dY.device)
    if dW is None:
        dW = torch.empty((K, N), dtype=torch.float32, device=dY.device)
    w = _ws(workspace_bytes(FP4_OP_BWD, M, K, N, _dt(A)), ws)
    _check(lib().fp4_linear_bwd(_ptr(dY), _ptr(A), _ptr(W), C.byref(wq.c) if wq is not None else None, _dt(A), M, K, N,
                                C.byref(ctx.c), float(dge_k), float(dge_cap), _ptr(dA), _ptr(dW), _ptr(w), w.numel(),
                                _stream()), "fp4_linear_bwd")
    return dA, dW


def fp4_gemm(codes_l: torch.Tensor, gamma_l: Optional[torch.Tensor], codes_rt: torch.Tensor,
             gamma_r: Optional[torch.Tensor], out_dtype=torch.float32, addend: Optional[torch.Tensor] = None,
             out: Optional[torch.Tensor] = None) -> torch.Tensor:
    _dev_check(codes_l, gamma_l, codes_rt, gamma_r, addend)
    P, kb = codes_l.shape
    Q, kb2 = codes_rt.shape
    if kb != kb2:
        raise ValueError("operands disagree in K")
    ldo = Q
    if out is None:
        ldo = (Q + 7) // 8 * 8          # the ABI wants a leading dimension that is a multiple of 8
        full = torch.empty((P, ldo), dtype=out_dtype, device=codes_l.device)
        out = full[:, :Q]
        if addend is not None and ldo != Q:
            pad = torch.zeros((P, ldo), dtype=torch.float32, device=codes_l.device)
            pad[:, :Q] = addend
            addend = pad
    _check(lib().fp4_gemm(_ptr(codes_l), _ptr(gamma_l), _ptr(codes_rt), _ptr(gamma_r), P, Q, 2 * kb,
                          _ptr(addend), _ptr(out), _dt(out), ldo, _stream()), "fp4_gemm")
    return out


def fp8_quantize(x: torch.Tensor, axis: int, ws: Optional[Workspace] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """E4M3 codes (one per byte; COL: transposed) and scales gamma = 448 / absmax."""
    _dev_check(x)
    rows, cols = x.shape
    shape, n = ((rows, cols), rows) if axis == FP4_AXIS_ROW else ((cols, rows), cols)
    codes = torch.empty(shape, dtype=torch.uint8, device=x.device)
    gamma = torch.empty(n, dtype=torch.float32, device=x.device)
    w = _ws(workspace_bytes(FP4_OP_QUANTIZE, rows, cols, 0, _dt(x)), ws)
    _check(lib().fp8_quantize(_ptr(x), _dt(x), rows, cols, cols, axis, _ptr(codes), _ptr(gamma), _ptr(w), w.numel(),
                              _stream()), "fp8_quantize")
    return codes, gamma


def fp4_gemm_mixed(codes_l: torch.Tensor, fmt_l: int, gamma_l: Optional[torch.Tensor], codes_rt: torch.Tensor, fmt_r: int,
                   gamma_r: Optional[torch.Tensor], out_dtype=torch.float32, addend: Optional[torch.Tensor] = None):
    _dev_check(codes_l, gamma_l, codes_rt, gamma_r, addend)
    P, Q = codes_l.shape[0], codes_rt.shape[0]
    Kc = codes_l.shape[1] * (1 if fmt_l == FP4_FMT_E4M3 else 2)
    if Kc != codes_rt.shape[1] * (1 if fmt_r == FP4_FMT_E4M3 else 2):
        raise ValueError("operands disagree in K")
    if Q % 8:
        raise ValueError("Q must be a multiple of 8 here")
    out = torch.empty((P, Q), dtype=out_dtype, device=codes_l.device)
    _check(lib().fp4_gemm_mixed(_ptr(codes_l), fmt_l, _ptr(gamma_l), _ptr(codes_rt), fmt_r, _ptr(gamma_r), P, Q, Kc,
                                _ptr(addend), _ptr(out), _dt(out), Q, _stream()), "fp4_gemm_mixed")
    return out


def fp4_linear_fwd_mixed(A: torch.Tensor, W: torch.Tensor, act_fmt: int, wgt_fmt: int, alpha: float = 1.0,
                         ctx: Optional[FwdCtx] = None, Y: Optional[torch.Tensor] = None, ws: Optional[Workspace] = None):
    _dev_check(A, W, Y)
    M, K = A.shape
    K2, N = W.shape
    if K2 != K or A.dtype != W.dtype:
        raise ValueError("A [M,K] and W [K,N] must agree in K and dtype")
    if ctx is None:
        ctx = FwdCtx(M, K, N, alpha, A.device)
    if Y is None:
        Y = torch.empty((M, N), dtype=A.dtype, device=A.device)
    w = _ws(workspace_bytes(FP4_OP_FWD_MIXED, M, K, N, _dt(A)), ws)
    _check(lib().fp4_linear_fwd_mixed(_ptr(A), _ptr(W), _dt(A), M, K, N, act_fmt, wgt_fmt, float(alpha), _ptr(Y),
                                      C.byref(ctx.c), _ptr(w), w.numel(), _stream()), "fp4_linear_fwd_mixed")
    return Y, ctx


def fp4_linear_fwd_granularity(A: torch.Tensor, W: torch.Tensor, act_tensorwise: bool, wgt_tensorwise: bool,
                               alpha: float = 1.0, ctx: Optional[FwdCtx] = None, Y: Optional[torch.Tensor] = None,
                               ws: Optional[Workspace] = None):
    """Forward pass with tensor-wise scaling of the activations and / or the weights."""
    _dev_check(A, W, Y)
    M, K = A.shape
    K2, N = W.shape
    if K2 != K or A.dtype != W.dtype:
        raise ValueError("A [M,K] and W [K,N] must agree in K and dtype")
    if ctx is None:
        ctx = FwdCtx(M, K, N, alpha, A.device)
    if Y is None:
        Y = torch.empty((M, N), dtype=A.dtype, device=A.device)
    w = _ws(workspace_bytes(FP4_OP_FWD, M, K, N, _dt(A)), ws)
    _check(lib().fp4_linear_fwd_granularity(_ptr(A), _ptr(W), _dt(A), M, K, N, int(bool(act_tensorwise)),
                                            int(bool(wgt_tensorwise)), float(alpha), _ptr(Y), C.byref(ctx.c), _ptr(w),
                                            w.numel(), _stream()), "fp4_linear_fwd_granularity")
    return Y, ctx


def fp8_host_round_codes(x_host):
    """numpy fp32 array (host) -> uint8 E4M3 codes, through the library's own rounding routine."""
    import numpy as np
    x = np.ascontiguousarray(x_host, dtype=np.float32)
    out = np.empty(x.shape, dtype=np.uint8)
    _check(lib().fp8_host_round_codes(x.ctypes.data_as(C.c_void_p), x.size, out.ctypes.data_as(C.c_void_p)),
           "fp8_host_round_codes")
    return out


MX_BLOCK, MX_PITCH = 32, 512


def mx_pitch(length: int) -> int:
    """Elements that a line of `length` takes in an MX tensor."""
    return -(-length // MX_PITCH) * MX_PITCH


class MxTensor:
    """Codes and block scales of a matrix, blocks of 32 along its lines.

    codes [lines, mx_pitch(length) / 2] (4 bits) or [2, lines, mx_pitch(length) / 2] (8 bits), scales [lines, mx_pitch(length) / 32],
    uint8.  transposed: the lines are the columns of the matrix that the tensor stands for."""

    __slots__ = ("_codes", "_scales", "_room", "bits", "lines", "length", "transposed", "device", "use", "c", "ref")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, length: int, transposed: bool = False):
        pitch, shape, lines = mx_pitch(length), tuple(codes.shape), scales.shape[0]
        if codes.dtype != torch.uint8 or scales.dtype != torch.uint8:
            raise TypeError("codes and scales must be uint8")
        if tuple(scales.shape) != (lines, pitch // MX_BLOCK) or shape not in ((lines, pitch // 2), (2, lines, pitch // 2)):
            raise ValueError("codes %s and scales %s do not hold lines of %d elements" % (shape, tuple(scales.shape), length))
        if not codes.is_cuda or codes.device != scales.device:
            raise ValueError("codes and scales must live on one GPU")
        if not codes.is_contiguous() or not scales.is_contiguous():
            raise ValueError("codes and scales must be contiguous")
        self._codes, self._scales, self._room = codes, scales, None
        self._set(codes.data_ptr(), scales.data_ptr(), 4 * (len(shape) - 1), lines, length, transposed, codes.device)

    def _set(self, codes, scales, bits, lines, length, transposed, device):
        self.bits, self.lines, self.length, self.transposed, self.device = bits, lines, length, transposed, device
        self.use = None   # "fwd" or "bwd": which of a layer's two forms of its weights this is
        self.c = fp4_mx(codes, scales, lines, length, bits)
        self.ref = C.byref(self.c)

    @property
    def codes(self) -> torch.Tensor:
        if self._codes is None:
            half = mx_pitch(self.length) // 2
            self._codes = self._room[:self.bits // 4 * self.lines * half].view((self.lines, half) if self.bits == 4 else (2, self.lines, half))
        return self._codes

    @property
    def scales(self) -> torch.Tensor:
        if self._scales is None:
            per_line = mx_pitch(self.length) // MX_BLOCK
            self._scales = self._room[16 * self.bits // 4 * self.lines * per_line:].view(self.lines, per_line)
        return self._scales

    @property
    def shape(self) -> Tuple[int, int]:
        """Of the matrix that the tensor stands for."""
        return (self.length, self.lines) if self.transposed else (self.lines, self.length)


def mx_empty(lines: int, length: int, bits: int = 4, transposed: bool = False, device="cuda") -> MxTensor:
    """Room for an MX tensor: one allocation, the scales behind the codes."""
    if bits not in (4, 8):
        raise ValueError("an MX element has 4 or 8 bits")
    codes = lines * mx_pitch(length) // 8 * bits
    t = MxTensor.__new__(MxTensor)
    t._codes = t._scales = None
    t._room = room = torch.empty(codes + lines * mx_pitch(length) // MX_BLOCK, dtype=torch.uint8, device=device)
    at = room.data_ptr()
    t._set(at, at + codes, bits, lines, length, transposed, room.device)
    return t


def _ld(t: torch.Tensor, name: str) -> int:
    """Leading dimension of a matrix whose rows may lie apart."""
    if not t.is_cuda:
        raise ValueError("tensors must live on the GPU")
    shape = t.shape
    if len(shape) != 2:
        raise ValueError("%s must be a matrix" % name)
    (rows, cols), (ld, step) = shape, t.stride()
    if step != 1 and cols > 1:
        raise ValueError("%s's rows must be contiguous" % name)
    return ld if rows > 1 and cols > 0 else max(8, -(-cols // 8) * 8)


def _same_device(x, *mx: Optional[MxTensor]):
    device = x.device
    for t in mx:
        if t is not None and t.device != device:
            raise ValueError("all tensors must live on one device")


def _out(t: Optional[torch.Tensor], shape, dtype, device: torch.device, name: str) -> torch.Tensor:
    """The caller's output, checked, or a new one; its rows begin at multiples of 16 bytes."""
    if t is None:
        rows, cols = shape
        if cols % 8 == 0:
            return torch.empty(shape, dtype=dtype, device=device)
        return torch.empty((rows, -(-cols // 8) * 8), dtype=dtype, device=device)[:, :cols]
    if t.shape != shape or t.dtype != dtype or t.device != device:
        raise ValueError("%s must be %s %s on %s" % (name, tuple(shape), dtype, device))
    return t


@functools.lru_cache(maxsize=1024)   # the answer to a query does not change; a server asks for ever new token counts
def _mx_room(op: int, M: int, K: int, N: int) -> int:
    return workspace_bytes(op, M, K, N, FP4_BF16)


def _stream_of(t: torch.Tensor) -> int:
    """Handle of the current stream of t's device, which has to be the current one.  (torch.cuda.current_stream() takes 4 us, as long as a
    small kernel.)"""
    index = t.device.index
    if index != torch._C._cuda_getDevice():
        _current(index)
    return torch._C._cuda_getCurrentRawStream(index)


def _along(t: MxTensor, transposed: bool, name: str):
    if bool(t.transposed) != transposed:
        raise ValueError("%s must %sbe marked transposed: %s" % (name, "" if transposed else "not ", "its lines are columns" if transposed else "its lines are rows"))


def _other_pass(use: str):
    raise ValueError("these weights are laid out for the other pass: this one takes MxWeights.%s" % use)


def _mx_ws(op: int, M: int, K: int, N: int, ws: Optional[Workspace], like: torch.Tensor):
    """(workspace pointer, its bytes, stream handle) of an MX layer call."""
    need = _mx_room(op, M, K, N)
    stream = _stream_of(like)
    buf = _default_workspace(like.device.index, stream)._sized(need) if ws is None else ws.get(need)
    return buf.data_ptr(), buf.numel(), stream


def mx_quantize(x: torch.Tensor, axis: int, bits: int = 4, out: Optional[MxTensor] = None) -> MxTensor:
    """x along its rows (FP4_AXIS_ROW) or along its columns, transposed (FP4_AXIS_COL).  An `out` has bits and an orientation of its own."""
    if axis not in (FP4_AXIS_ROW, FP4_AXIS_COL):
        raise ValueError("MX blocks lie along rows or columns")
    ld = _ld(x, "x")
    rows, cols = x.shape
    lines, length = (rows, cols) if axis == FP4_AXIS_ROW else (cols, rows)
    if out is None:
        out = mx_empty(lines, length, bits, axis == FP4_AXIS_COL, x.device)
    _along(out, axis == FP4_AXIS_COL, "out")
    _same_device(x, out)
    _check(lib().mx_quantize(x.data_ptr(), _dt(x), rows, cols, ld, out.ref if axis == FP4_AXIS_ROW else None,
                             out.ref if axis == FP4_AXIS_COL else None, _stream_of(x)), "mx_quantize")
    return out


def mx_quantize_both(x: torch.Tensor, row_bits: int = 4, col_bits: int = 4) -> Tuple[MxTensor, MxTensor]:
    """x along its rows and along its columns from one read."""
    ld = _ld(x, "x")
    rows, cols = x.shape
    r, c = mx_empty(rows, cols, row_bits, False, x.device), mx_empty(cols, rows, col_bits, True, x.device)
    _check(lib().mx_quantize(x.data_ptr(), _dt(x), rows, cols, ld, r.ref, c.ref, _stream_of(x)), "mx_quantize")
    return r, c


def mx_dequantize(t: MxTensor, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The matrix that t stands for, in the values of its codes."""
    x = _out(out, t.shape, dtype, t.device, "out")
    _check(lib().mx_dequantize(t.ref, int(t.transposed), x.data_ptr(), _dt(x), _ld(x, "out"), _stream_of(x)), "mx_dequantize")
    return x


def _gemm_arguments(l: MxTensor, rt: MxTensor, out_dtype: torch.dtype, addend: Optional[torch.Tensor], out: Optional[torch.Tensor]):
    """(out, its leading dimension, the addend's address) of a product, checked."""
    if l.length != rt.length:
        raise ValueError("operands disagree in the contraction's length")
    if l.device != rt.device:
        raise ValueError("all tensors must live on one device")
    out = _out(out, (l.lines, rt.lines), out.dtype if out is not None else out_dtype, l.device, "out")
    ldo = _ld(out, "out")
    if addend is None:
        return out, ldo, None
    if addend.shape != out.shape or addend.dtype != torch.float32 or addend.device != out.device:
        raise ValueError("addend must be %s float32 on %s" % (tuple(out.shape), out.device))
    if _ld(addend, "addend") != ldo:
        raise ValueError("addend and out must have the same leading dimension")
    return out, ldo, addend.data_ptr()


def mx_gemm(l: MxTensor, rt: MxTensor, out_dtype: torch.dtype = torch.float32, addend: Optional[torch.Tensor] = None,
            out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """l . rt^T over their lines' common length (+ addend)."""
    out, ldo, add = _gemm_arguments(l, rt, out_dtype, addend, out)
    _check(lib().mx_gemm(l.ref, rt.ref, add, out.data_ptr(), _dt(out), ldo, _stream_of(out)), "mx_gemm")
    return out


def mx_gemm_by_tile(l: MxTensor, rt: MxTensor, tile: int, out_dtype: torch.dtype = torch.float32, addend: Optional[torch.Tensor] = None) -> torch.Tensor:
    """mx_gemm by one kind of tile (16, 32, 64, 128, 192, 256), for tests and measuring; addend has the output's leading dimension."""
    out, ldo, add = _gemm_arguments(l, rt, out_dtype, addend, None)
    _check(lib().mx_gemm_by_tile(l.ref, rt.ref, add, out.data_ptr(), _dt(out), ldo, tile, _stream_of(out)), "mx_gemm_by_tile")
    return out


def mx_gemm_tile(P: int, Q: int, Kc: int, bits_l: int = 4, bits_r: int = 4, compute_units: int = 256) -> Tuple[int, int]:
    """The tile that mx_gemm takes, and how many tiles of a last round are cut smaller (host arithmetic, no GPU)."""
    last_round = C.c_int(0)
    tile = lib().mx_gemm_tile(P, Q, Kc, bits_l, bits_r, compute_units, C.byref(last_round))
    if tile < 0:
        _check(tile, "mx_gemm_tile")
    return tile, last_round.value


def mx_checkpoint(M: int, K: int, bits: int = 8, device="cuda") -> MxTensor:
    """Room for the checkpoint of activations [M, K]: what mx_linear_fwd leaves for the weight gradient."""
    return mx_empty(K, M, bits, True, device)


def mx_checkpoint_save(x: torch.Tensor, bits: int = 8) -> MxTensor:
    """The checkpoint by itself; mx_linear_fwd writes the same from the read that it makes anyway."""
    return mx_quantize(x, FP4_AXIS_COL, bits)


class MxWeights:
    """Both orientations of a layer's weights W [K, N]: fwd (lines N, length K) for the forward pass, bwd (lines K, length N) for the
    activation gradient.  Made once per weight version.  Those of mx_prepare_weights are refused by the other's pass, also where W is
    square and their sizes agree."""

    def __init__(self, fwd: MxTensor, bwd: MxTensor):
        self.fwd, self.bwd = fwd, bwd


def mx_prepare_weights(W: torch.Tensor) -> MxWeights:
    bwd, fwd = mx_quantize_both(W)
    fwd.use, bwd.use = "fwd", "bwd"
    return MxWeights(fwd, bwd)


def mx_linear_fwd(A: torch.Tensor, W: MxTensor, act_bits: int = 4, saved: Optional[MxTensor] = None,
                  Y: Optional[torch.Tensor] = None, ws: Optional[Workspace] = None) -> torch.Tensor:
    """Y = Q(A) W; saved: an mx_checkpoint that the pass fills for the weight gradient."""
    lda = _ld(A, "A")
    M, K = A.shape
    N = W.lines
    if W.length != K:
        raise ValueError("A [M,K] and W (lines N, length K) must agree in K")
    if W.use == "bwd":
        _other_pass("fwd")
    if saved is not None:
        if (saved.lines, saved.length) != (K, M):
            raise ValueError("the checkpoint holds %d x %d activations, not %d x %d" % (saved.length, saved.lines, M, K))
        _along(saved, True, "the checkpoint")
    _same_device(A, W, saved)
    Y = _out(Y, (M, N), A.dtype, A.device, "Y")
    room, nbytes, stream = _mx_ws(FP4_OP_MX_FWD, M, K, N, ws, A)
    _check(lib().mx_linear_fwd(A.data_ptr(), _dt(A), M, K, N, lda, act_bits, W.ref, Y.data_ptr(), _ld(Y, "Y"), None if saved is None else saved.ref,
                               room, nbytes, stream), "mx_linear_fwd")
    return Y


def mx_linear_bwd_dgrad(dY: torch.Tensor, W: MxTensor, dA: Optional[torch.Tensor] = None, ws: Optional[Workspace] = None) -> torch.Tensor:
    """dA = Q(dY) W^T, W along its rows (lines K, length N)."""
    ldy = _ld(dY, "dY")
    M, N = dY.shape
    K = W.lines
    if W.length != N:
        raise ValueError("dY [M,N] and W (lines K, length N) must agree in N")
    if W.use == "fwd":
        _other_pass("bwd")
    _same_device(dY, W)
    dA = _out(dA, (M, K), dY.dtype, dY.device, "dA")
    room, nbytes, stream = _mx_ws(FP4_OP_MX_DGRAD, M, K, N, ws, dY)
    _check(lib().mx_linear_bwd_dgrad(dY.data_ptr(), _dt(dY), M, K, N, ldy, W.ref, dA.data_ptr(), _ld(dA, "dA"), room, nbytes, stream),
           "mx_linear_bwd_dgrad")
    return dA


def mx_linear_bwd_wgrad(dY: torch.Tensor, saved: MxTensor, grad_bits: int = 4, dW: Optional[torch.Tensor] = None,
                        accumulate: bool = False, ws: Optional[Workspace] = None) -> torch.Tensor:
    """dW (+)= saved . Q(dY), contracting over the tokens."""
    ldy = _ld(dY, "dY")
    M, N = dY.shape
    K = saved.lines
    if saved.length != M:
        raise ValueError("dY [M,N] and the checkpoint must agree in M")
    _along(saved, True, "the checkpoint")
    if accumulate and dW is None:
        raise ValueError("accumulate needs the dW to add to")
    _same_device(dY, saved)
    dW = _out(dW, (K, N), torch.float32, dY.device, "dW")
    room, nbytes, stream = _mx_ws(FP4_OP_MX_WGRAD, M, K, N, ws, dY)
    _check(lib().mx_linear_bwd_wgrad(dY.data_ptr(), _dt(dY), M, K, N, ldy, saved.ref, grad_bits, int(accumulate), dW.data_ptr(), _ld(dW, "dW"), room,
                                     nbytes, stream), "mx_linear_bwd_wgrad")
    return dW


def mx_linear_bwd(dY: torch.Tensor, saved: MxTensor, W: MxTensor, grad_bits: int = 4, dA: Optional[torch.Tensor] = None,
                  dW: Optional[torch.Tensor] = None, accumulate: bool = False, ws: Optional[Workspace] = None):
    """Both gradients, dY read once.  Returns (dA, dW)."""
    ldy = _ld(dY, "dY")
    M, N = dY.shape
    K = W.lines
    if W.length != N or (saved.lines, saved.length) != (K, M):
        raise ValueError("dY [M,N], W (lines K, length N) and the checkpoint must agree")
    if W.use == "fwd":
        _other_pass("bwd")
    _along(saved, True, "the checkpoint")
    if accumulate and dW is None:
        raise ValueError("accumulate needs the dW to add to")
    _same_device(dY, W, saved)
    dA = _out(dA, (M, K), dY.dtype, dY.device, "dA")
    dW = _out(dW, (K, N), torch.float32, dY.device, "dW")
    room, nbytes, stream = _mx_ws(FP4_OP_MX_BWD, M, K, N, ws, dY)
    _check(lib().mx_linear_bwd(dY.data_ptr(), _dt(dY), M, K, N, ldy, W.ref, saved.ref, grad_bits, dA.data_ptr(), _ld(dA, "dA"), int(accumulate),
                               dW.data_ptr(), _ld(dW, "dW"), room, nbytes, stream), "mx_linear_bwd")
    return dA, dW


def _hp_vector(t: Optional[torch.Tensor], n: int, dtype: torch.dtype, device: torch.device, name: str):
    """Address of a vector of so many elements, or None."""
    if t is None:
        return None
    if t.shape != (n,) or t.dtype is not dtype or t.device != device or not (n < 2 or t.stride(0) == 1):
        raise ValueError("%s must be [%d] contiguous %s on %s" % (name, n, dtype, device))
    return t.data_ptr()


def _hp_matrix(t: Optional[torch.Tensor], shape, dtype: torch.dtype, device: torch.device, name: str):
    """(address, leading dimension) of a matrix, or nothing."""
    if t is None:
        return None, 0
    if t.shape != shape or t.dtype is not dtype or t.device != device:
        raise ValueError("%s must be %s %s on %s" % (name, tuple(shape), dtype, device))
    return t.data_ptr(), _ld(t, name)


def _hp_out(t: Optional[torch.Tensor], like: Optional[torch.Tensor], shape, dtype: torch.dtype, device: torch.device, name: str):
    """(the caller's output, checked, or a new one; its address; its leading dimension)."""
    if t is not None:
        return (t, *_hp_matrix(t, shape, dtype, device, name))
    cols = shape[1]
    ld = -(-cols // 8) * 8 or 8
    if ld == cols and like is not None and like.is_contiguous():
        t = torch.empty_like(like)   # half a microsecond less than by shape and type, of the ten that a short call takes
    else:
        t = torch.empty_strided(shape, (ld, 1), dtype=dtype, device=device)
    return t, t.data_ptr(), ld


class HpNorm:
    """The joint of two blocks: what hp_norm_fwd and hp_norm_bwd take besides the tokens.

    w_before [D]: weights of the norm before the next block (None: there is none); w_after [D]: of the norm after the block; gate: [D], one
    for all tokens, or [M, D], a row for each (a vector that was expanded to that is refused); scale: of the residual stream."""

    __slots__ = ("w_before", "w_after", "gate", "scale", "eps")

    def __init__(self, w_before: Optional[torch.Tensor] = None, w_after: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                 scale: float = 1.0, eps: float = 1e-5):
        if not eps > 0:
            raise ValueError("eps must be positive")
        if gate is not None and gate.dim() not in (1, 2):
            raise ValueError("a gate is [D] or [M, D]")
        self.w_before, self.w_after, self.gate, self.scale, self.eps = w_before, w_after, gate, float(scale), float(eps)

    def _arguments(self, shape, dtype: torch.dtype, device: torch.device):
        """The structure for tokens of that kind, checked."""
        D = shape[1]
        gate, ld_gate = self.gate, 0
        if gate is not None:
            if gate.dim() == 1:
                gate = _hp_vector(gate, D, dtype, device, "gate")
            else:
                gate, ld_gate = _hp_matrix(gate, shape, dtype, device, "gate")
                if ld_gate < D:   # 0 would be read as one vector, whose gradient is [D]
                    raise ValueError("a gate's rows overlap: one vector for all tokens is given as [D], not expanded")
        return C.byref(hp_norm(_hp_vector(self.w_before, D, dtype, device, "w_before"), _hp_vector(self.w_after, D, dtype, device, "w_after"), gate, ld_gate,
                               self.scale, self.eps))


class HpNormSaved:
    """What the forward pass of a joint leaves for its backward pass: each token's inverse norms (fp32 [M])."""

    __slots__ = ("r_before", "r_after")

    def __init__(self, r_before: Optional[torch.Tensor], r_after: Optional[torch.Tensor] = None):
        self.r_before, self.r_after = r_before, r_after


def hp_norm_saved(norm: HpNorm, M: int, device="cuda") -> HpNormSaved:
    """Room for them."""
    return HpNormSaved(*(None if w is None else torch.empty(M, dtype=torch.float32, device=device) for w in (norm.w_before, norm.w_after)))


def hp_norm_fwd(norm: HpNorm, x: torch.Tensor, block: Optional[torch.Tensor] = None, saved: Optional[HpNormSaved] = None,
                h: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None):
    """(h, y): the residual stream scale x + gate norm(block), and it normed for the next block (None without w_before).  saved: filled for the
    backward pass.  h or y may be x or block."""
    ldx = _ld(x, "x")
    dt, stream = _dt(x), _stream_of(x)
    shape, dtype, device = like = x.shape, x.dtype, x.device
    M, D = shape
    pb, ldb = _hp_matrix(block, *like, "block")
    if block is None and (norm.w_after is not None or norm.gate is not None):
        raise ValueError("a norm after a block or a gate needs the block")
    ref = norm._arguments(*like)
    h, ph, ldh = _hp_out(h, x, *like, "h")
    py, ldy = None, 0
    if norm.w_before is not None:
        y, py, ldy = _hp_out(y, x, *like, "y")
    elif y is not None:
        raise ValueError("y needs w_before")
    rb = ra = None
    if saved is not None:
        rb = _hp_vector(saved.r_before, M, torch.float32, device, "r_before") if norm.w_before is not None else None
        ra = _hp_vector(saved.r_after, M, torch.float32, device, "r_after") if norm.w_after is not None else None
    _check(lib().hp_norm_fwd(ref, dt, M, D, x.data_ptr(), ldx, pb, ldb, ph, ldh, py, ldy, rb, ra, stream), "hp_norm_fwd")
    return h, y


class HpNormGrads(NamedTuple):
    """dx, dblock [M, D]; dgate: fp32 [D], or [M, D] of the tokens' type; dw_before, dw_after: fp32 [D]; None where the joint has none."""
    dx: torch.Tensor
    dblock: Optional[torch.Tensor]
    dgate: Optional[torch.Tensor]
    dw_before: Optional[torch.Tensor]
    dw_after: Optional[torch.Tensor]


def hp_norm_bwd(norm: HpNorm, saved: HpNormSaved, h: torch.Tensor, dy: Optional[torch.Tensor] = None, dh: Optional[torch.Tensor] = None,
                block: Optional[torch.Tensor] = None, into: Optional[HpNormGrads] = None, accumulate: bool = False,
                ws: Optional[Workspace] = None) -> HpNormGrads:
    """Gradients of a joint from those of y and of h (either may be None).  into: tensors to write them to; accumulate adds to its sums over
    tokens (dw_before, dw_after, dgate [D])."""
    if dy is None and dh is None:
        raise ValueError("a gradient of y or of h is needed")
    if dy is not None and norm.w_before is None:
        raise ValueError("a gradient of y needs w_before")
    if block is None and (norm.w_after is not None or norm.gate is not None):
        raise ValueError("a norm after a block or a gate needs the block")
    if accumulate and into is None:
        raise ValueError("accumulate needs the gradients to add to")
    ldh = _ld(h, "h")
    dt, stream = _dt(h), _stream_of(h)
    like = h.shape, h.dtype, h.device
    M, D = h.shape
    pdy, ld_dy = _hp_matrix(dy, *like, "dy")
    pdh, ld_dh = _hp_matrix(dh, *like, "dh")
    pb, ldb = _hp_matrix(block, *like, "block")
    ref = norm._arguments(*like)
    rb = _hp_vector(saved.r_before, M, torch.float32, h.device, "r_before") if dy is not None else None
    ra = _hp_vector(saved.r_after, M, torch.float32, h.device, "r_after") if norm.w_after is not None else None
    if (dy is not None and rb is None) or (norm.w_after is not None and ra is None):
        raise ValueError("the saved inverse norms are missing")
    given = into if into is not None else HpNormGrads(None, None, None, None, None)

    def sums(t, name):
        if t is None:
            if accumulate:
                raise ValueError("accumulate needs the %s to add to" % name)
            t = torch.empty(D, dtype=torch.float32, device=h.device)
        return t, _hp_vector(t, D, torch.float32, h.device, name)

    dblock = dgate = dw_before = dw_after = pdblock = pdgate = pwb = pwa = None
    ld_dblock = ld_dgate = 0
    dx, pdx, ld_dx = _hp_out(given.dx, h, *like, "dx")
    if block is not None:
        dblock, pdblock, ld_dblock = _hp_out(given.dblock, h, *like, "dblock")
    if norm.gate is not None:
        if norm.gate.dim() == 1:
            dgate, pdgate = sums(given.dgate, "dgate")
        else:
            dgate, pdgate, ld_dgate = _hp_out(given.dgate, h, *like, "dgate")
    if dy is not None:
        dw_before, pwb = sums(given.dw_before, "dw_before")
    if norm.w_after is not None:
        dw_after, pwa = sums(given.dw_after, "dw_after")
    need = _mx_room(FP4_OP_HP_NORM_BWD, M, D, 0)
    room = _default_workspace(h.device.index, stream)._sized(need) if ws is None else ws.get(need)
    _check(lib().hp_norm_bwd(ref, dt, M, D, pdy, ld_dy, pdh, ld_dh, h.data_ptr(), ldh, pb, ldb, rb, ra, pdx, ld_dx, pdblock, ld_dblock, pdgate, ld_dgate, pwb, pwa,
                             int(accumulate), room.data_ptr(), room.numel(), stream), "hp_norm_bwd")
    return HpNormGrads(dx, dblock, dgate, dw_before, dw_after)


def _hp_ids(ids: torch.Tensor, device: torch.device, name: str) -> int:
    if ids.dim() != 1 or ids.dtype is not torch.int64 or ids.device != device or not (ids.stride(0) == 1 or ids.shape[0] < 2):
        raise ValueError("%s must be [M] contiguous int64 on %s" % (name, device))
    return ids.data_ptr()


def hp_embed_fwd(ids: torch.Tensor, table: torch.Tensor, scale: float = 1.0, y: Optional[torch.Tensor] = None) -> torch.Tensor:
    """scale table[ids], table [V, D]; zeros for ids outside [0, V)."""
    ldt, dt, stream, device = _ld(table, "table"), _dt(table), _stream_of(table), table.device
    at = _hp_ids(ids, device, "ids")
    M, (V, D) = ids.shape[0], table.shape
    y, py, ldy = _hp_out(y, None, (M, D), table.dtype, device, "y")
    _check(lib().hp_embed_fwd(at, dt, M, D, V, table.data_ptr(), ldt, scale, py, ldy, stream), "hp_embed_fwd")
    return y


def hp_embed_bwd(dy: torch.Tensor, ids: torch.Tensor, V: int, scale: float = 1.0, dtable: Optional[torch.Tensor] = None, accumulate: bool = False,
                 ws: Optional[Workspace] = None) -> torch.Tensor:
    """The table's gradient [V, D] in fp32: scale times the sums of dy's rows by id.  accumulate adds them to dtable and leaves the other rows alone."""
    ld, dt, stream = _ld(dy, "dy"), _dt(dy), _stream_of(dy)
    at = _hp_ids(ids, dy.device, "ids")
    M, D = dy.shape
    if ids.shape[0] != M:
        raise ValueError("dy [M,D] and ids [M] must agree in M")
    if accumulate and dtable is None:
        raise ValueError("accumulate needs the dtable to add to")
    dtable, pt, ld_table = _hp_out(dtable, None, (V, D), torch.float32, dy.device, "dtable")
    need = _mx_room(FP4_OP_HP_EMBED_BWD, M, D, V)
    room = _default_workspace(dy.device.index, stream)._sized(need) if ws is None else ws.get(need)
    _check(lib().hp_embed_bwd(at, dt, M, D, V, dy.data_ptr(), ld, scale, int(accumulate), pt, ld_table, room.data_ptr(), room.numel(), stream),
           "hp_embed_bwd")
    return dtable


def _head_arguments(x: torch.Tensor, w: torch.Tensor, targets: torch.Tensor):
    ldx, ldw, stream = _ld(x, "x"), _ld(w, "w"), _stream_of(x)
    if x.dtype != torch.bfloat16 or w.dtype != torch.bfloat16:
        raise TypeError("the head takes bfloat16, got %s and %s" % (x.dtype, w.dtype))
    if w.device != x.device:
        raise ValueError("all tensors must live on one device")
    M, D = x.shape
    if w.shape[1] != D or targets.shape != (M,):
        raise ValueError("x [M,D], w [V,D] and targets [M] must agree")
    return ldx, ldw, stream, _hp_ids(targets, x.device, "targets")


def hp_head_fwd(x: torch.Tensor, w: torch.Tensor, targets: torch.Tensor, loss: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                ws: Optional[Workspace] = None):
    """(loss, lse), fp32 [M]: softmax cross entropy of logits x w^T, which are not kept, and the logarithm of their sum of exponentials.  Targets
    outside [0, V) have a loss of 0."""
    ldx, ldw, stream, at = _head_arguments(x, w, targets)
    M, D = x.shape
    V = w.shape[0]
    loss = torch.empty(M, dtype=torch.float32, device=x.device) if loss is None else loss
    lse = torch.empty(M, dtype=torch.float32, device=x.device) if lse is None else lse
    to = (_hp_vector(loss, M, torch.float32, x.device, "loss"), _hp_vector(lse, M, torch.float32, x.device, "lse"))
    need = _mx_room(FP4_OP_HP_HEAD_FWD, M, D, V)
    room = _default_workspace(x.device.index, stream)._sized(need) if ws is None else ws.get(need)
    _check(lib().hp_head_fwd(x.data_ptr(), w.data_ptr(), at, FP4_BF16, M, D, V, ldx, ldw, *to, room.data_ptr(), room.numel(), stream), "hp_head_fwd")
    return loss, lse


def hp_head_bwd(x: torch.Tensor, w: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor, dloss: torch.Tensor, dx: Optional[torch.Tensor] = None,
                dw: Optional[torch.Tensor] = None, dw_dtype: torch.dtype = torch.float32, accumulate: bool = False, want_dx: bool = True,
                want_dw: bool = True, ws: Optional[Workspace] = None):
    """(dx, dw) from each loss's gradient dloss [M]; dw [V, D] in fp32 or bfloat16.  accumulate adds to an fp32 dw (that of a tied embedding, or
    several micro-batches).  A head or an input that is not trained: want_dw or want_dx False, and None comes back."""
    ldx, ldw, stream, at = _head_arguments(x, w, targets)
    M, D = x.shape
    V = w.shape[0]
    if not want_dx and not want_dw:
        raise ValueError("one of the gradients has to be wanted")
    if accumulate and want_dw and (dw is None or dw.dtype != torch.float32):
        raise ValueError("accumulate needs the fp32 dw to add to")
    pdx = pdw = None
    ld_dx = ld_dw = 0
    if want_dx:
        dx, pdx, ld_dx = _hp_out(dx, x, x.shape, torch.bfloat16, x.device, "dx")
    if want_dw:
        dw, pdw, ld_dw = _hp_out(dw, None, w.shape, dw.dtype if dw is not None else dw_dtype, x.device, "dw")
    given = (_hp_vector(lse, M, torch.float32, x.device, "lse"), _hp_vector(dloss, M, torch.float32, x.device, "dloss"))
    need = _mx_room(FP4_OP_HP_HEAD_BWD, M, D, V)
    room = _default_workspace(x.device.index, stream)._sized(need) if ws is None else ws.get(need)
    _check(lib().hp_head_bwd(x.data_ptr(), w.data_ptr(), at, *given, FP4_BF16, M, D, V, ldx, ldw, pdx, ld_dx, pdw, _dt(dw) if want_dw else FP4_BF16, ld_dw,
                             int(accumulate and want_dw), room.data_ptr(), room.numel(), stream), "hp_head_bwd")
    return dx if want_dx else None, dw if want_dw else None


def fp4_unpack(codes: torch.Tensor) -> torch.Tensor:
    _dev_check(codes)
    rows, half = codes.shape
    out = torch.empty((rows, 2 * half), dtype=torch.uint8, device=codes.device)
    _check(lib().fp4_unpack(_ptr(codes), rows, 2 * half, _ptr(out), _stream()), "fp4_unpack")
    return out


def fp4_dge_apply(G: torch.Tensor, W: torch.Tensor, gamma_W: torch.Tensor, dge_k: float = 5.0,
                  dge_cap: float = 3.0, dW: Optional[torch.Tensor] = None) -> torch.Tensor:
    _dev_check(G, W, gamma_W, dW)
    K, N = W.shape
    if dW is None:
        dW = torch.empty_like(G)
    _check(lib().fp4_dge_apply(_ptr(G), _ptr(W), _dt(W), _ptr(gamma_W), K, N, float(dge_k), float(dge_cap),
                               _ptr(dW), _stream()), "fp4_dge_apply")
    return dW


def fp4_residual_spmm(row_ptr: torch.Tensor, col_idx: torch.Tensor, val: torch.Tensor, Q: int,
                      D: torch.Tensor, R: Optional[torch.Tensor] = None, ws: Optional[Workspace] = None) -> torch.Tensor:
    return _residual_spmm("fp4_residual_spmm_bounded", (col_idx.numel(),), row_ptr, col_idx, val, Q, D, R, ws)


def fp4_residual_spmm_general(row_ptr: torch.Tensor, col_idx: torch.Tensor, val: torch.Tensor, Q: int,
                              D: torch.Tensor, R: Optional[torch.Tensor] = None, ws: Optional[Workspace] = None) -> torch.Tensor:
    return _residual_spmm("fp4_residual_spmm_general", (), row_ptr, col_idx, val, Q, D, R, ws)


def fp4_residual_spmm_gathers(P: int, Q: int, N: int, dt: int, entries: int) -> bool:
    """Whether a residual product is the gathering kernel's (host arithmetic, no GPU)."""
    return bool(lib().fp4_residual_spmm_gathers(P, Q, N, dt, entries))


def _residual_spmm(name, capacity, row_ptr, col_idx, val, Q, D, R, ws):
    _dev_check(row_ptr, col_idx, val, D, R)
    P = row_ptr.numel() - 1
    N = D.shape[1]
    if R is None:
        R = torch.empty((P, N), dtype=torch.float32, device=D.device)
    w = _ws(workspace_bytes(FP4_OP_SPMM, P, Q, N, _dt(D)), ws)
    _check(getattr(lib(), name)(_ptr(row_ptr), _ptr(col_idx), _ptr(val), *capacity, P, Q, _ptr(D), _dt(D), N,
                                _ptr(R), _ptr(w), w.numel(), _stream()), name)
    return R


def fp4_quantize_cols_folds(rows: int, cols: int) -> bool:
    """Whether the tiles of a tensor's column-wise quantization form their scales themselves (host arithmetic, no GPU)."""
    return bool(lib().fp4_quantize_cols_folds(rows, cols))


FP4_SELECT_WINDOWS, FP4_SELECT_SAMPLE, FP4_SELECT_FOUND, FP4_SELECT_APART = 1, 2, 4, 8


def fp4_select_route(rows: int, cols: int, dt: int, ld: Optional[int] = None) -> int:
    """Which passes find a tensor's thresholds (host arithmetic, no GPU)."""
    return int(lib().fp4_select_route(rows, cols, cols if ld is None else ld, dt))


def fp4_select_beside(M: int, K: int, N: int, dt: int, compute_units: int = 256) -> int:
    """Tiles a workgroup of W's column-wise codes beside the first digit pass over A, or 0 (host arithmetic, no GPU)."""
    return int(lib().fp4_select_beside(M, K, N, dt, compute_units))


def fp4_transpose_beside(M: int, K: int, N: int, compute_units: int = 256) -> int:
    """Tiles a workgroup of a weight gradient's codes beside the transposition's last pass, or 0 (host arithmetic, no GPU)."""
    return int(lib().fp4_transpose_beside(M, K, N, compute_units))


def fp4_count_beside(M: int, K: int, N: int, dt: int, capacity: int, cached: bool = False, compute_units: int = 256) -> bool:
    """Whether the transposition's first pass goes with the launch that begins a backward pass (host arithmetic, no GPU)."""
    return lib().fp4_count_beside(M, K, N, dt, int(cached), capacity, compute_units) == 1


def fp4_residual_transpose_positions(P: int, Q: int) -> int:
    """Where the places of a transposed residual's entries come from (host arithmetic, no GPU)."""
    return int(lib().fp4_residual_transpose_positions(P, Q))


def fp4_residual_transpose(row_ptr: torch.Tensor, col_idx: torch.Tensor, val: torch.Tensor, nnz: torch.Tensor, Q: int,
                           positions: int = 0, ws: Optional[Workspace] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """CSR of the transpose as a weight gradient takes it; col_idx and val have room for what row_ptr counts."""
    _dev_check(row_ptr, col_idx, val, nnz)
    P = row_ptr.numel() - 1
    t_ptr = torch.empty(Q + 1, dtype=torch.int64, device=val.device)
    t_idx, t_val = torch.empty_like(col_idx), torch.empty_like(val)
    w = _ws(workspace_bytes(FP4_OP_WGRAD, P, Q, 32, FP4_F32), ws)
    _check(lib().fp4_residual_transpose(_ptr(row_ptr), _ptr(col_idx), _ptr(val), _ptr(nnz), P, Q, col_idx.numel(), positions, _ptr(t_ptr),
                                        _ptr(t_idx), _ptr(t_val), _ptr(w), w.numel(), _stream()), "fp4_residual_transpose")
    return t_ptr, t_idx, t_val


def fp4_host_round_codes(x_host):
    """numpy fp32 array (host) -> uint8 codes, through the library's own rounding routine."""
    import numpy as np
    x = np.ascontiguousarray(x_host, dtype=np.float32)
    out = np.empty(x.shape, dtype=np.uint8)
    _check(lib().fp4_host_round_codes(x.ctypes.data_as(C.c_void_p), x.size, out.ctypes.data_as(C.c_void_p)),
           "fp4_host_round_codes")
    return out


def fp4_device_round_codes(x):
    """fp32 CUDA tensor (numel a multiple of 8) -> uint8 codes, through the quantization kernels' packing routine."""
    import torch
    assert x.dtype == torch.float32
    _dev_check(x)
    out = torch.empty(x.shape, dtype=torch.uint8, device=x.device)
    _check(lib().fp4_device_round_codes(x.data_ptr(), x.numel(), out.data_ptr(), _stream()), "fp4_device_round_codes")
    return out


def fp4_device_round_sweep(device="cuda:0") -> int:
    """Number of fp32 bit patterns (times eight word positions) where the device's packing routine and its
    comparison-chain routine disagree; 0 is the only acceptable result."""
    import torch
    cnt = torch.zeros(1, dtype=torch.int64, device=device)
    _dev_check(cnt)
    _check(lib().fp4_device_round_sweep(cnt.data_ptr(), _stream()), "fp4_device_round_sweep")
    return int(cnt.item())


FP4_TRACE_GEMM, FP4_TRACE_SPMM = 0, 1


def fp4_gemm_tiling(P: int, Q: int, Kc: int, factor: bool = False, w_bf16: bool = False, addend: bool = False,
                    out_bf16: bool = False, compute_units: int = 256) -> Tuple[int, int, int]:
    """Tile size of the FP4 GEMM, how many tiles of a last round are cut smaller, and the delay between quarters of the
    workgroups (host arithmetic, no GPU)."""
    last_round, stagger = C.c_int(0), C.c_int(0)
    tile = lib().fp4_gemm_tiling(P, Q, Kc, int(factor), int(w_bf16), int(addend), int(out_bf16), compute_units,
                                 C.byref(last_round), C.byref(stagger))
    if tile < 0:
        _check(tile, "fp4_gemm_tiling")
    return tile, last_round.value, stagger.value


def fp4_gemm_splits(P: int, Q: int, Kc: int, factor: bool = False, compute_units: int = 256) -> bool:
    """Whether fp4_gemm_tiling's tiles are 32 x 32, whatever the types (host arithmetic, no GPU)."""
    return lib().fp4_gemm_splits(P, Q, Kc, int(factor), compute_units) == 1


def fp4_trace_begin(max_launches: int) -> None:
    _check(lib().fp4_trace_begin(int(max_launches)), "fp4_trace_begin")


def fp4_trace_end(max_launches: int):
    """[(kind, ms)] of the GEMM / tiled sparse-product launches recorded since fp4_trace_begin, in order."""
    buf = (C.c_float * max_launches)()
    kinds = (C.c_int * max_launches)()
    n = lib().fp4_trace_end(C.cast(buf, C.c_void_p), C.cast(kinds, C.c_void_p), max_launches)
    if n < 0:
        raise Fp4Error(n, "fp4_trace_end")
    return [(int(kinds[i]), float(buf[i])) for i in range(min(n, max_launches))]


def fp4_probe_mfma(operand_bytes: torch.Tensor, workgroups: int, iters: int, sink: torch.Tensor) -> None:
    _dev_check(operand_bytes, sink)
    _check(lib().fp4_probe_mfma(_ptr(operand_bytes), operand_bytes.numel() * operand_bytes.element_size(),
                                int(workgroups), int(iters), _ptr(sink), _stream()), "fp4_probe_mfma")


def fp4_probe_copy(src: torch.Tensor, dst: torch.Tensor) -> None:
    _dev_check(src, dst)
    _check(lib().fp4_probe_copy(_ptr(src), _ptr(dst), src.numel() * src.element_size(), _stream()),
           "fp4_probe_copy")
