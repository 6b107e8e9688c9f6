"""ctypes binding of liboptima.so: argument marshalling only.

Every function has the name of the C entry point it wraps, takes torch tensors
(device memory) and passes their data pointers and the current HIP stream
through. No computation of the method happens here. The library must exist:
importing this module without it raises, there is no fallback path.
"""
from __future__ import annotations

import ctypes
import functools
import os
from dataclasses import dataclass, fields

import torch

# OPTIMA_LIBRARY names another build of the same library (the host-sanitized
# build that the ABI tests run against); by default the in-tree library.
_LIB_PATH = os.environ.get("OPTIMA_LIBRARY") or os.path.join(
    os.path.dirname(os.path.abspath(__file__)), "liboptima.so")

OPTIMA_OK = 0
OPTIMA_E_INVAL = -1
OPTIMA_E_HIP = -2
OPTIMA_E_NONFINITE = -3
OPTIMA_E_WORKSPACE = -4
OPTIMA_E_UNSUPPORTED = -5
DTYPE_F32 = 0
DTYPE_BF16 = 1
DTYPE_F64 = 2
DTYPE_I8 = 3
DTYPE_MX4 = 4
METHOD_RAPDHG = 0
METHOD_CG = 1
PREC_FP32 = 0
PREC_BF16X3 = 1


class OptimaError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{message} (status {status})")
        self.status = status


if not os.path.exists(_LIB_PATH):
    raise ImportError(
        f"{_LIB_PATH} is missing: build it with `python paper_2512_13886_amd/build.py`")
_lib = ctypes.CDLL(_LIB_PATH)

_i64, _i32, _sz, _vp, _f32 = ctypes.c_int64, ctypes.c_int, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_float


class _Opts(ctypes.Structure):
    _fields_ = [("max_iters", ctypes.c_int64), ("check_every", ctypes.c_int32),
                ("fixed_iters", ctypes.c_int32), ("eps_rel", ctypes.c_float),
                ("eps_abs", ctypes.c_float), ("beta_sufficient", ctypes.c_float),
                ("beta_necessary", ctypes.c_float), ("beta_artificial", ctypes.c_float),
                ("step_safety", ctypes.c_float), ("restarts", ctypes.c_int32),
                ("precision", ctypes.c_int32), ("method", ctypes.c_int32),
                ("col_scale", ctypes.c_void_p), ("sparse", ctypes.c_int32),
                ("cooperative", ctypes.c_int32)]


class _Stats(ctypes.Structure):
    _fields_ = [("iters", _vp), ("restarts", _vp), ("converged", _vp),
                ("f_initial", _vp), ("f_final", _vp), ("kkt_final", _vp)]


class _Info(ctypes.Structure):
    _fields_ = [("iterations", ctypes.c_int64), ("gemm_calls", ctypes.c_int64),
                ("row_products", ctypes.c_int64), ("checks", ctypes.c_int64),
                ("timed_launches", ctypes.c_int64), ("timed_row_products", ctypes.c_int64),
                ("timed_product_ms", ctypes.c_double), ("sparse_products", ctypes.c_int64),
                ("few_launches", ctypes.c_int64), ("few_row_products", ctypes.c_int64),
                ("few_product_ms", ctypes.c_double), ("persistent_launches", ctypes.c_int64)]


def _sig(name, res, args):
    f = getattr(_lib, name)
    f.restype = res
    f.argtypes = args
    return f


_status_string = _sig("optima_status_string", ctypes.c_char_p, [_i32])
_abi_version = _sig("optima_abi_version", _i32, [])
# The structs above mirror include/optima.h at this ABI version.
ABI_VERSION = 13
if _abi_version() != ABI_VERSION:
    raise ImportError(f"{_LIB_PATH} has ABI version {_abi_version()}, the binding expects "
                      f"{ABI_VERSION}: rebuild the library")
_hess_ws = _sig("optima_hessian_workspace_bytes", _sz, [_i64, _i64, _i32])
_hess_acc = _sig("optima_hessian_accumulate", _i32,
                 [_vp, _i32, _i64, _i64, _vp, _i32, _vp, _sz, _vp])
_damp = _sig("optima_hessian_damp", _i32, [_vp, _i64, _f32, _vp, _vp])
_jacobi = _sig("optima_hessian_jacobi", _i32, [_vp, _i64, _vp, _vp])
_spec_ws = _sig("optima_spectral_norm_workspace_bytes", _sz, [_i64, _i32])
_spec = _sig("optima_spectral_norm", _i32,
             [_vp, _i64, _vp, _i32, _i32, _f32, _vp, _sz, _vp, _vp, _vp])
_spec_na = _sig("optima_spectral_norm_noalloc", _i32,
                [_vp, _i64, _vp, _i32, _i32, _f32, _vp, _vp, _vp])
_lz_ws = _sig("optima_spectral_lanczos_workspace_bytes", _sz, [_i64, _i32])
_lz = _sig("optima_spectral_lanczos", _i32,
           [_vp, _i64, _vp, _i32, _f32, _vp, _sz, _vp, _vp, _vp])
_mask = _sig("optima_wanda_mask", _i32,
             [_vp, _i64, _i64, _vp, _i32, _i64, _i32, ctypes.c_double, _vp, _vp])
_fwd_ws = _sig("optima_linear_forward_workspace_bytes", _sz, [_i64, _i64, _i64])
_fwd = _sig("optima_linear_forward", _i32,
            [_vp, _i64, _i64, _vp, _i64, _i32, _vp, _i32, _vp, _vp, _vp, _sz, _vp])
_opts_default = _sig("optima_solver_opts_default", None, [ctypes.POINTER(_Opts)])
_qp_ws = _sig("optima_qp_workspace_bytes", _sz, [_i64, _i64])
_qp_solve = _sig("optima_qp_solve_batched", _i32,
                 [_vp, _i64, _vp, _vp, _vp, _i64, ctypes.POINTER(_Opts), _vp, _sz, _vp,
                  ctypes.POINTER(_Stats), ctypes.POINTER(_Info), _vp])
_norm = _sig("optima_rms_norm", _i32,
             [_vp, _i64, _vp, _i64, _i32, _i64, _i64, _vp, _i32, _f32, _vp, _i64, _vp, _i64, _i32,
              _vp, _i64, _vp])
_norm_bwd_ws = _sig("optima_rms_norm_backward_workspace_bytes", _sz, [_i64, _i64])
_norm_bwd = _sig("optima_rms_norm_backward", _i32,
                 [_vp, _i64, _vp, _i32, _vp, _i64, _vp, _i64, _i32, _i64, _i64, _f32, _vp, _i64,
                  _vp, _i32, _vp, _sz, _vp])
_gated_ws = _sig("optima_gated_forward_workspace_bytes", _sz, [_i64, _i64, _i64])
_gated = _sig("optima_gated_forward", _i32,
              [_vp, _i64, _i64, _i64, _vp, _vp, _i64, _i32, _vp, _i64, _i32, _vp, _i64, _vp, _i64,
               _vp, _sz, _vp])
_gated_bwd_ws = _sig("optima_gated_backward_workspace_bytes", _sz, [_i64, _i64, _i64])
_gated_bwd = _sig("optima_gated_backward", _i32,
                  [_vp, _i64, _i64, _i64, _vp, _vp, _i64, _i32, _vp, _i64, _vp, _i64, _vp, _i64,
                   _vp, _i64, _i32, _vp, _vp, _i32, _vp, _vp, _i32, _vp, _sz, _vp])
_w4_row = _sig("optima_w4_row_bytes", _sz, [_i64])
_w4_pack = _sig("optima_w4_pack", _i32, [_vp, _i32, _i64, _i64, _i64, _vp, _vp, _vp])
_w4_linear = _sig("optima_w4_linear", _i32,
                  [_vp, _i64, _i32, _vp, _i64, _i64, _i64, _vp, _vp, _i64, _i64, _vp, _i64, _i32,
                   _vp, _sz, _vp])
_w4_ws = _sig("optima_w4_workspace_bytes", _sz, [_i64, _i64, _i64, _i32])
_w4_gated = _sig("optima_w4_gated", _i32,
                 [_vp, _i64, _i32, _vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _i64, _i64, _i32,
                  _vp, _i64, _i32, _vp, _sz, _vp])

_mx4_row = _sig("optima_mx4_row_bytes", _sz, [_i64])
_mx4_scale_row = _sig("optima_mx4_scale_bytes", _sz, [_i64])
_mx4_pack = _sig("optima_mx4_pack", _i32, [_vp, _i64, _i32, _i64, _i64, _vp, _vp, _vp])
_mx4_unpack = _sig("optima_mx4_unpack", _i32, [_vp, _vp, _i64, _i64, _vp, _i64, _i32, _vp])
_mx4_ws = _sig("optima_mx4_workspace_bytes", _sz, [_i64, _i64, _i64])
_mx4_linear = _sig("optima_mx4_linear", _i32,
                   [_vp, _i64, _i32, _vp, _i64, _i64, _vp, _vp, _i64, _vp, _i64, _i32, _vp, _sz,
                    _vp])
_logprobs_ws = _sig("optima_token_logprobs_workspace_bytes", _sz, [_i64, _i64, _i64])
_logprobs = _sig("optima_token_logprobs", _i32,
                 [_vp, _i64, _i32, _i64, _i64, _vp, _f32, _vp, _vp, _vp, _i64, _vp, _vp, _vp, _sz,
                  _vp])
_logprobs_bwd = _sig("optima_token_logprobs_backward", _i32,
                     [_vp, _i64, _i32, _i64, _i64, _vp, _f32, _vp, _vp, _vp, _vp, _vp, _vp, _i64,
                      _vp])


def library_path() -> str:
    return _LIB_PATH


def optima_status_string(status: int) -> str:
    return _status_string(int(status)).decode()


def optima_abi_version() -> int:
    return int(_abi_version())


def _check(status: int):
    if status != OPTIMA_OK:
        raise OptimaError(status, optima_status_string(status))


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _need_cuda(name, t, dtype=None):
    if t is None:
        raise ValueError(f"{name} is required")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")


def _workspace(nbytes: int, ws, device, stream=None):
    """The caller's workspace, or a new one allocated on the stream the call
    runs on. torch's caching allocator ties a block to the stream it was
    allocated on, so the block freed when the call returns is handed only to
    later work on that stream, which runs after the library's kernels."""
    if ws is not None:
        _need_cuda("ws", ws)
        return ws, ws.numel() * ws.element_size()
    n = max(int(nbytes), 1)
    if stream is None:
        return torch.empty(n, dtype=torch.uint8, device=device), int(nbytes)
    with torch.cuda.stream(stream):
        return torch.empty(n, dtype=torch.uint8, device=device), int(nbytes)


@dataclass
class SolverOpts:
    """Mirror of optima_solver_opts; defaults come from the library."""
    max_iters: int = 0
    check_every: int = 0
    fixed_iters: int = 0
    eps_rel: float = 0.0
    eps_abs: float = 0.0
    beta_sufficient: float = 0.0
    beta_necessary: float = 0.0
    beta_artificial: float = 0.0
    step_safety: float = 0.0
    restarts: int = 0
    precision: int = 0
    method: int = 0
    col_scale: "torch.Tensor | None" = None  # [d] float32 device scaling D, or None
    sparse: int = 0
    cooperative: int = 0

    @classmethod
    def default(cls, **overrides) -> "SolverOpts":
        c = _Opts()
        _opts_default(ctypes.byref(c))
        o = cls(**{f.name: getattr(c, f.name) for f in fields(cls)})
        for k, v in overrides.items():
            if not hasattr(o, k):
                raise AttributeError(k)
            setattr(o, k, v)
        return o

    def _c(self) -> _Opts:
        vals = {f.name: getattr(self, f.name) for f in fields(self)}
        scale = vals.pop("col_scale")
        c = _Opts(**vals)
        c.col_scale = None if scale is None else scale.data_ptr()
        return c


def optima_hessian_workspace_bytes(n_tok: int, d: int, dtype: int) -> int:
    return int(_hess_ws(n_tok, d, dtype))


def optima_hessian_accumulate(X: torch.Tensor, H: torch.Tensor, accumulate: bool = False,
                              ws: torch.Tensor | None = None, stream=None) -> None:
    """H (+)= X^T X for X [n_tok, d] (float32 or bfloat16), H [d, d] float32."""
    _need_cuda("X", X)
    _need_cuda("H", H, torch.float32)
    if X.dim() != 2 or H.shape != (X.shape[1], X.shape[1]):
        raise ValueError("X must be [n_tok, d] and H [d, d]")
    dtype = {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16}.get(X.dtype)
    if dtype is None:
        raise ValueError("X must be float32 or bfloat16")
    n_tok, d = X.shape
    ws, nbytes = _workspace(optima_hessian_workspace_bytes(n_tok, d, dtype), ws, X.device,
                           stream)
    _check(_hess_acc(_ptr(X), dtype, n_tok, d, _ptr(H), int(bool(accumulate)), _ptr(ws),
                     nbytes, _stream(stream)))


def optima_hessian_damp(H: torch.Tensor, rel_damp: float, lambda_out: torch.Tensor,
                        stream=None) -> None:
    _need_cuda("H", H, torch.float32)
    _need_cuda("lambda_out", lambda_out, torch.float32)
    _check(_damp(_ptr(H), H.shape[0], float(rel_damp), _ptr(lambda_out), _stream(stream)))


SPECTRAL_MAX_BLOCK = 16


def optima_hessian_jacobi(H: torch.Tensor, scale_out: torch.Tensor, stream=None) -> None:
    """H <- D H D in place with D = diag(H)^(-1/2); scale_out [d] receives D."""
    _need_cuda("H", H, torch.float32)
    _need_cuda("scale_out", scale_out, torch.float32)
    if H.dim() != 2 or H.shape[0] != H.shape[1] or scale_out.numel() != H.shape[0]:
        raise ValueError("H must be [d, d] and scale_out [d]")
    _check(_jacobi(_ptr(H), H.shape[0], _ptr(scale_out), _stream(stream)))


def optima_spectral_norm_workspace_bytes(d: int, block: int = 1) -> int:
    return int(_spec_ws(d, block))


def optima_spectral_norm(H: torch.Tensor, V0: torch.Tensor, lambda_max: torch.Tensor,
                         max_iters: int = 1000, tol: float = 1e-6,
                         ws: torch.Tensor | None = None, iters: torch.Tensor | None = None,
                         stream=None) -> None:
    """lambda_max(H). V0 is one start vector [d] (power iteration) or a block
    of start vectors [block, d] (subspace iteration with Rayleigh-Ritz)."""
    _need_cuda("H", H, torch.float32)
    _need_cuda("V0", V0, torch.float32)
    _need_cuda("lambda_max", lambda_max, torch.float32)
    if iters is not None:
        _need_cuda("iters", iters, torch.int32)
    d = H.shape[0]
    if V0.dim() == 1:
        block = 1
    elif V0.dim() == 2:
        block = V0.shape[0]
    else:
        raise ValueError("V0 must be [d] or [block, d]")
    if V0.shape[-1] != d:
        raise ValueError("V0 vectors must have length d")
    ws, nbytes = _workspace(optima_spectral_norm_workspace_bytes(d, block), ws, H.device,
                           stream)
    _check(_spec(_ptr(H), d, _ptr(V0), int(block), int(max_iters), float(tol), _ptr(ws), nbytes,
                 _ptr(lambda_max), _ptr(iters), _stream(stream)))


SPECTRAL_NOALLOC_MAX_DIM = 16384


def optima_spectral_norm_noalloc(H: torch.Tensor, V0: torch.Tensor, lambda_max: torch.Tensor,
                                 max_iters: int = 1000, tol: float = 1e-6,
                                 iters: torch.Tensor | None = None, stream=None) -> None:
    """optima_spectral_norm with the library's fixed per-device work array
    instead of a workspace: nothing is allocated (d <= SPECTRAL_NOALLOC_MAX_DIM;
    calls that overlap on one device race on that array)."""
    _need_cuda("H", H, torch.float32)
    _need_cuda("V0", V0, torch.float32)
    _need_cuda("lambda_max", lambda_max, torch.float32)
    if iters is not None:
        _need_cuda("iters", iters, torch.int32)
    d = H.shape[0]
    if V0.dim() not in (1, 2) or V0.shape[-1] != d:
        raise ValueError("V0 must be [d] or [block, d]")
    block = 1 if V0.dim() == 1 else V0.shape[0]
    _check(_spec_na(_ptr(H), d, _ptr(V0), int(block), int(max_iters), float(tol),
                    _ptr(lambda_max), _ptr(iters), _stream(stream)))


LANCZOS_MAX_STEPS = 256


def optima_spectral_lanczos_workspace_bytes(d: int, max_steps: int = LANCZOS_MAX_STEPS) -> int:
    return int(_lz_ws(d, max_steps))


def optima_spectral_lanczos(H: torch.Tensor, v0: torch.Tensor, lambda_max: torch.Tensor,
                            max_steps: int = LANCZOS_MAX_STEPS, tol: float = 1e-7,
                            ws: torch.Tensor | None = None, steps: torch.Tensor | None = None,
                            stream=None) -> None:
    """lambda_max(H) by the Lanczos process started from v0 [d]."""
    _need_cuda("H", H, torch.float32)
    _need_cuda("v0", v0, torch.float32)
    _need_cuda("lambda_max", lambda_max, torch.float32)
    if steps is not None:
        _need_cuda("steps", steps, torch.int32)
    d = H.shape[0]
    if v0.dim() != 1 or v0.shape[0] != d:
        raise ValueError("v0 must be [d]")
    ws, nbytes = _workspace(optima_spectral_lanczos_workspace_bytes(d, max_steps), ws, H.device,
                           stream)
    _check(_lz(_ptr(H), d, _ptr(v0), int(max_steps), float(tol), _ptr(ws), nbytes,
               _ptr(lambda_max), _ptr(steps), _stream(stream)))


ACT_NONE = 0
ACT_SILU = 1


def optima_linear_forward_workspace_bytes(n_tok: int, d_in: int, d_out: int) -> int:
    return int(_fwd_ws(n_tok, d_in, d_out))


def optima_linear_forward(X: torch.Tensor, W: torch.Tensor, Y: torch.Tensor | None = None,
                          act: int = ACT_NONE, Y_ref: torch.Tensor | None = None,
                          err_out: torch.Tensor | None = None, ws: torch.Tensor | None = None,
                          stream=None) -> None:
    """Y = act(X W^T) for X [n_tok, d_in] bfloat16 and W [d_out, d_in] float32
    (rounded to bf16 on the device); Y bfloat16 or float32 [n_tok, d_out].
    With Y_ref (float32 [n_tok, d_out]) err_out (float64 [1]) receives the sum
    of (X W^T - Y_ref)^2."""
    _need_cuda("X", X, torch.bfloat16)
    _need_cuda("W", W, torch.float32)
    if X.dim() != 2 or W.dim() != 2 or W.shape[1] != X.shape[1]:
        raise ValueError("X must be [n_tok, d_in] and W [d_out, d_in]")
    n_tok, d_in = X.shape
    d_out = W.shape[0]
    y_dtype = -1
    if Y is not None:
        _need_cuda("Y", Y)
        y_dtype = {torch.bfloat16: DTYPE_BF16, torch.float32: DTYPE_F32}.get(Y.dtype, -1)
        if y_dtype < 0 or Y.shape != (n_tok, d_out):
            raise ValueError("Y must be bfloat16 or float32 [n_tok, d_out]")
    if Y_ref is not None:
        _need_cuda("Y_ref", Y_ref, torch.float32)
        if Y_ref.shape != (n_tok, d_out):
            raise ValueError("Y_ref must be [n_tok, d_out]")
    if (Y_ref is None) != (err_out is None):
        raise ValueError("Y_ref and err_out go together")
    if err_out is not None:
        _need_cuda("err_out", err_out, torch.float64)
    ws, nbytes = _workspace(optima_linear_forward_workspace_bytes(n_tok, d_in, d_out), ws,
                            W.device, stream)
    empty = n_tok == 0  # an empty tensor may report a null address
    _check(_fwd(None if empty else _ptr(X), n_tok, d_in, _ptr(W), d_out, int(act),
                None if empty else _ptr(Y), y_dtype, None if empty else _ptr(Y_ref),
                _ptr(err_out), _ptr(ws), nbytes, _stream(stream)))


MASK_UNSTRUCTURED = 0
MASK_2TO4 = 1


def optima_wanda_mask(W0: torch.Tensor, col_sq: torch.Tensor, mask: torch.Tensor,
                      pattern: int = MASK_UNSTRUCTURED, sparsity: float = 0.5,
                      col_sq_stride: int = 1, stream=None) -> None:
    """Wanda mask of W0 [n_cols, d] into mask [n_cols, d] (uint8, 1 keeps).

    col_sq holds the squared input norms, element i at flat index
    i * col_sq_stride (float32 or float64); the undamped Hessian H [d, d] with
    col_sq_stride = d + 1 passes its diagonal."""
    _need_cuda("W0", W0, torch.float32)
    _need_cuda("col_sq", col_sq)
    _need_cuda("mask", mask, torch.uint8)
    if W0.dim() != 2 or mask.shape != W0.shape:
        raise ValueError("W0 and mask must be [n_cols, d]")
    n, d = W0.shape
    dt = {torch.float32: DTYPE_F32, torch.float64: DTYPE_F64}.get(col_sq.dtype)
    if dt is None:
        raise ValueError("col_sq must be float32 or float64")
    if d > 0 and (d - 1) * int(col_sq_stride) + 1 > col_sq.numel():
        raise ValueError("col_sq too short for d and the stride")
    _check(_mask(_ptr(W0), n, d, _ptr(col_sq), dt, int(col_sq_stride), int(pattern),
                 float(sparsity), _ptr(mask), _stream(stream)))


def optima_qp_workspace_bytes(d: int, n_cols: int) -> int:
    return int(_qp_ws(d, n_cols))


def optima_qp_solve_batched(H: torch.Tensor, lambda_max: torch.Tensor | None, W0: torch.Tensor,
                            mask: torch.Tensor, W_out: torch.Tensor,
                            opts: SolverOpts | None = None, ws: torch.Tensor | None = None,
                            stats: dict | None = None, stream=None) -> dict:
    """Solves every row QP of W0 under `mask`; returns the run totals.

    lambda_max may be None with opts.method == METHOD_CG. stats: optional dict
    of device tensors with keys among iters (int32), restarts (int32),
    converged (uint8), f_initial, f_final, kkt_final (float32).
    """
    _need_cuda("H", H, torch.float32)
    if lambda_max is not None:
        _need_cuda("lambda_max", lambda_max, torch.float32)
    _need_cuda("W0", W0, torch.float32)
    _need_cuda("mask", mask, torch.uint8)
    _need_cuda("W_out", W_out, torch.float32)
    n_cols, d = W0.shape
    if H.shape != (d, d) or mask.shape != W0.shape or W_out.shape != W0.shape:
        raise ValueError("shape mismatch between H, W0, mask and W_out")
    opts = opts or SolverOpts.default()
    if opts.col_scale is not None:
        _need_cuda("opts.col_scale", opts.col_scale, torch.float32)
        if opts.col_scale.numel() != d:
            raise ValueError("opts.col_scale must have d entries")
    ws, nbytes = _workspace(optima_qp_workspace_bytes(d, n_cols), ws, W0.device, stream)
    st = _Stats()
    kinds = {"iters": torch.int32, "restarts": torch.int32, "converged": torch.uint8,
             "f_initial": torch.float32, "f_final": torch.float32, "kkt_final": torch.float32}
    for key, t in (stats or {}).items():
        if key not in kinds:
            raise KeyError(key)
        _need_cuda(key, t, kinds[key])
        if t.numel() != n_cols:
            raise ValueError(f"stats[{key}] must have n_cols entries")
        setattr(st, key, t.data_ptr())
    info = _Info()
    c_opts = opts._c()
    _check(_qp_solve(_ptr(H), d, _ptr(lambda_max), _ptr(W0), _ptr(mask), n_cols,
                     ctypes.byref(c_opts), _ptr(ws), nbytes, _ptr(W_out), ctypes.byref(st),
                     ctypes.byref(info), _stream(stream)))
    return {f[0]: getattr(info, f[0]) for f in _Info._fields_}


_ROW_DTYPES = {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16, torch.int8: DTYPE_I8}


def _rows(name, t, shape, dtypes):
    """(address, row pitch, dtype code) of a token matrix: rows of consecutive elements,
    any pitch. The address of a matrix without rows is NULL."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    if t.dtype not in dtypes:
        raise ValueError(f"{name} must be one of {dtypes}, got {t.dtype}")
    n, d = shape
    ld = t.stride(0) if n > 1 else d
    if (d > 1 and t.stride(1) != 1) or ld < d:
        raise ValueError(f"{name} must have rows of consecutive elements that do not overlap")
    return (t.data_ptr() if n else None), ld, _ROW_DTYPES[t.dtype]


def _take(name, t, shape, dtypes):
    """_rows, for a contiguous tensor with fewer questions: a third of its time, of which a
    call of a decoding step takes several."""
    dtype = t.dtype
    if t.is_contiguous() and dtype in dtypes and t.is_cuda and t.shape == shape:
        return (t.data_ptr() if shape[0] else None), shape[1], _ROW_DTYPES[dtype]
    return _rows(name, t, shape, dtypes)


def _launch_stream(stream):
    """The stream's address, as _stream's. The decoding calls take a few microseconds, of
    which making a Stream object would be two or three."""
    if stream is not None:
        return stream.cuda_stream
    return _raw_stream(_current_device())


_current_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else \
    torch.cuda.current_device
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _addr(t):
    return None if t is None else t.data_ptr()


def _opt_rows(name, t, shape, dtypes):
    return (None, shape[1], 0) if t is None else _take(name, t, shape, dtypes)


def _need_shape(name, t, shape, dtypes):
    if t is not None and t.is_contiguous() and t.dtype in dtypes and t.is_cuda and \
            t.shape == shape:
        return
    _need_cuda(name, t)
    if t.dtype not in dtypes:
        raise ValueError(f"{name} must be one of {dtypes}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")


_F = (torch.float32, torch.bfloat16)
_B = (torch.bfloat16,)
NORM_MAX_DIM = 16384


def optima_rms_norm(X: torch.Tensor, weight: torch.Tensor, Y: torch.Tensor, eps: float = 1e-6,
                    R: torch.Tensor | None = None, S: torch.Tensor | None = None,
                    scales: torch.Tensor | None = None, group: int = 0, stream=None) -> None:
    """Y = s * weight / sqrt(mean(s^2) + eps) with s = X + R, row by row; S receives s.

    X, R, S [n_tok, d] float32 or bfloat16 (one type); weight [d] float32 or bfloat16; Y
    float32, bfloat16, or int8 codes with scales (float32 [n_tok, ceil(d / group)], or
    [n_tok, 1] with group = 0). S may be X or R. Rows may have any pitch."""
    if X.dim() != 2:
        raise ValueError("X must be [n_tok, d]")
    n, d = X.shape
    x, ldx, dt = _take("X", X, (n, d), _F)
    r, ldr, _ = _opt_rows("R", R, (n, d), (X.dtype,))
    s, lds, _ = _opt_rows("S", S, (n, d), (X.dtype,))
    y, ldy, y_dt = _take("Y", Y, (n, d), (*_F, torch.int8))
    _need_shape("weight", weight, (d,), _F)
    if (Y.dtype == torch.int8) != (scales is not None):
        raise ValueError("scales go with an int8 Y")
    if scales is not None:
        groups = -(-d // group) if group > 0 else 1
        _need_shape("scales", scales, (n, groups), (torch.float32,))
    _check(_norm(x, ldx, r, ldr, dt, n, d, _addr(weight), _ROW_DTYPES[weight.dtype], float(eps), s,
                 lds, y, ldy, y_dt, _addr(scales), int(group), _launch_stream(stream)))


def optima_rms_norm_backward_workspace_bytes(n_tok: int, d: int) -> int:
    return int(_norm_bwd_ws(n_tok, d))


def optima_rms_norm_backward(S: torch.Tensor, weight: torch.Tensor, dY: torch.Tensor,
                             dX: torch.Tensor, eps: float = 1e-6, dS: torch.Tensor | None = None,
                             dweight: torch.Tensor | None = None, accumulate: bool = False,
                             ws: torch.Tensor | None = None, stream=None) -> None:
    """dX, the gradient of X and of R, and dweight (float32 [d]; + what it holds with
    accumulate) of optima_rms_norm at the S it stored, from dY and the gradient dS that
    reaches S itself. S, dY, dS and dX are [n_tok, d] of one type; dX may be dY or dS."""
    if S.dim() != 2:
        raise ValueError("S must be [n_tok, d]")
    n, d = S.shape
    s, lds, dt = _take("S", S, (n, d), _F)
    dy, lddy, _ = _take("dY", dY, (n, d), (S.dtype,))
    ds, ldds, _ = _opt_rows("dS", dS, (n, d), (S.dtype,))
    dx, lddx, _ = _take("dX", dX, (n, d), (S.dtype,))
    _need_shape("weight", weight, (d,), _F)
    nbytes = 0
    if dweight is not None:
        _need_shape("dweight", dweight, (d,), (torch.float32,))
        ws, nbytes = _workspace(optima_rms_norm_backward_workspace_bytes(n, d), ws, S.device,
                                stream)
    _check(_norm_bwd(s, lds, _addr(weight), _ROW_DTYPES[weight.dtype], dy, lddy, ds, ldds, dt, n, d,
                     float(eps), dx, lddx, _addr(dweight), int(bool(accumulate)), _addr(ws), nbytes,
                     _launch_stream(stream)))


def optima_gated_forward_workspace_bytes(n_tok: int, d_in: int, d_ff: int) -> int:
    return int(_gated_ws(n_tok, d_in, d_ff))


def _gated_weights(X, Wg, Wu):
    if X.dim() != 2 or Wg.dim() != 2:
        raise ValueError("X must be [n_tok, d_in] and Wg, Wu [d_ff, d_in]")
    n, d = X.shape
    ff = Wg.shape[0]
    _need_shape("Wg", Wg, (ff, d), _B)
    _need_shape("Wu", Wu, (ff, d), _B)
    return n, d, ff


def optima_gated_forward(X: torch.Tensor, Wg: torch.Tensor, Wu: torch.Tensor, H: torch.Tensor,
                         act: int = ACT_SILU, G: torch.Tensor | None = None,
                         U: torch.Tensor | None = None, ws: torch.Tensor | None = None,
                         stream=None) -> None:
    """H = act(X Wg^T) * (X Wu^T) for X [n_tok, d_in] and Wg, Wu [d_ff, d_in] bfloat16; H
    bfloat16 or float32 [n_tok, d_ff]. G and U (bfloat16) receive the two products, which
    optima_gated_backward takes."""
    n, d, ff = _gated_weights(X, Wg, Wu)
    x, ldx, _ = _take("X", X, (n, d), _B)
    h, ldh, h_dt = _take("H", H, (n, ff), _F)
    g, ldg, _ = _opt_rows("G", G, (n, ff), _B)
    u, ldu, _ = _opt_rows("U", U, (n, ff), _B)
    need = optima_gated_forward_workspace_bytes(n, d, ff)
    nbytes = 0
    if need or ws is not None:
        ws, nbytes = _workspace(need, ws, X.device, stream)
    _check(_gated(x, ldx, n, d, _addr(Wg), _addr(Wu), ff, int(act), h, ldh, h_dt, g, ldg, u, ldu,
                  _addr(ws), nbytes, _launch_stream(stream)))


def optima_gated_backward_workspace_bytes(n_tok: int, d_in: int, d_ff: int) -> int:
    return int(_gated_bwd_ws(n_tok, d_in, d_ff))


def optima_gated_backward(X: torch.Tensor, Wg: torch.Tensor, Wu: torch.Tensor, G: torch.Tensor,
                          U: torch.Tensor, dH: torch.Tensor, dX: torch.Tensor | None = None,
                          dWg: torch.Tensor | None = None, dWu: torch.Tensor | None = None,
                          act: int = ACT_SILU, mask_g: torch.Tensor | None = None,
                          mask_u: torch.Tensor | None = None, accumulate: bool = False,
                          ws: torch.Tensor | None = None, stream=None) -> None:
    """Gradients of optima_gated_forward: dX [n_tok, d_in] and dWg, dWu [d_ff, d_in], each
    bfloat16 or float32 (dWg and dWu of one type, + what they hold with accumulate). Where
    mask_g or mask_u (uint8 [d_ff, d_in]) is 0 the weight's gradient is exactly 0."""
    n, d, ff = _gated_weights(X, Wg, Wu)
    x, ldx, _ = _take("X", X, (n, d), _B)
    g, ldg, _ = _take("G", G, (n, ff), _B)
    u, ldu, _ = _take("U", U, (n, ff), _B)
    dh, lddh, _ = _take("dH", dH, (n, ff), _B)
    dx, lddx, dx_dt = _opt_rows("dX", dX, (n, d), _F)
    if (dWg is None) != (dWu is None):
        raise ValueError("dWg and dWu go together")
    dw_dt = 0
    if dWg is not None:
        _need_shape("dWg", dWg, (ff, d), _F)
        _need_shape("dWu", dWu, (ff, d), (dWg.dtype,))
        dw_dt = _ROW_DTYPES[dWg.dtype]
    for name, m in (("mask_g", mask_g), ("mask_u", mask_u)):
        if m is not None:
            _need_shape(name, m, (ff, d), (torch.uint8,))
    ws, nbytes = _workspace(optima_gated_backward_workspace_bytes(n, d, ff), ws, X.device, stream)
    _check(_gated_bwd(x, ldx, n, d, _addr(Wg), _addr(Wu), ff, int(act), g, ldg, u, ldu, dh, lddh, dx,
                      lddx, dx_dt, _addr(dWg), _addr(dWu), dw_dt, _addr(mask_g), _addr(mask_u),
                      int(bool(accumulate)), _addr(ws), nbytes, _launch_stream(stream)))


def optima_w4_row_bytes(d: int) -> int:
    return int(_w4_row(d))


def optima_w4_pack(W: torch.Tensor, Q: torch.Tensor, scales: torch.Tensor, group: int = 128,
                   stream=None) -> None:
    """4-bit codes and scales of W [n, d] (float32 or bfloat16): Q uint8
    [n, optima_w4_row_bytes(d)], scales bfloat16 [n, ceil(d / group)], group 32, 64 or
    128. Zero weights stay exactly zero."""
    if W.dim() != 2:
        raise ValueError("W must be [n, d]")
    n, d = W.shape
    _need_shape("W", W, (n, d), _F)
    _w4_weights("Q", Q, "scales", scales, n, d, group)
    _check(_w4_pack(_addr(W), _ROW_DTYPES[W.dtype], n, d, int(group), _addr(Q), _addr(scales),
                    _launch_stream(stream)))


def _w4_weights(q_name, Q, s_name, scales, n, d, group):
    if group not in (32, 64, 128):
        raise ValueError("group must be 32, 64 or 128")
    _need_shape(q_name, Q, (n, -(-d // 128) * 64), (torch.uint8,))
    _need_shape(s_name, scales, (n, -(-d // group)), _B)


def _w4_tokens(X, x_scales, x_group, group):
    if X.dim() != 2:
        raise ValueError("X must be [n_tok, d]")
    n, d = X.shape
    x, ldx, x_dt = _take("X", X, (n, d), (torch.bfloat16, torch.int8))
    if (X.dtype == torch.int8) != (x_scales is not None):
        raise ValueError("x_scales go with an int8 X")
    if x_scales is not None:
        if x_group not in (0, group):
            raise ValueError("x_group must be the weights' group, or 0 (one scale a token)")
        _need_shape("x_scales", x_scales, (n, -(-d // x_group) if x_group else 1),
                    (torch.float32,))
    return n, d, x, ldx, x_dt


def optima_w4_workspace_bytes(n_tok: int, d: int, d_out: int, n_mats: int = 1) -> int:
    return int(_w4_ws(n_tok, d, d_out, n_mats))


def _w4_space(n, d, n_out, mats, ws, device, stream):
    """(address, bytes) of the workspace; up to 16 tokens need none. One made here is
    freed when the call returns, for later work on the stream (see _workspace)."""
    need = optima_w4_workspace_bytes(n, d, n_out, mats) if n > 16 else 0
    if not need and ws is None:
        return None, 0
    ws, nbytes = _workspace(need, ws, device, stream)
    return ws.data_ptr(), nbytes


def optima_w4_linear(X: torch.Tensor, Q: torch.Tensor, scales: torch.Tensor, Y: torch.Tensor,
                     group: int = 128, x_scales: torch.Tensor | None = None, x_group: int = 0,
                     ws: torch.Tensor | None = None, stream=None) -> None:
    """Y = X W^T for the weights W [d_out, d] that Q and scales stand for (optima_w4_pack).
    X [n_tok, d] bfloat16, or int8 with x_scales as optima_rms_norm writes them (x_group is
    its group: the weights' group, or 0); Y [n_tok, d_out] bfloat16 or float32."""
    n, d, x, ldx, x_dt = _w4_tokens(X, x_scales, x_group, group)
    n_out = Q.shape[0]
    _w4_weights("Q", Q, "scales", scales, n_out, d, group)
    y, ldy, y_dt = _take("Y", Y, (n, n_out), _F)
    ws, nbytes = _w4_space(n, d, n_out, 1, ws, X.device, stream)
    _check(_w4_linear(x, ldx, x_dt, _addr(x_scales), int(x_group), n, d, _addr(Q), _addr(scales),
                      int(group), n_out, y, ldy, y_dt, ws, nbytes, _launch_stream(stream)))


def optima_w4_gated(X: torch.Tensor, Qg: torch.Tensor, scales_g: torch.Tensor, Qu: torch.Tensor,
                    scales_u: torch.Tensor, H: torch.Tensor, group: int = 128,
                    act: int = ACT_SILU, x_scales: torch.Tensor | None = None, x_group: int = 0,
                    ws: torch.Tensor | None = None, stream=None) -> None:
    """H = act(X Wg^T) * (X Wu^T) with both weights in 4 bits; arguments as in
    optima_w4_linear."""
    n, d, x, ldx, x_dt = _w4_tokens(X, x_scales, x_group, group)
    ff = Qg.shape[0]
    _w4_weights("Qg", Qg, "scales_g", scales_g, ff, d, group)
    _w4_weights("Qu", Qu, "scales_u", scales_u, ff, d, group)
    h, ldh, h_dt = _take("H", H, (n, ff), _F)
    ws, nbytes = _w4_space(n, d, ff, 2, ws, X.device, stream)
    _check(_w4_gated(x, ldx, x_dt, _addr(x_scales), int(x_group), n, d, _addr(Qg), _addr(scales_g),
                     _addr(Qu), _addr(scales_u), int(group), ff, int(act), h, ldh, h_dt, ws,
                     nbytes, _launch_stream(stream)))


@functools.lru_cache(maxsize=None)
def _devices() -> int:
    return torch.cuda.device_count()


def _need_one_device(stream, *tensors):
    """A call launches on the current device, or its stream's: all its tensors are there."""
    if _devices() < 2:
        return
    at = _current_device() if stream is None else stream.device.index
    for t in tensors:
        if t is not None and t.is_cuda and t.get_device() != at:
            raise ValueError(f"a tensor is on device {t.get_device()}, the call runs on {at}")


def optima_mx4_row_bytes(d: int) -> int:
    return int(_mx4_row(d))


def optima_mx4_scale_bytes(d: int) -> int:
    return int(_mx4_scale_row(d))


def _mx4_codes(q_name, Q, s_name, scales, n, d):
    if Q.dtype == scales.dtype == torch.uint8 and Q.is_cuda and scales.is_cuda and \
            Q.is_contiguous() and scales.is_contiguous() and \
            Q.shape == (n, (d + 255) // 256 * 128) and scales.shape == (n, (d + 511) // 512 * 16):
        return
    _need_shape(q_name, Q, (n, -(-d // 256) * 128), (torch.uint8,))
    _need_shape(s_name, scales, (n, -(-d // 512) * 16), (torch.uint8,))


def _mx4_addr(t):
    return t.data_ptr() or None  # an empty tensor may report a null address


def optima_mx4_pack(X: torch.Tensor, Q: torch.Tensor, scales: torch.Tensor, stream=None) -> None:
    """Microscaled 4-bit floating point codes and scales of X [n, d] (float32 or bfloat16, weights
    or tokens; rows may have any pitch): Q uint8 [n, optima_mx4_row_bytes(d)], scales uint8
    [n, optima_mx4_scale_bytes(d)]. Zeros stay exactly zero."""
    if X.dim() != 2:
        raise ValueError("X must be [n, d]")
    n, d = X.shape
    x, ldx, dt = _take("X", X, (n, d), _F)
    _mx4_codes("Q", Q, "scales", scales, n, d)
    _need_one_device(stream, X, Q, scales)
    _check(_mx4_pack(x, ldx, dt, n, d, _mx4_addr(Q), _mx4_addr(scales), _launch_stream(stream)))


def optima_mx4_unpack(Q: torch.Tensor, scales: torch.Tensor, Y: torch.Tensor,
                      stream=None) -> None:
    """Y [n, d] (float32 or bfloat16), the values that Q and scales stand for (optima_mx4_pack)."""
    if Y.dim() != 2:
        raise ValueError("Y must be [n, d]")
    n, d = Y.shape
    y, ldy, dt = _take("Y", Y, (n, d), _F)
    _mx4_codes("Q", Q, "scales", scales, n, d)
    _need_one_device(stream, Q, scales, Y)
    _check(_mx4_unpack(_mx4_addr(Q), _mx4_addr(scales), n, d, y, ldy, dt, _launch_stream(stream)))


@functools.lru_cache(maxsize=4096)
def optima_mx4_workspace_bytes(n_tok: int, d: int, d_out: int) -> int:
    return int(_mx4_ws(n_tok, d, d_out))


def optima_mx4_linear(X: torch.Tensor, Q: torch.Tensor, scales: torch.Tensor, Y: torch.Tensor,
                      x_scales: torch.Tensor | None = None, ws: torch.Tensor | None = None,
                      stream=None) -> None:
    """Y = X W^T for the weights W [d_out, d] that Q and scales stand for (optima_mx4_pack). X
    [n_tok, d] bfloat16, or the codes of packed tokens with x_scales; Y [n_tok, d_out] bfloat16
    or float32."""
    if X.dim() != 2 or Q.dim() != 2:
        raise ValueError("X must be [n_tok, d], or codes, and Q codes")
    n, n_out = X.shape[0], Q.shape[0]
    if (X.dtype == torch.uint8) != (x_scales is not None):
        raise ValueError("x_scales go with the codes of packed tokens")
    if x_scales is None:
        d = X.shape[1]
        x, ldx, x_dt = _take("X", X, (n, d), _B)
        _mx4_codes("Q", Q, "scales", scales, n_out, d)
    else:
        # The padding's codes are 0: the width up to it does as well as the tokens' own.
        d = 2 * X.shape[1]
        _mx4_codes("X", X, "x_scales", x_scales, n, d)
        _mx4_codes("Q", Q, "scales", scales, n_out, d)
        x, ldx, x_dt, xs = _mx4_addr(X), 0, DTYPE_MX4, _mx4_addr(x_scales)
    y, ldy, y_dt = _take("Y", Y, (n, n_out), _F)
    _need_one_device(stream, X, x_scales, Q, scales, Y, ws)
    need = optima_mx4_workspace_bytes(n, d, n_out) if n > 8 else 0
    nbytes = 0
    if need or ws is not None:
        ws, nbytes = _workspace(need, ws, X.device, stream)
    _check(_mx4_linear(x, ldx, x_dt, None if x_scales is None else xs, n, d, _addr(Q),
                       _addr(scales), n_out, y, ldy, y_dt, _addr(ws), nbytes,
                       _launch_stream(stream)))


TOP_MAX = 32


@functools.lru_cache(maxsize=4096)
def optima_token_logprobs_workspace_bytes(n: int, vocab: int, top: int = 0) -> int:
    return int(_logprobs_ws(n, vocab, top))


def _logits(logits):
    if logits.dim() != 2:
        raise ValueError("logits must be [n, vocab]")
    n, vocab = logits.shape
    return (n, vocab, *_take("logits", logits, (n, vocab), _F))


def _row_values(name, t, shape, dtype):
    """The address of a contiguous tensor or None, NULL without elements."""
    if t is None:
        return None
    if not (t.dtype == dtype and t.is_cuda and t.shape == shape and t.is_contiguous()):
        _need_shape(name, t, shape, (dtype,))
    return t.data_ptr() or None


def optima_token_logprobs(logits: torch.Tensor, tokens: torch.Tensor | None,
                          logp: torch.Tensor | None, lse: torch.Tensor | None = None,
                          entropy: torch.Tensor | None = None,
                          top_index: torch.Tensor | None = None,
                          top_logp: torch.Tensor | None = None, scale: float = 1.0,
                          ws: torch.Tensor | None = None, stream=None) -> None:
    """Log probabilities of the given tokens (int64 [n]; a negative one is none: 0) under the
    logits [n, vocab] (float32 or bfloat16; rows may have any pitch) times scale, with the
    logarithm of the sum of exponentials lse and the entropy, float32 [n]; and the k most probable
    alternatives, top_index int64 and top_logp float32 [n, k], equal ones by rising index."""
    n, vocab, x, ldx, dt = _logits(logits)
    rows = (n,)
    t = _row_values("tokens", tokens, rows, torch.int64)
    if logp is not None and tokens is None:
        raise ValueError("logp goes with tokens")
    p = _row_values("logp", logp, rows, torch.float32)
    s = _row_values("lse", lse, rows, torch.float32)
    h = _row_values("entropy", entropy, rows, torch.float32)
    k, index, top = 0, None, None
    if top_index is not None or top_logp is not None:
        shape = (top_logp if top_index is None else top_index).shape
        if len(shape) != 2:
            raise ValueError("top_index and top_logp must be [n, k]")
        k = shape[1]
        if not 0 < k <= min(vocab, TOP_MAX):
            raise ValueError(f"k must be 1 to {min(vocab, TOP_MAX)}, got {k}")
        index = _row_values("top_index", top_index, (n, k), torch.int64)
        top = _row_values("top_logp", top_logp, (n, k), torch.float32)
    elif logp is None and lse is None and entropy is None:
        raise ValueError("one output is needed")
    _need_one_device(stream, logits, tokens, logp, lse, entropy, top_index, top_logp, ws)
    need = optima_token_logprobs_workspace_bytes(n, vocab, k)
    nbytes = 0
    if need or ws is not None:
        ws, nbytes = _workspace(need, ws, logits.device, stream)
    _check(_logprobs(x, ldx, dt, n, vocab, t, float(scale), p, s, h, k, index, top, _addr(ws), nbytes,
                     _launch_stream(stream)))


def optima_token_logprobs_backward(logits: torch.Tensor, lse: torch.Tensor,
                                   dlogits: torch.Tensor, tokens: torch.Tensor | None = None,
                                   dlogp: torch.Tensor | None = None,
                                   entropy: torch.Tensor | None = None,
                                   dentropy: torch.Tensor | None = None,
                                   dlse: torch.Tensor | None = None, scale: float = 1.0,
                                   stream=None) -> None:
    """dlogits [n, vocab], of the logits' type, from the gradients that reach logp (with tokens),
    the entropy (with the entropy) and lse, float32 [n] each, and the lse that
    optima_token_logprobs stored. dlogits may be the logits themselves."""
    n, vocab, x, ldx, dt = _logits(logits)
    dx, lddx, _ = _take("dlogits", dlogits, (n, vocab), (logits.dtype,))
    t = _row_values("tokens", tokens, (n,), torch.int64)
    if lse is None:
        raise ValueError("lse is required")
    if dlogp is None and dentropy is None and dlse is None:
        raise ValueError("one of dlogp, dentropy and dlse is needed")
    if dlogp is not None and tokens is None:
        raise ValueError("dlogp goes with tokens")
    if dentropy is not None and entropy is None:
        raise ValueError("dentropy goes with the entropy")
    rows = [_row_values(name, o, (n,), torch.float32)
            for name, o in (("lse", lse), ("entropy", entropy), ("dlogp", dlogp),
                            ("dentropy", dentropy), ("dlse", dlse))]
    _need_one_device(stream, logits, lse, dlogits, tokens, dlogp, entropy, dentropy, dlse)
    _check(_logprobs_bwd(x, ldx, dt, n, vocab, t, float(scale), *rows, dx, lddx,
                         _launch_stream(stream)))
