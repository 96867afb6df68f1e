"""ctypes binding of libflashdiff.so: argument marshalling only.

Every function here has the name of the C entry point it wraps and passes
torch tensors' device pointers straight through; all arithmetic happens in
the library's HIP kernels.  PyTorch provides device memory (outputs and the
workspace) and the current HIP stream.  There is no fallback: if the library
is missing, or a call fails, an exception is raised.

The library must be loaded after ``import torch`` so that it binds to the
HIP runtime torch has already loaded (both carry the same soname).
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import Optional, Sequence

import torch  # noqa: F401  (load torch's HIP runtime first)

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libflashdiff.so")

FD_OK = 0
STATUS = {
    0: "FD_OK", 1: "FD_ERR_INVALID_ARG", 2: "FD_ERR_UNSUPPORTED", 3: "FD_ERR_WORKSPACE",
    4: "FD_ERR_HIP", 5: "FD_ERR_NOT_CONVERGED", 6: "FD_ERR_PERRON_WALL",
}
FD_F32, FD_BF16 = 0, 1
FD_OP_KERNEL_MATMUL, FD_OP_DEGREE, FD_OP_BLOCK_LANCZOS, FD_OP_CONTINUATION = 0, 1, 2, 3
FD_OP_BETA_FLOW = 4
FD_OP_DEGREE_DYADIC = 5
FLOW_EXIT = {0: "bracket", 1: "wall", 2: "budget", 3: "range"}

EXPORTS = (
    "fd_lanczos_default_opts", "fd_workspace_size", "fd_kernel_matmul", "fd_degree",
    "fd_block_lanczos", "fd_continuation", "fd_last_error", "fd_status_string",
    "fd_profile_enable", "fd_profile_read", "fd_flow_default_opts", "fd_beta_flow",
    "fd_beta_flow_cascade", "fd_degree_dyadic", "fd_kernel_matmul_noalloc",
    "fd_kernel_matmul_noalloc_limit", "fd_layer_norm", "fd_layer_norm_workspace_size",
    "fd_layer_norm_backward", "fd_gated_saved_size", "fd_gated_workspace_size",
    "fd_gated_forward", "fd_gated_backward", "fd_adamw_default_opts", "fd_adamw_step",
)
FD_ACT = {"silu": 0, "gelu": 1}
FD_GATED_FINE = 0x100
FD_ROUNDING = {"nearest": 0, "unbiased": 1}
FD_KERNEL_PRODUCT, FD_KERNEL_ROWSUM = 0, 1


class FdError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS.get(status, status)}: {msg}")
        self.status = status
        self.msg = msg


class LanczosOpts(ctypes.Structure):
    _fields_ = [("tol", ctypes.c_double), ("max_restarts", ctypes.c_int32),
                ("max_basis_blocks", ctypes.c_int32), ("keep", ctypes.c_int32),
                ("max_matvecs", ctypes.c_int32), ("verbose", ctypes.c_int32),
                ("seed", ctypes.c_uint64)]


class LanczosInfo(ctypes.Structure):
    _fields_ = [("restarts", ctypes.c_int32), ("block_matvecs", ctypes.c_int32),
                ("nconv", ctypes.c_int32), ("wall", ctypes.c_int32),
                ("gap_perron", ctypes.c_double), ("s_off", ctypes.c_double),
                ("max_residual", ctypes.c_double), ("seconds", ctypes.c_double)]

    def as_dict(self) -> dict:
        return {f: getattr(self, f) for f, _ in self._fields_}


class FlowOpts(ctypes.Structure):
    _fields_ = [("beta_start", ctypes.c_double), ("eta", ctypes.c_double),
                ("kappa", ctypes.c_double), ("p", ctypes.c_double),
                ("max_probes", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class FlowProbe(ctypes.Structure):
    _fields_ = [("beta", ctypes.c_double), ("s_off", ctypes.c_double),
                ("gap_perron", ctypes.c_double), ("v_bias", ctypes.c_double),
                ("v_mach", ctypes.c_double), ("n_eff", ctypes.c_double),
                ("v_stat", ctypes.c_double), ("v_total", ctypes.c_double),
                ("d_hat", ctypes.c_double), ("seconds", ctypes.c_double),
                ("role", ctypes.c_int32), ("admissible", ctypes.c_int32),
                ("status", ctypes.c_int32), ("block_matvecs", ctypes.c_int32),
                ("nconv", ctypes.c_int32), ("level", ctypes.c_int32)]

    def as_dict(self) -> dict:
        return {f: getattr(self, f) for f, _ in self._fields_ if f != "reserved"}


class GatedBlock(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int64), ("D", ctypes.c_int64), ("F", ctypes.c_int64),
                ("O", ctypes.c_int64), ("type", ctypes.c_int32), ("act", ctypes.c_int32),
                ("X", ctypes.c_void_p), ("Wg", ctypes.c_void_p), ("Wu", ctypes.c_void_p),
                ("Wd", ctypes.c_void_p), ("bg", ctypes.c_void_p), ("bu", ctypes.c_void_p),
                ("bd", ctypes.c_void_p), ("ldx", ctypes.c_int64), ("ldwi", ctypes.c_int64),
                ("ldwd", ctypes.c_int64)]


class GatedGradsC(ctypes.Structure):
    _fields_ = [("dX", ctypes.c_void_p), ("dWg", ctypes.c_void_p), ("dWu", ctypes.c_void_p),
                ("dWd", ctypes.c_void_p), ("dbg", ctypes.c_void_p), ("dbu", ctypes.c_void_p),
                ("dbd", ctypes.c_void_p), ("lddx", ctypes.c_int64), ("lddwi", ctypes.c_int64),
                ("lddwd", ctypes.c_int64)]


class AdamwTensor(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("g", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("m_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("copy", ctypes.c_void_p), ("n", ctypes.c_int64),
                ("gt", ctypes.c_int32), ("decay", ctypes.c_float)]


class AdamwOpts(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("weight_decay", ctypes.c_double),
                ("grad_scale", ctypes.c_double), ("step", ctypes.c_int64),
                ("state_bits", ctypes.c_int32), ("rounding", ctypes.c_int32)]


_c_i64 = ctypes.c_int64
_c_p = ctypes.c_void_p
_LIB = None


def load(path: str = LIB_PATH):
    """Load the library (once) and declare the signatures."""
    global _LIB
    if _LIB is not None:
        return _LIB
    if not os.path.exists(path):
        raise FdError(2, f"{path} is not built; run __graft_entry__.build() or "
                         "python -m paper_2609_38198_amd.build")
    lib = ctypes.CDLL(path)
    lib.fd_lanczos_default_opts.argtypes = [ctypes.POINTER(LanczosOpts)]
    lib.fd_lanczos_default_opts.restype = None
    lib.fd_workspace_size.argtypes = [ctypes.c_int, _c_i64, _c_i64, _c_i64, _c_i64, _c_i64,
                                      ctypes.POINTER(LanczosOpts)]
    lib.fd_workspace_size.restype = ctypes.c_size_t
    lib.fd_kernel_matmul.argtypes = [_c_p, _c_i64, _c_p, _c_i64, _c_i64, _c_i64, ctypes.c_int,
                                     ctypes.c_float, _c_p, _c_p, _c_p, _c_i64, _c_i64, _c_p,
                                     _c_i64, _c_p, ctypes.c_size_t, _c_p]
    lib.fd_kernel_matmul.restype = ctypes.c_int
    lib.fd_kernel_matmul_noalloc.argtypes = [_c_p, _c_i64, _c_p, _c_i64, _c_i64, _c_i64,
                                             ctypes.c_int, ctypes.c_float, _c_p, _c_p, _c_p,
                                             _c_i64, _c_i64, _c_p, _c_i64, _c_p]
    lib.fd_kernel_matmul_noalloc.restype = ctypes.c_int
    lib.fd_kernel_matmul_noalloc_limit.argtypes = []
    lib.fd_kernel_matmul_noalloc_limit.restype = ctypes.c_size_t
    lib.fd_degree.argtypes = [_c_p, ctypes.c_int, _c_i64, _c_i64, _c_i64, ctypes.c_float,
                              ctypes.c_float, _c_p, _c_p, _c_p, _c_p, _c_p, ctypes.c_size_t, _c_p]
    lib.fd_degree.restype = ctypes.c_int
    lib.fd_degree_dyadic.argtypes = [_c_p, ctypes.c_int, _c_i64, _c_i64, _c_i64, ctypes.c_float,
                                     ctypes.c_int32, ctypes.c_float, _c_p, _c_p, _c_p, _c_p, _c_p,
                                     ctypes.c_size_t, _c_p]
    lib.fd_degree_dyadic.restype = ctypes.c_int
    lib.fd_block_lanczos.argtypes = [
        _c_p, ctypes.c_int, _c_i64, _c_i64, _c_i64, ctypes.c_float, ctypes.c_float, _c_i64, _c_i64,
        _c_p, _c_i64, _c_i64, ctypes.c_int32, ctypes.POINTER(LanczosOpts), _c_p, _c_p, _c_p, _c_p,
        ctypes.POINTER(LanczosInfo), _c_p, ctypes.c_size_t, _c_p]
    lib.fd_block_lanczos.restype = ctypes.c_int
    lib.fd_continuation.argtypes = [
        _c_p, ctypes.c_int, _c_i64, _c_i64, _c_i64, ctypes.c_float, _c_p, _c_p, _c_i64, _c_i64,
        _c_i64, _c_p, _c_i64, _c_i64, ctypes.POINTER(LanczosOpts), _c_p, _c_p, _c_p,
        ctypes.POINTER(LanczosInfo), ctypes.c_int32, _c_p, _c_p, ctypes.c_size_t, _c_p]
    lib.fd_continuation.restype = ctypes.c_int
    lib.fd_flow_default_opts.argtypes = [ctypes.POINTER(FlowOpts)]
    lib.fd_flow_default_opts.restype = None
    lib.fd_beta_flow.argtypes = [
        _c_p, ctypes.c_int, _c_i64, _c_i64, _c_i64, ctypes.c_float, _c_i64, _c_i64,
        ctypes.POINTER(FlowOpts), ctypes.POINTER(LanczosOpts), ctypes.POINTER(FlowProbe),
        ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_double),
        ctypes.POINTER(ctypes.c_int32), _c_p, _c_p, _c_p, _c_p, ctypes.c_size_t, _c_p]
    lib.fd_beta_flow.restype = ctypes.c_int
    lib.fd_beta_flow_cascade.argtypes = [
        ctypes.POINTER(_c_p), ctypes.POINTER(ctypes.c_int), ctypes.POINTER(ctypes.c_int64),
        ctypes.c_int32, _c_i64, _c_i64, ctypes.c_float, _c_i64, _c_i64,
        ctypes.POINTER(FlowOpts), ctypes.POINTER(LanczosOpts), ctypes.POINTER(FlowProbe),
        ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_double),
        ctypes.POINTER(ctypes.c_int32), _c_p, _c_p, _c_p, _c_p, ctypes.c_size_t, _c_p]
    lib.fd_beta_flow_cascade.restype = ctypes.c_int
    lib.fd_layer_norm.argtypes = [_c_p, ctypes.c_int, _c_i64, _c_i64, _c_i64, _c_p, _c_p,
                                  ctypes.c_int, ctypes.c_float, _c_p, _c_i64, _c_p, _c_p]
    lib.fd_layer_norm.restype = ctypes.c_int
    lib.fd_layer_norm_workspace_size.argtypes = [_c_i64, _c_i64]
    lib.fd_layer_norm_workspace_size.restype = ctypes.c_size_t
    lib.fd_layer_norm_backward.argtypes = [_c_p, _c_i64, _c_p, ctypes.c_int, _c_i64, _c_i64,
                                           _c_i64, _c_p, ctypes.c_int, _c_p, _c_p, _c_i64, _c_p,
                                           _c_i64, _c_p, _c_p, _c_p, ctypes.c_size_t, _c_p]
    lib.fd_layer_norm_backward.restype = ctypes.c_int
    lib.fd_gated_saved_size.argtypes = [ctypes.POINTER(GatedBlock)]
    lib.fd_gated_saved_size.restype = ctypes.c_size_t
    lib.fd_gated_workspace_size.argtypes = [ctypes.POINTER(GatedBlock), ctypes.c_int32]
    lib.fd_gated_workspace_size.restype = ctypes.c_size_t
    lib.fd_gated_forward.argtypes = [ctypes.POINTER(GatedBlock), _c_p, _c_i64, _c_p, _c_i64, _c_p,
                                     ctypes.c_size_t, _c_p, ctypes.c_size_t, _c_p]
    lib.fd_gated_forward.restype = ctypes.c_int
    lib.fd_gated_backward.argtypes = [ctypes.POINTER(GatedBlock), _c_p, _c_i64, _c_p,
                                      ctypes.c_size_t, ctypes.POINTER(GatedGradsC), _c_p,
                                      ctypes.c_size_t, _c_p]
    lib.fd_gated_backward.restype = ctypes.c_int
    lib.fd_adamw_default_opts.argtypes = [ctypes.POINTER(AdamwOpts)]
    lib.fd_adamw_default_opts.restype = None
    lib.fd_adamw_step.argtypes = [ctypes.POINTER(AdamwTensor), _c_i64, ctypes.POINTER(AdamwOpts),
                                  _c_p]
    lib.fd_adamw_step.restype = ctypes.c_int
    lib.fd_last_error.argtypes = []
    lib.fd_last_error.restype = ctypes.c_char_p
    lib.fd_status_string.argtypes = [ctypes.c_int]
    lib.fd_status_string.restype = ctypes.c_char_p
    lib.fd_profile_enable.argtypes = [ctypes.c_int32]
    lib.fd_profile_enable.restype = None
    lib.fd_profile_read.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_double),
                                    ctypes.POINTER(ctypes.c_int64)]
    lib.fd_profile_read.restype = ctypes.c_int
    _LIB = lib
    return lib


def _check(status: int, allow=(FD_OK,)) -> int:
    if status not in allow:
        raise FdError(status, load().fd_last_error().decode())
    return status


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(device: torch.device):
    return ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)


def _dtype_code(X: torch.Tensor) -> int:
    if X.dtype == torch.float32:
        return FD_F32
    if X.dtype in (torch.bfloat16, torch.int16, torch.uint16):
        return FD_BF16
    raise TypeError(f"X must be float32 or bfloat16, got {X.dtype}")


def _check_dev(*ts):
    """All tensors on one GPU (the workspace too: kernels write through its address)."""
    ts = [t for t in ts if t is not None]
    if any(not t.is_cuda for t in ts):
        raise ValueError("all tensors must live on the GPU")
    if len({t.get_device() for t in ts}) > 1:
        raise ValueError("all tensors must live on the same GPU")


def _workspace(nbytes: int, device) -> torch.Tensor:
    # torch's caching allocator returns 256-byte aligned blocks
    return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device)


def fd_profile_enable(on: bool = True) -> None:
    load().fd_profile_enable(int(bool(on)))


def fd_profile_read(kind: int) -> "tuple[float, int]":
    """(summed kernel milliseconds, timed launches) of one kernel kind; clears it."""
    ms = ctypes.c_double(0.0)
    n = ctypes.c_int64(0)
    _check(load().fd_profile_read(kind, ctypes.byref(ms), ctypes.byref(n)))
    return ms.value, n.value


def default_opts(**kw) -> LanczosOpts:
    o = LanczosOpts()
    load().fd_lanczos_default_opts(ctypes.byref(o))
    for k, v in kw.items():
        if not hasattr(o, k):
            raise AttributeError(k)
        setattr(o, k, v)
    return o


def fd_workspace_size(op: int, Nr: int, Nc: int, D: int, b: int = 1, k: int = 1,
                      opts: Optional[LanczosOpts] = None) -> int:
    return int(load().fd_workspace_size(op, Nr, Nc, D, b, k,
                                        None if opts is None else ctypes.byref(opts)))


def fd_kernel_matmul(Xr: torch.Tensor, Xc: Optional[torch.Tensor], beta: float, V: torch.Tensor,
                     sl: Optional[torch.Tensor] = None, sr: Optional[torch.Tensor] = None,
                     Y: Optional[torch.Tensor] = None,
                     ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Y = diag(sl) K(Xr, Xc) diag(sr) V (Xc = None: the square product on Xr)."""
    lib = load()
    if Xc is None:
        Xc = Xr
    _check_dev(Xr, Xc, V, sl, sr, Y, ws)
    if Xr.dim() != 2 or Xc.dim() != 2 or Xr.shape[1] != Xc.shape[1]:
        raise ValueError("Xr and Xc must be N x D with the same D")
    if Xr.stride(1) != 1 or Xc.stride(1) != 1 or Xr.stride(0) != Xc.stride(0):
        raise ValueError("Xr and Xc must be row-major with the same leading dimension")
    V2 = V.unsqueeze(1) if V.dim() == 1 else V
    if V2.dtype != torch.float32 or V2.stride(1) != 1:
        raise ValueError("V must be float32 row-major")
    Nr, D = Xr.shape
    Nc = Xc.shape[0]
    b = V2.shape[1]
    if V2.shape[0] != Nc:
        raise ValueError("V must have Nc rows")
    if Y is None:
        Y = torch.empty((Nr, b), dtype=torch.float32, device=Xr.device)
    Y2 = Y.unsqueeze(1) if Y.dim() == 1 else Y
    for t, n in ((sl, Nr), (sr, Nc)):
        if t is not None and (t.dtype != torch.float32 or t.numel() != n or not t.is_contiguous()):
            raise ValueError("sl / sr must be contiguous float32 vectors of matching length")
    need = fd_workspace_size(FD_OP_KERNEL_MATMUL, Nr, Nc, D, b)
    if need == 0:
        raise FdError(1, "unsupported sizes")
    if ws is None or ws.numel() < need:
        ws = _workspace(need, Xr.device)
    _check(lib.fd_kernel_matmul(_ptr(Xr), Nr, _ptr(Xc), Nc, D, Xr.stride(0), _dtype_code(Xr),
                                float(beta), _ptr(sl), _ptr(sr), _ptr(V2), b, V2.stride(0),
                                _ptr(Y2), Y2.stride(0), _ptr(ws), ws.numel(),
                                _stream(Xr.device)))
    return Y


def fd_kernel_matmul_noalloc(Xr: torch.Tensor, Xc: Optional[torch.Tensor], beta: float,
                             V: torch.Tensor, Y: torch.Tensor,
                             sl: Optional[torch.Tensor] = None,
                             sr: Optional[torch.Tensor] = None) -> torch.Tensor:
    """fd_kernel_matmul into a caller-provided Y, using the library's built-in
    scratch instead of a workspace (the call allocates nothing)."""
    lib = load()
    if Xc is None:
        Xc = Xr
    _check_dev(Xr, Xc, V, sl, sr, Y)
    if Xr.dim() != 2 or Xc.dim() != 2 or Xr.shape[1] != Xc.shape[1]:
        raise ValueError("Xr and Xc must be N x D with the same D")
    if Xr.stride(1) != 1 or Xc.stride(1) != 1 or Xr.stride(0) != Xc.stride(0):
        raise ValueError("Xr and Xc must be row-major with the same leading dimension")
    if V.dim() != 2 or Y.dim() != 2 or V.stride(1) != 1 or Y.stride(1) != 1:
        raise ValueError("V and Y must be row-major N x b")
    if V.dtype != torch.float32 or Y.dtype != torch.float32:
        raise ValueError("V and Y must be float32")
    Nr, D = Xr.shape
    Nc, b = Xc.shape[0], V.shape[1]
    if V.shape[0] != Nc or Y.shape[0] != Nr or Y.shape[1] != b:
        raise ValueError("V must be Nc x b and Y Nr x b")
    for t, n in ((sl, Nr), (sr, Nc)):
        if t is not None and (t.dtype != torch.float32 or t.numel() != n or not t.is_contiguous()):
            raise ValueError("sl / sr must be contiguous float32 vectors of matching length")
    _check(lib.fd_kernel_matmul_noalloc(_ptr(Xr), Nr, _ptr(Xc), Nc, D, Xr.stride(0),
                                        _dtype_code(Xr), float(beta), _ptr(sl), _ptr(sr),
                                        _ptr(V), b, V.stride(0), _ptr(Y), Y.stride(0),
                                        _stream(Xr.device)))
    return Y


def fd_kernel_matmul_noalloc_limit() -> int:
    return int(load().fd_kernel_matmul_noalloc_limit())


@dataclass
class Degree:
    q: torch.Tensor
    d: torch.Tensor
    s: torch.Tensor
    s_off: torch.Tensor   # one float64 on the device


def fd_degree(X: torch.Tensor, beta: float, alpha: float = 0.5,
              ws: Optional[torch.Tensor] = None) -> Degree:
    """q = K 1, d = w (K w) with w = q^-alpha, s = w d^-1/2, S_off = sum(q) - N."""
    lib = load()
    _check_dev(X, ws)
    if X.dim() != 2 or X.stride(1) != 1:
        raise ValueError("X must be row-major N x D")
    N, D = X.shape
    dev = X.device
    q = torch.empty(N, dtype=torch.float32, device=dev)
    d = torch.empty_like(q)
    s = torch.empty_like(q)
    s_off = torch.empty(1, dtype=torch.float64, device=dev)
    need = fd_workspace_size(FD_OP_DEGREE, N, N, D)
    if need == 0:
        raise FdError(1, "unsupported sizes")
    if ws is None or ws.numel() < need:
        ws = _workspace(need, dev)
    _check(lib.fd_degree(_ptr(X), _dtype_code(X), N, D, X.stride(0), float(beta), float(alpha),
                         _ptr(q), _ptr(d), _ptr(s), _ptr(s_off), _ptr(ws), ws.numel(),
                         _stream(dev)))
    return Degree(q, d, s, s_off)


def fd_degree_dyadic(X: torch.Tensor, beta0: float, nbeta: int, alpha: float = 0.5,
                     ws: Optional[torch.Tensor] = None) -> Degree:
    """fd_degree at beta0 * 2^l for l < nbeta: q, d, s are nbeta x N, s_off nbeta."""
    lib = load()
    _check_dev(X, ws)
    if X.dim() != 2 or X.stride(1) != 1:
        raise ValueError("X must be row-major N x D")
    N, D = X.shape
    dev = X.device
    q = torch.empty((nbeta, N), dtype=torch.float32, device=dev)
    d = torch.empty_like(q)
    s = torch.empty_like(q)
    s_off = torch.empty(nbeta, dtype=torch.float64, device=dev)
    need = fd_workspace_size(FD_OP_DEGREE_DYADIC, N, N, D)
    if need == 0:
        raise FdError(1, "unsupported sizes")
    if ws is None or ws.numel() < need:
        ws = _workspace(need, dev)
    _check(lib.fd_degree_dyadic(_ptr(X), _dtype_code(X), N, D, X.stride(0), float(beta0),
                                int(nbeta), float(alpha), _ptr(q), _ptr(d), _ptr(s),
                                _ptr(s_off), _ptr(ws), ws.numel(), _stream(dev)))
    return Degree(q, d, s, s_off)


@dataclass
class Eigen:
    evals: "list[float]"
    evecs: torch.Tensor
    psi: Optional[torch.Tensor]
    residuals: "list[float]"
    info: dict
    status: int


def fd_block_lanczos(X: torch.Tensor, beta: float, k: int, b: int, alpha: float = 0.5,
                     V0: Optional[torch.Tensor] = None, warm_is_psi: bool = True,
                     opts: Optional[LanczosOpts] = None, want_psi: bool = True,
                     ws: Optional[torch.Tensor] = None, allow_not_converged: bool = False) -> Eigen:
    """Top-k eigenpairs of M = diag(s) K diag(s) (Perron pair included)."""
    lib = load()
    _check_dev(X, V0, ws)
    N, D = X.shape
    dev = X.device
    o = opts if opts is not None else default_opts()
    evals = (ctypes.c_double * k)()
    res = (ctypes.c_double * k)()
    info = LanczosInfo()
    evecs = torch.empty((N, k), dtype=torch.float32, device=dev)
    psi = torch.empty((N, k), dtype=torch.float32, device=dev) if want_psi else None
    k0 = 0 if V0 is None else V0.shape[1]
    ldv0 = 0 if V0 is None else V0.stride(0)
    need = fd_workspace_size(FD_OP_BLOCK_LANCZOS, N, N, D, b, k, o)
    if need == 0:
        raise FdError(1, "unsupported sizes")
    if ws is None or ws.numel() < need:
        ws = _workspace(need, dev)
    allow = (FD_OK, 5) if allow_not_converged else (FD_OK,)
    st = _check(lib.fd_block_lanczos(_ptr(X), _dtype_code(X), N, D, X.stride(0), float(beta),
                                     float(alpha), b, k, _ptr(V0), k0, ldv0, int(warm_is_psi),
                                     ctypes.byref(o), evals, _ptr(evecs), _ptr(psi), res,
                                     ctypes.byref(info), _ptr(ws), ws.numel(), _stream(dev)),
                allow)
    return Eigen(list(evals), evecs, psi, list(res), info.as_dict(), st)


@dataclass
class Ladder:
    evals: "list[list[float]]"
    evecs: torch.Tensor
    psi: Optional[torch.Tensor]
    info: "list[dict]"
    steps_done: int
    status: int


def fd_continuation(X: torch.Tensor, n_steps: Sequence[int], beta_steps: Sequence[float], k: int,
                    b: int, alpha: float = 0.5, V0: Optional[torch.Tensor] = None,
                    opts: Optional[LanczosOpts] = None, stop_at_wall: bool = False,
                    want_psi: bool = True, ws: Optional[torch.Tensor] = None,
                    allow=(FD_OK,)) -> Ladder:
    """Warm-started ladder over prefixes X[:n_t] and bandwidths beta_t."""
    lib = load()
    _check_dev(X, V0, ws)
    N, D = X.shape
    dev = X.device
    T = len(n_steps)
    if T != len(beta_steps) or T == 0:
        raise ValueError("n_steps and beta_steps must have the same non-zero length")
    o = opts if opts is not None else default_opts()
    ns = (ctypes.c_int64 * T)(*[int(n) for n in n_steps])
    bs = (ctypes.c_float * T)(*[float(x) for x in beta_steps])
    evals = (ctypes.c_double * (T * k))()
    infos = (LanczosInfo * T)()
    nlast = int(n_steps[-1])
    evecs = torch.empty((nlast, k), dtype=torch.float32, device=dev)
    psi = torch.empty((nlast, k), dtype=torch.float32, device=dev) if want_psi else None
    done = ctypes.c_int64(0)
    k0 = 0 if V0 is None else V0.shape[1]
    ldv0 = 0 if V0 is None else V0.stride(0)
    need = fd_workspace_size(FD_OP_CONTINUATION, max(int(n) for n in n_steps), T, D, b, k, o)
    if need == 0:
        raise FdError(1, "unsupported sizes")
    if ws is None or ws.numel() < need:
        ws = _workspace(need, dev)
    st = _check(lib.fd_continuation(_ptr(X), _dtype_code(X), N, D, X.stride(0), float(alpha), ns, bs,
                                    T, b, k, _ptr(V0), k0, ldv0, ctypes.byref(o), evals,
                                    _ptr(evecs), _ptr(psi), infos, int(stop_at_wall),
                                    ctypes.byref(done), _ptr(ws), ws.numel(), _stream(dev)),
                allow)
    ev = [[evals[t * k + i] for i in range(k)] for t in range(T)]
    return Ladder(ev, evecs, psi, [infos[t].as_dict() for t in range(T)], done.value, st)


def flow_default_opts(**kw) -> FlowOpts:
    o = FlowOpts()
    load().fd_flow_default_opts(ctypes.byref(o))
    for key, v in kw.items():
        setattr(o, key, v)
    return o


@dataclass
class Flow:
    probes: list       # per-probe records (dicts), in the order run
    beta_x: float      # achieved bandwidth
    reason: str        # "bracket", "wall", "budget" or "range"
    evals: list
    evecs: torch.Tensor
    psi: Optional[torch.Tensor]
    status: int


def fd_beta_flow(X: torch.Tensor, k: int, b: int, alpha: float = 0.5,
                 fopts: Optional[FlowOpts] = None, opts: Optional[LanczosOpts] = None,
                 want_psi: bool = True, ws: Optional[torch.Tensor] = None,
                 allow=(FD_OK,)) -> Flow:
    """Bandwidth selection by the beta-function flow; eigenpairs at beta_x."""
    lib = load()
    _check_dev(X, ws)
    N, D = X.shape
    dev = X.device
    fo = fopts if fopts is not None else flow_default_opts()
    o = opts if opts is not None else default_opts()
    cap = int(fo.max_probes) + 2
    recs = (FlowProbe * cap)()
    nrec = ctypes.c_int64(0)
    bx = ctypes.c_double(0.0)
    why = ctypes.c_int32(0)
    evals = (ctypes.c_double * k)()
    evecs = torch.empty((N, k), dtype=torch.float32, device=dev)
    psi = torch.empty((N, k), dtype=torch.float32, device=dev) if want_psi else None
    need = fd_workspace_size(FD_OP_BETA_FLOW, N, N, D, b, k, o)
    if need == 0:
        raise FdError(1, "unsupported sizes")
    if ws is None or ws.numel() < need:
        ws = _workspace(need, dev)
    st = _check(lib.fd_beta_flow(_ptr(X), _dtype_code(X), N, D, X.stride(0), float(alpha), b, k,
                                 ctypes.byref(fo), ctypes.byref(o), recs, ctypes.byref(nrec),
                                 ctypes.byref(bx), ctypes.byref(why), evals, _ptr(evecs),
                                 _ptr(psi), _ptr(ws), ws.numel(), _stream(dev)), allow)
    return Flow([recs[i].as_dict() for i in range(nrec.value)], bx.value,
                FLOW_EXIT.get(why.value, str(why.value)), [evals[i] for i in range(k)], evecs,
                psi, st)


def fd_beta_flow_cascade(Xs: Sequence[torch.Tensor], k: int, b: int, alpha: float = 0.5,
                         fopts: Optional[FlowOpts] = None, opts: Optional[LanczosOpts] = None,
                         want_psi: bool = True, ws: Optional[torch.Tensor] = None,
                         allow=(FD_OK,)) -> Flow:
    """Precision cascade of the flow: the same points in each dtype of Xs, lowest first."""
    lib = load()
    Xs = list(Xs)
    if not 1 <= len(Xs) <= 4:
        raise ValueError("the cascade takes 1 to 4 levels")
    _check_dev(*Xs, ws)
    for X in Xs:
        if X.dim() != 2 or X.stride(1) != 1 or X.shape != Xs[0].shape:
            raise ValueError("every level must be the same row-major N x D points")
    N, D = Xs[0].shape
    dev = Xs[0].device
    fo = fopts if fopts is not None else flow_default_opts()
    o = opts if opts is not None else default_opts()
    cap = len(Xs) * (int(fo.max_probes) + 2)
    recs = (FlowProbe * cap)()
    nrec = ctypes.c_int64(0)
    bx = ctypes.c_double(0.0)
    why = ctypes.c_int32(0)
    evals = (ctypes.c_double * k)()
    evecs = torch.empty((N, k), dtype=torch.float32, device=dev)
    psi = torch.empty((N, k), dtype=torch.float32, device=dev) if want_psi else None
    need = fd_workspace_size(FD_OP_BETA_FLOW, N, N, D, b, k, o)
    if need == 0:
        raise FdError(1, "unsupported sizes")
    if ws is None or ws.numel() < need:
        ws = _workspace(need, dev)
    ptrs = (_c_p * len(Xs))(*[X.data_ptr() for X in Xs])
    codes = (ctypes.c_int * len(Xs))(*[_dtype_code(X) for X in Xs])
    lds = (ctypes.c_int64 * len(Xs))(*[X.stride(0) for X in Xs])
    st = _check(lib.fd_beta_flow_cascade(ptrs, codes, lds, len(Xs), N, D, float(alpha), b, k,
                                         ctypes.byref(fo), ctypes.byref(o), recs,
                                         ctypes.byref(nrec), ctypes.byref(bx), ctypes.byref(why),
                                         evals, _ptr(evecs), _ptr(psi), _ptr(ws), ws.numel(),
                                         _stream(dev)), allow)
    return Flow([recs[i].as_dict() for i in range(nrec.value)], bx.value,
                FLOW_EXIT.get(why.value, str(why.value)), [evals[i] for i in range(k)], evecs,
                psi, st)


# ---- a parametric extension of the coordinates ----


def _net_code(dtype: torch.dtype, what: str) -> int:
    if dtype == torch.float32:
        return FD_F32
    if dtype == torch.bfloat16:
        return FD_BF16
    raise TypeError(f"{what} must be float32 or bfloat16, got {dtype}")


def _net_dtype(t: torch.Tensor, what: str) -> int:
    return _net_code(t.dtype, what)


def _net_device(X: torch.Tensor) -> int:
    if not X.is_cuda:
        raise ValueError("all tensors must live on the GPU")
    return X.get_device()


def _net_place(t: torch.Tensor, dev: int, what: str) -> None:
    if t.get_device() != dev:
        raise ValueError(f"{what} must live on the GPU of the other tensors")


def _net_matrix(t: torch.Tensor, rows: int, cols: int, dtype: torch.dtype, dev: int,
                what: str) -> int:
    """The leading dimension of a row-major rows x cols matrix."""
    _net_place(t, dev, what)
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != cols:
        raise ValueError(f"{what} must be {rows} x {cols}, got {tuple(t.shape)}")
    if t.dtype != dtype:
        raise TypeError(f"{what} must be {dtype}, got {t.dtype}")
    ld, one = t.stride()
    if one != 1 and cols > 1:
        raise ValueError(f"{what} must be row-major")
    if rows > 1:
        if ld < cols:
            raise ValueError(f"{what} has overlapping rows")
        return ld
    return cols  # of one row whatever its stride says


def _net_vector(t: Optional[torch.Tensor], n: int, dtype: torch.dtype, dev: int, what: str):
    if t is None:
        return None
    _net_place(t, dev, what)
    if t.dim() != 1 or t.shape[0] != n or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{what} must be {n} contiguous values of {dtype}")
    return t.data_ptr()


def _net_workspace(ws: Optional[torch.Tensor], need: int, like: torch.Tensor) -> torch.Tensor:
    if ws is not None:
        _net_room(ws, like.get_device(), "ws")
        if ws.numel() * ws.element_size() >= need:
            return ws
    return like.new_empty(max(need, 1), dtype=torch.uint8)


def _net_room(t: torch.Tensor, dev: int, what: str) -> None:
    """A buffer that the kernels address by its start and its bytes."""
    _net_place(t, dev, what)
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")


def _net_stream(dev: int) -> int:
    # the current stream's handle without building a torch.cuda.Stream, which
    # takes 2 us of a call's 12
    return torch._C._cuda_getCurrentRawStream(dev)


def fd_layer_norm(X: torch.Tensor, gamma: Optional[torch.Tensor] = None,
                  beta: Optional[torch.Tensor] = None, eps: float = 1e-5,
                  Y: Optional[torch.Tensor] = None, stats: Optional[torch.Tensor] = None
                  ) -> "tuple[torch.Tensor, torch.Tensor]":
    """(Y, stats): (x - mean) rstd gamma + beta of each row of X, and its (mean, rstd).
    The results have no autograd history (nor have those of the calls below)."""
    lib = load()
    if X.dim() != 2:
        raise ValueError("X must be N x D")
    N, D = X.shape
    xt = _net_dtype(X, "X")
    dev = _net_device(X)
    ldx = _net_matrix(X, N, D, X.dtype, dev, "X")
    w = gamma if gamma is not None else beta
    wdtype = X.dtype if w is None else w.dtype
    wt = xt if w is None else _net_dtype(w, "gamma and beta")
    pg = _net_vector(gamma, D, wdtype, dev, "gamma")
    pb = _net_vector(beta, D, wdtype, dev, "beta")
    if Y is None:
        Y = X.new_empty((N, D))
    if stats is None:
        stats = X.new_empty((N, 2), dtype=torch.float32)
    _net_matrix(stats, N, 2, torch.float32, dev, "stats")
    if not stats.is_contiguous():
        raise ValueError("stats must be contiguous")
    ldy = _net_matrix(Y, N, D, X.dtype, dev, "Y")
    _check(lib.fd_layer_norm(X.data_ptr(), xt, N, D, ldx, pg, pb, wt, eps, Y.data_ptr(), ldy,
                             stats.data_ptr(), _net_stream(dev)))
    return Y, stats


@dataclass
class LayerNormGrads:
    dX: torch.Tensor
    dgamma: Optional[torch.Tensor]
    dbeta: Optional[torch.Tensor]


def fd_layer_norm_backward(dY: torch.Tensor, X: torch.Tensor, gamma: Optional[torch.Tensor],
                           stats: torch.Tensor, add: Optional[torch.Tensor] = None,
                           weight_grads: bool = True, dX: Optional[torch.Tensor] = None,
                           dgamma: Optional[torch.Tensor] = None,
                           dbeta: Optional[torch.Tensor] = None,
                           ws: Optional[torch.Tensor] = None,
                           wdtype: Optional[torch.dtype] = None) -> LayerNormGrads:
    """Gradients of fd_layer_norm, into dX, dgamma and dbeta where given; `add`, a
    residual branch's gradient, is added to dX.  dgamma and dbeta have gamma's type; without
    gamma, that of the array given for one of them, or wdtype, or X's."""
    lib = load()
    if X.dim() != 2:
        raise ValueError("X must be N x D")
    N, D = X.shape
    xt = _net_dtype(X, "X")
    dev = _net_device(X)
    ldx = _net_matrix(X, N, D, X.dtype, dev, "X")
    lddy = _net_matrix(dY, N, D, X.dtype, dev, "dY")
    ldadd = 0 if add is None else _net_matrix(add, N, D, X.dtype, dev, "add")
    given = [w.dtype for w in (gamma, dgamma, dbeta) if w is not None]
    if wdtype is None:
        wdtype = given[0] if given else X.dtype
    wt = _net_code(wdtype, "gamma, dgamma and dbeta")
    pg = _net_vector(gamma, D, wdtype, dev, "gamma")
    _net_matrix(stats, N, 2, torch.float32, dev, "stats")
    if not stats.is_contiguous():
        raise ValueError("stats must be contiguous")
    if dX is None:
        dX = X.new_empty((N, D))
    lddx = _net_matrix(dX, N, D, X.dtype, dev, "dX")
    if weight_grads:
        dgamma = X.new_empty(D, dtype=wdtype) if dgamma is None else dgamma
        dbeta = X.new_empty(D, dtype=wdtype) if dbeta is None else dbeta
    pdg = _net_vector(dgamma, D, wdtype, dev, "dgamma")
    pdb = _net_vector(dbeta, D, wdtype, dev, "dbeta")
    ws = _net_workspace(ws, lib.fd_layer_norm_workspace_size(N, D), X)
    _check(lib.fd_layer_norm_backward(
        dY.data_ptr(), lddy, X.data_ptr(), xt, N, D, ldx, pg, wt, stats.data_ptr(),
        None if add is None else add.data_ptr(), ldadd, dX.data_ptr(), lddx,
        pdg, pdb, ws.data_ptr(), ws.numel() * ws.element_size(), _net_stream(dev)))
    return LayerNormGrads(dX, dgamma, dbeta)


def _gated_block(X, Wg, Wu, Wd, bg, bu, bd, act, fine=False) -> GatedBlock:
    if X.dim() != 2 or Wg.dim() != 2 or Wd.dim() != 2:
        raise ValueError("X, Wg, Wu and Wd must be matrices")
    if act not in FD_ACT:
        raise ValueError(f"act must be one of {sorted(FD_ACT)}, got {act!r}")
    N, D = X.shape
    F, O = Wg.shape[0], Wd.shape[0]
    t = X.dtype
    code = _net_dtype(X, "X")
    dev = _net_device(X)
    ldx = _net_matrix(X, N, D, t, dev, "X")
    ldwi = _net_matrix(Wg, F, D, t, dev, "Wg")
    if _net_matrix(Wu, F, D, t, dev, "Wu") != ldwi:
        raise ValueError("Wg and Wu must have the same leading dimension")
    ldwd = _net_matrix(Wd, O, F, t, dev, "Wd")
    return GatedBlock(N, D, F, O, code, FD_ACT[act] | (FD_GATED_FINE if fine else 0), X.data_ptr(), Wg.data_ptr(), Wu.data_ptr(),
                      Wd.data_ptr(), _net_vector(bg, F, t, dev, "bg"), _net_vector(bu, F, t, dev, "bu"),
                      _net_vector(bd, O, t, dev, "bd"), ldx, ldwi, ldwd)


def fd_gated_forward(X: torch.Tensor, Wg: torch.Tensor, Wu: torch.Tensor, Wd: torch.Tensor,
                     bg: Optional[torch.Tensor] = None, bu: Optional[torch.Tensor] = None,
                     bd: Optional[torch.Tensor] = None, R: Optional[torch.Tensor] = None,
                     act: str = "silu", save: bool = False, Y: Optional[torch.Tensor] = None,
                     ws: Optional[torch.Tensor] = None, fine: bool = False
                     ) -> "tuple[torch.Tensor, Optional[torch.Tensor]]":
    """(Y, saved): Y = (act(X Wg^T + bg) * (X Wu^T + bu)) Wd^T + bd [+ R];
    saved (with save) is what fd_gated_backward takes to spare computing the
    inner activations again.  fine: bfloat16 inner values are not rounded to one
    bfloat16, at any size."""
    lib = load()
    b = _gated_block(X, Wg, Wu, Wd, bg, bu, bd, act, fine)
    dev = X.get_device()
    if Y is None:
        Y = X.new_empty((b.N, b.O))
    ldy = _net_matrix(Y, b.N, b.O, X.dtype, dev, "Y")
    ldr = 0 if R is None else _net_matrix(R, b.N, b.O, X.dtype, dev, "R")
    saved, nsaved = None, 0
    if save:
        nsaved = lib.fd_gated_saved_size(b)
        saved = X.new_empty(max(nsaved, 1), dtype=torch.uint8)
    need = lib.fd_gated_workspace_size(b, 0)
    ws = _net_workspace(ws, need, X)
    _check(lib.fd_gated_forward(b, None if R is None else R.data_ptr(), ldr, Y.data_ptr(), ldy,
                                saved.data_ptr() if save else None, nsaved, ws.data_ptr(),
                                ws.numel() * ws.element_size(), _net_stream(dev)))
    return Y, saved


@dataclass
class GatedGrads:
    dX: Optional[torch.Tensor]
    dWg: torch.Tensor
    dWu: torch.Tensor
    dWd: torch.Tensor
    dbg: Optional[torch.Tensor]
    dbu: Optional[torch.Tensor]
    dbd: Optional[torch.Tensor]


def fd_gated_backward(dY: torch.Tensor, X: torch.Tensor, Wg: torch.Tensor, Wu: torch.Tensor,
                      Wd: torch.Tensor, bg: Optional[torch.Tensor] = None,
                      bu: Optional[torch.Tensor] = None, bd: Optional[torch.Tensor] = None,
                      act: str = "silu", saved: Optional[torch.Tensor] = None,
                      want_dx: bool = True, grads: Optional[GatedGrads] = None,
                      ws: Optional[torch.Tensor] = None, fine: bool = False) -> GatedGrads:
    """Gradients of fd_gated_forward (R's is dY itself), into `grads` where
    given; a bias has one where it was given.  fine: as in the forward pass, by itself."""
    lib = load()
    b = _gated_block(X, Wg, Wu, Wd, bg, bu, bd, act, fine)
    dev, t = X.get_device(), X.dtype
    lddy = _net_matrix(dY, b.N, b.O, t, dev, "dY")
    if grads is None:
        def like(x):
            return None if x is None else x.new_empty(x.shape)

        grads = GatedGrads(like(X) if want_dx else None, like(Wg), like(Wu), like(Wd), like(bg),
                           like(bu), like(bd))
    g = grads
    lddwi = _net_matrix(g.dWg, b.F, b.D, t, dev, "dWg")
    if _net_matrix(g.dWu, b.F, b.D, t, dev, "dWu") != lddwi:
        raise ValueError("dWg and dWu must have the same leading dimension")
    c = GatedGradsC(None if g.dX is None else g.dX.data_ptr(), g.dWg.data_ptr(),
                    g.dWu.data_ptr(), g.dWd.data_ptr(), _net_vector(g.dbg, b.F, t, dev, "dbg"),
                    _net_vector(g.dbu, b.F, t, dev, "dbu"), _net_vector(g.dbd, b.O, t, dev, "dbd"),
                    0 if g.dX is None else _net_matrix(g.dX, b.N, b.D, t, dev, "dX"), lddwi,
                    _net_matrix(g.dWd, b.O, b.F, t, dev, "dWd"))
    if saved is not None:
        _net_room(saved, dev, "saved")
    nsaved = 0 if saved is None else saved.numel() * saved.element_size()
    need = lib.fd_gated_workspace_size(b, 2 if saved is None else 1)
    ws = _net_workspace(ws, need, X)
    _check(lib.fd_gated_backward(b, dY.data_ptr(), lddy,
                                 None if saved is None else saved.data_ptr(), nsaved, c,
                                 ws.data_ptr(), ws.numel() * ws.element_size(), _net_stream(dev)))
    return grads


@dataclass
class AdamwState:
    """Moments, a tensor per parameter: float32 m and v; or, with scales,
    float8_e4m3fn m and v = the second moment's square root, and a float32 scale
    for each 256 elements."""
    m: "list[torch.Tensor]"
    v: "list[torch.Tensor]"
    m_scale: "Optional[list[torch.Tensor]]" = None
    v_scale: "Optional[list[torch.Tensor]]" = None


def fd_adamw_state(params: Sequence[torch.Tensor], bits: int = 32) -> AdamwState:
    """Cleared states for a first step."""
    if bits not in (32, 8):
        raise ValueError("bits must be 32 or 8")

    def zeros(dtype, per=1):
        return [torch.zeros(-(-p.numel() // per), dtype=dtype, device=p.device) for p in params]

    if bits == 32:
        return AdamwState(zeros(torch.float32), zeros(torch.float32))
    return AdamwState(zeros(torch.float8_e4m3fn), zeros(torch.float8_e4m3fn),
                      zeros(torch.float32, 256), zeros(torch.float32, 256))


@dataclass
class AdamwPlan:
    """The tensors of a step, checked once; it keeps them alive."""
    tensors: "list"
    table: "ctypes.Array"
    bits: int
    device: torch.device


def fd_adamw_plan(params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor],
                  state: AdamwState, copies: Optional[Sequence[torch.Tensor]] = None,
                  decay: Optional[Sequence[float]] = None) -> AdamwPlan:
    """Tensors that fd_adamw_step updates, by their addresses (gradients that moved take a
    new plan, 2.5 us a tensor): float32 params from float32 or bfloat16 grads, optionally
    bfloat16 copies of the params, and a multiplier of the weight decay for each (default 1)."""
    n = len(params)
    bits = 32 if state.m_scale is None else 8
    lists = [params, grads, state.m, state.v]
    lists += [] if bits == 32 else [state.m_scale, state.v_scale]
    lists += [] if copies is None else [copies]
    if any(len(x) != n for x in lists) or (decay is not None and len(decay) != n):
        raise ValueError("one tensor for each parameter is wanted")
    moment = torch.float32 if bits == 32 else torch.float8_e4m3fn
    dev = _net_device(params[0]) if n else -1
    table = (AdamwTensor * n)()
    for i, p in enumerate(params):
        size = p.numel()

        def at(t, dtypes, what, count=size):
            _net_place(t, dev, f"{what} of tensor {i}")
            if t.numel() != count or t.dtype not in dtypes or not t.is_contiguous():
                raise ValueError(f"{what} of tensor {i} must be {count} contiguous values of "
                                 f"{' or '.join(map(str, dtypes))}")
            return t.data_ptr()

        blocks = -(-size // 256)
        table[i] = AdamwTensor(
            at(p, (torch.float32,), "the parameters"),
            at(grads[i], (torch.float32, torch.bfloat16), "the gradient"),
            at(state.m[i], (moment,), "m"), at(state.v[i], (moment,), "v"),
            None if bits == 32 else at(state.m_scale[i], (torch.float32,), "m_scale", blocks),
            None if bits == 32 else at(state.v_scale[i], (torch.float32,), "v_scale", blocks),
            None if copies is None else at(copies[i], (torch.bfloat16,), "the copy"), size,
            FD_F32 if grads[i].dtype == torch.float32 else FD_BF16,
            1.0 if decay is None else decay[i])
    device = params[0].device if n else torch.device("cuda", torch.cuda.current_device())
    return AdamwPlan([list(x) for x in lists], table, bits, device)


def fd_adamw_step(plan: AdamwPlan, step: int, lr: float = 1e-3, beta1: float = 0.9,
                  beta2: float = 0.999, eps: float = 1e-8, weight_decay: float = 0.01,
                  grad_scale: float = 1.0, rounding: str = "nearest") -> None:
    """One AdamW step over the plan's tensors, in place; `step` counts from 1.

    rounding, of 8-bit states: "nearest", or "unbiased" by a fixed hash of step and
    element, with which the moments follow their formulas over many steps (rounded to
    nearest, the second moment hardly moves)."""
    if rounding not in FD_ROUNDING:
        raise ValueError(f"rounding must be one of {sorted(FD_ROUNDING)}, got {rounding!r}")
    o = AdamwOpts(lr, beta1, beta2, eps, weight_decay, grad_scale, step, plan.bits,
                  FD_ROUNDING[rounding])
    _check(load().fd_adamw_step(plan.table, len(plan.table), o, _net_stream(plan.device.index)))
