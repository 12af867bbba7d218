"""Thin Python binding of the microscaled 4-bit operators (include/ozimmu_mx.h): quantisation, reading back, product, and a
linear layer with its gradient.

Argument marshalling only: device pointers of torch tensors and the current HIP stream go to the entry points of the same name.
There is no CPU fallback.  Matrices are 2-D tensors with unit stride along their rows, in float32, bfloat16 or float16; results that
are not handed over are allocated, workspaces too.  All tensors of a call have to be on the current device (torch.cuda.device), whose
current stream it goes to.

No operations are recorded for torch's autograd: linear_backward is called by the user, in torch.no_grad() or in the backward of a
torch.autograd.Function.  linear and linear_backward refuse a tensor that requires a gradient while torch records.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

from . import ozimmu
from .ozimmu import OzimmuError

_lib = ozimmu._lib
_i64, _int, _vp, _sz, _float = ctypes.c_int64, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float

_SIGNATURES = {
    "ozimmu_mx_bytes": (_sz, [_i64, _i64]),
    "ozimmu_mx_quantize": (_int, [_int, _i64, _i64, _vp, _i64, _vp, _vp, _vp]),
    "ozimmu_mx_dequantize": (_int, [_int, _i64, _i64, _vp, _vp, _i64, _vp]),
    "ozimmu_mx_pack": (_int, [_i64, _i64, _vp, _i64, _vp, _i64, _vp, _vp]),
    "ozimmu_mx_unpack": (_int, [_i64, _i64, _vp, _vp, _i64, _vp, _i64, _vp]),
    "ozimmu_mx_workspace_bytes": (_sz, [_i64, _i64, _i64]),
    "ozimmu_mx_backward_workspace_bytes": (_sz, [_i64, _i64, _i64]),
    "ozimmu_mx_gemm": (_int, [_i64, _i64, _i64, _float, _vp, _vp, _float, _int, _vp, _i64, _vp]),
    "ozimmu_mx_gemm_way": (_int, [_int, _i64, _i64, _i64, _float, _vp, _vp, _float, _int, _vp, _i64, _vp]),
    "ozimmu_mx_choose": (_int, [_i64, _i64, _i64, _i64]),
    "ozimmu_mx_linear": (_int, [_i64, _i64, _i64, _float, _int, _vp, _i64, _vp, _float, _int, _vp, _i64, _vp, _sz, _vp]),
    "ozimmu_mx_linear_backward": (_int, [_i64, _i64, _i64, _float, _int, _vp, _i64, _vp, _i64, _vp, _float, _int, _vp, _i64,
                                         _float, _int, _vp, _i64, _vp, _sz, _vp]),
}
for _name, (_restype, _argtypes) in _SIGNATURES.items():
    getattr(_lib, _name).restype, getattr(_lib, _name).argtypes = _restype, _argtypes
EXPORTS = list(_SIGNATURES)

TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
BLOCK = 32
FEW_ROWS = 16  # up to here a layer takes no workspace, whatever its sizes (asking the library for it is a quarter of a microsecond)
WAYS = {"auto": -1, "direct": 0, "tile": 1, "half": 2}
_uint8 = torch.uint8
_several_devices = torch.cuda.device_count() > 1  # (where there is one, there is nothing to tell apart)


def _on_current_device(t) -> None:
    device = getattr(t, "device", None)
    if device is not None and device.index != ozimmu._current_device():
        raise ValueError(f"tensor on {device}, while the current device is cuda:{ozimmu._current_device()}")


def _not_recorded(t, what: str) -> None:
    if getattr(t, "requires_grad", False) and torch.is_grad_enabled():
        raise ValueError(f"{what} requires a gradient, which the result would not carry: call this in torch.no_grad() or a torch.autograd.Function")


class Packed:
    """A matrix of rows x n in the packed form: `data` holds its bytes (on the GPU, private layout; see pack and unpack)."""
    __slots__ = ("data", "rows", "n")

    def __init__(self, data: torch.Tensor, rows: int, n: int):
        if not (data.is_cuda and data.dtype is _uint8 and data.dim() == 1 and data.is_contiguous()):
            raise ValueError("packed data is a contiguous 1-D uint8 tensor on the GPU")
        if data.numel() < packed_bytes(rows, n):
            raise ValueError(f"{data.numel()} bytes for a packed matrix of {rows} x {n}, which takes {packed_bytes(rows, n)}")
        self.data, self.rows, self.n = data, rows, n

    @property
    def shape(self) -> Tuple[int, int]:
        return self.rows, self.n


def _matrix(t: torch.Tensor) -> Tuple[int, int, int, int]:
    """Rows, columns, leading dimension and type number of a matrix on the GPU."""
    kind = TYPES.get(t.dtype)
    if kind is None:
        raise ValueError(f"expected float32, bfloat16 or float16, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError("tensor must live on the GPU")
    if _several_devices:
        _on_current_device(t)
    shape = t.shape
    if len(shape) != 2:
        raise ValueError("expected a 2-D tensor")
    rows, cols = shape
    ld, unit = t.stride()
    if (cols > 1 and unit != 1) or (rows > 1 and ld < cols):
        raise ValueError("expected a 2-D tensor with unit stride along rows that do not overlap")
    return rows, cols, ld if rows > 1 else max(cols, ld, 1), kind


def _output(D: Optional[torch.Tensor], like: torch.Tensor, rows: int, cols: int, dtype, usual, beta: float):
    """The caller's output, or a new one, of type `dtype` (None: the caller's, or `usual`); its leading dimension and type number."""
    if D is None:
        if beta != 0.0:
            raise ValueError("beta without the matrix that it multiplies")
        dtype = dtype or usual
        kind = TYPES.get(dtype)
        if kind is None:
            raise ValueError(f"expected float32, bfloat16 or float16, got {dtype}")
        return like.new_empty((rows, cols), dtype=dtype), max(cols, 1), kind
    m, n, ldd, kind = _matrix(D)
    if dtype is not None and dtype is not D.dtype:
        raise ValueError(f"output of {D.dtype} for a result of {dtype}")
    if m != rows or n != cols:
        raise ValueError(f"output of {m} x {n} for a result of {rows} x {cols}")
    return D, ldd, kind


def _packed(P: Packed, what: str) -> Packed:
    if not isinstance(P, Packed):
        raise ValueError(f"{what} has to be a packed matrix (see quantize and pack), got {type(P).__name__}")
    if _several_devices:
        _on_current_device(P.data)
    return P


def _check(status: int) -> None:
    if status:
        raise OzimmuError(status)


def packed_bytes(rows: int, n: int) -> int:
    return int(_lib.ozimmu_mx_bytes(rows, n))


def workspace_bytes(m: int, n: int, p: int) -> int:
    return int(_lib.ozimmu_mx_workspace_bytes(m, n, p))


def backward_workspace_bytes(m: int, n: int, p: int) -> int:
    return int(_lib.ozimmu_mx_backward_workspace_bytes(m, n, p))


def alloc_workspace(m: int, n: int, p: int, device="cuda", backward: bool = False) -> torch.Tensor:
    """Workspace for linear with these sizes; with `backward` for linear_backward too."""
    nbytes = max(workspace_bytes(m, n, p), backward_workspace_bytes(m, n, p) if backward else 0)
    return torch.empty(max(nbytes, 256), dtype=_uint8, device=device)


def _workspace(workspace: Optional[torch.Tensor], nbytes: int, like: torch.Tensor):
    """The caller's workspace, or a new one (none where none is needed): the tensor, its address and size."""
    if workspace is None:
        if not nbytes:
            return None, None, 0
        workspace = like.new_empty(nbytes, dtype=_uint8)
    elif not (workspace.is_cuda and workspace.dtype is _uint8 and workspace.is_contiguous()):
        raise ValueError("a workspace is a contiguous uint8 tensor on the GPU")
    elif _several_devices:
        _on_current_device(workspace)
    return workspace, workspace.data_ptr(), workspace.numel()


def _empty(rows: int, n: int, like: torch.Tensor) -> Packed:
    P = Packed.__new__(Packed)
    P.data, P.rows, P.n = like.new_empty(_lib.ozimmu_mx_bytes(rows, n), dtype=_uint8), rows, n
    return P


def quantize(X: torch.Tensor, rows: bool = True, cols: bool = False) -> Tuple[Optional[Packed], Optional[Packed]]:
    """X quantised with blocks along its rows, and its transpose with blocks along the columns of X (None for what is not asked for)."""
    m, n, ldx, kind = _matrix(X)
    if not rows and not cols:
        raise ValueError("nothing asked for: rows, cols or both")
    by_row = _empty(m, n, X) if rows else None
    by_col = _empty(n, m, X) if cols else None
    status = _lib.ozimmu_mx_quantize(kind, m, n, X.data_ptr(), ldx, by_row.data.data_ptr() if rows else None,
                                     by_col.data.data_ptr() if cols else None, ozimmu._stream())
    if status:
        raise OzimmuError(status)
    return by_row, by_col


def dequantize(P: Packed, dtype=None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The values of a packed matrix (in float32, or the type of `out`, unless said otherwise)."""
    data = _packed(P, "the matrix").data
    X, ldx, kind = _output(out, data, P.rows, P.n, dtype, torch.float32, 0.0)
    status = _lib.ozimmu_mx_dequantize(kind, P.rows, P.n, data.data_ptr(), X.data_ptr(), ldx, ozimmu._stream())
    if status:
        raise OzimmuError(status)
    return X


def _bytes_matrix(t: torch.Tensor, rows: int, width: int, what: str) -> int:
    if not t.is_cuda or t.dtype is not torch.uint8 or t.dim() != 2 or tuple(t.shape) != (rows, width):
        raise ValueError(f"{what}: expected uint8 of {rows} x {width} on the GPU, got {t.dtype} of {tuple(t.shape)}")
    if _several_devices:
        _on_current_device(t)
    if width > 1 and t.stride(1) != 1 or rows > 1 and t.stride(0) < width:
        raise ValueError(f"{what}: expected unit stride along rows that do not overlap")
    return t.stride(0) if rows > 1 else max(width, 1)


def pack(codes: torch.Tensor, scales: torch.Tensor, n: Optional[int] = None) -> Packed:
    """A matrix of n columns (default: as many as there are codes) from the plain layout: per row ceil(n / 32) blocks of 16 bytes with
    two codes each, the first in the lower half, and as many scale bytes."""
    if scales.dim() != 2:
        raise ValueError("scales: expected a 2-D tensor")
    rows, blocks = scales.shape
    n = blocks * BLOCK if n is None else n
    if -(-n // BLOCK) != blocks:
        raise ValueError(f"{blocks} scales a row for {n} columns")
    ldc, lds = _bytes_matrix(codes, rows, blocks * BLOCK // 2, "codes"), _bytes_matrix(scales, rows, blocks, "scales")
    P = _empty(rows, n, codes)
    _check(_lib.ozimmu_mx_pack(rows, n, codes.data_ptr(), ldc, scales.data_ptr(), lds, P.data.data_ptr(), ozimmu._stream()))
    return P


def unpack(P: Packed) -> Tuple[torch.Tensor, torch.Tensor]:
    """Codes and scales of a packed matrix in the plain layout."""
    P = _packed(P, "the matrix")
    blocks = -(-P.n // BLOCK)
    codes = torch.empty((P.rows, blocks * BLOCK // 2), dtype=torch.uint8, device=P.data.device)
    scales = torch.empty((P.rows, blocks), dtype=torch.uint8, device=P.data.device)
    _check(_lib.ozimmu_mx_unpack(P.rows, P.n, P.data.data_ptr(), codes.data_ptr(), max(codes.shape[1], 1), scales.data_ptr(),
                                 max(blocks, 1), ozimmu._stream()))
    return codes, scales


def gemm(A: Packed, B: Packed, dtype=None, alpha: float = 1.0, beta: float = 0.0, D: Optional[torch.Tensor] = None,
         way: str = "auto") -> torch.Tensor:
    """D <- alpha A B^T + beta D from packed matrices (a new D in float32 unless said otherwise); `way` forces how it is run (see
    ozimmu_mx_gemm_way in the header)."""
    A, B = _packed(A, "A"), _packed(B, "B")
    if A.n != B.n:
        raise ValueError("inner dimensions differ")
    m, n, p = A.rows, A.n, B.rows
    D, ldd, kind = _output(D, A.data, m, p, dtype, torch.float32, beta)
    _check(_lib.ozimmu_mx_gemm_way(WAYS[way], m, n, p, alpha, A.data.data_ptr(), B.data.data_ptr(), beta, kind, D.data_ptr(), ldd,
                                   ozimmu._stream()))
    return D


def linear(X: torch.Tensor, W: Packed, dtype=None, alpha: float = 1.0, beta: float = 0.0, D: Optional[torch.Tensor] = None,
           workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """D <- alpha Q(X) W^T + beta D for rows X as they come and packed weights W (a new D in the type of X unless said otherwise)."""
    m, n, ldx, xkind = _matrix(X)
    _not_recorded(X, "X")
    if _packed(W, "W").n != n:
        raise ValueError("inner dimensions differ")
    p = W.rows
    D, ldd, dkind = _output(D, X, m, p, dtype, X.dtype, beta)
    nbytes = _lib.ozimmu_mx_workspace_bytes(m, n, p) if workspace is None and m > FEW_ROWS else 0
    workspace, room, size = _workspace(workspace, nbytes, X)
    status = _lib.ozimmu_mx_linear(m, n, p, alpha, xkind, X.data_ptr(), ldx, W.data.data_ptr(), beta, dkind, D.data_ptr(), ldd,
                                   room, size, ozimmu._stream())
    if status:
        raise OzimmuError(status)
    return D


def linear_backward(G: torch.Tensor, X: Optional[torch.Tensor], Wt: Optional[Packed], alpha: float = 1.0, beta_x: float = 0.0,
                    beta_w: float = 0.0, dX: Optional[torch.Tensor] = None, dW: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
    """Gradients of linear from the gradient G of its output: dX <- alpha Q(G) Wt^T + beta_x dX (Wt: the by-column form of the weights
    from quantize(W, cols=True); None: no dX) and dW <- alpha Q(G^T) Q(X^T)^T + beta_w dW (X None: no dW).  Unless they are handed over,
    dX comes in the type of G and dW in float32."""
    m, p, ldg, kind = _matrix(G)
    if X is None and Wt is None:
        raise ValueError("neither X (for dW) nor Wt (for dX) given")
    if (X is None and dW is not None) or (Wt is None and dX is not None):
        raise ValueError("dW takes X, dX takes Wt")
    _not_recorded(G, "G")
    _not_recorded(X, "X")
    ldx = lddx = lddw = dxkind = dwkind = 0
    x_at = wt_at = dx_at = dw_at = None
    if X is not None:
        rows, n, ldx, xkind = _matrix(X)
        if xkind != kind:
            raise ValueError("X and G have to be of one type")
        if rows != m:
            raise ValueError("X and G have to have as many rows")
        dW, lddw, dwkind = _output(dW, G, p, n, None, torch.float32, beta_w)
        x_at, dw_at = X.data_ptr(), dW.data_ptr()
    if Wt is not None:
        if X is None:
            n = _packed(Wt, "Wt").rows
        if _packed(Wt, "Wt").rows != n or Wt.n != p:
            raise ValueError(f"Wt of {Wt.rows} x {Wt.n} for a layer of {n} to {p}")
        dX, lddx, dxkind = _output(dX, G, m, n, None, G.dtype, beta_x)
        wt_at, dx_at = Wt.data.data_ptr(), dX.data_ptr()
    nbytes = _lib.ozimmu_mx_backward_workspace_bytes(m, n, p) if workspace is None else 0
    workspace, room, size = _workspace(workspace, nbytes, G)
    status = _lib.ozimmu_mx_linear_backward(m, n, p, alpha, kind, G.data_ptr(), ldg, x_at, ldx, wt_at, beta_x, dxkind, dx_at, lddx, beta_w,
                                            dwkind, dw_at, lddw, room, size, ozimmu._stream())
    if status:
        raise OzimmuError(status)
    return dX, dW
