"""Thin Python binding of the operators around a model's output layer (include/ozimmu_lm.h): a linear layer whose weights are stored in 4 bits with
a scale per group, and the cross entropy of a linear layer's outputs over a large vocabulary, with its gradient.

Argument marshalling only: device pointers of torch tensors and the current HIP stream go to the entry points of the same name.
There is no CPU fallback.  Matrices are 2-D tensors with unit stride along their rows; results that are not handed over are allocated,
workspaces too.  All tensors of a call have to be on the current device (torch.cuda.device), whose current stream it goes to.

No operations are recorded for torch's autograd: cross_entropy_backward is called by the user, in torch.no_grad() or in the backward of a
torch.autograd.Function.  linear, cross_entropy and cross_entropy_backward refuse a tensor that requires a gradient while torch records.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

from . import mx, ozimmu
from .mx import _matrix, _not_recorded, _on_current_device, _output, _workspace
from .ozimmu import OzimmuError

_lib = ozimmu._lib
_i64, _int, _vp, _sz, _float = ctypes.c_int64, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float

_SIGNATURES = {
    "ozimmu_lm_bytes": (_sz, [_i64, _i64, _int, _int]),
    "ozimmu_lm_quantize": (_int, [_int, _i64, _i64, _vp, _i64, _int, _int, _int, _vp, _vp]),
    "ozimmu_lm_dequantize": (_int, [_int, _i64, _i64, _int, _int, _int, _vp, _vp, _i64, _vp]),
    "ozimmu_lm_pack": (_int, [_i64, _i64, _int, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _vp]),
    "ozimmu_lm_unpack": (_int, [_i64, _i64, _int, _vp, _vp, _i64, _vp, _i64, _vp, _i64, _vp]),
    "ozimmu_lm_linear_workspace_bytes": (_sz, [_i64, _i64, _i64]),
    "ozimmu_lm_linear": (_int, [_i64, _i64, _i64, _float, _int, _vp, _i64, _int, _int, _int, _vp, _float, _int, _vp, _i64, _vp, _sz, _vp]),
    "ozimmu_lm_linear_way": (_int, [_int, _i64, _i64, _i64, _float, _int, _vp, _i64, _int, _int, _int, _vp, _float, _int, _vp, _i64, _vp, _sz,
                                    _vp]),
    "ozimmu_lm_linear_way_workspace_bytes": (_sz, [_int, _i64, _i64, _i64]),
    "ozimmu_lm_linear_choose": (_int, [_i64, _i64, _i64]),
    "ozimmu_lm_cross_entropy_workspace_bytes": (_sz, [_i64, _i64, _i64]),
    "ozimmu_lm_cross_entropy": (_int, [_int, _i64, _i64, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _i64, _vp, _vp, _vp, _sz, _vp]),
    "ozimmu_lm_cross_entropy_backward_workspace_bytes": (_sz, [_i64, _i64, _i64]),
    "ozimmu_lm_cross_entropy_backward": (_int, [_int, _i64, _i64, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _i64, _vp, _int, _vp, _i64,
                                                _float, _int, _vp, _i64, _vp, _sz, _vp]),
}
for _name, (_restype, _argtypes) in _SIGNATURES.items():
    getattr(_lib, _name).restype, getattr(_lib, _name).argtypes = _restype, _argtypes
EXPORTS = list(_SIGNATURES)

GROUPS = (32, 64, 128)
SCALE_TYPES = (torch.bfloat16, torch.float16)
WAYS = {"auto": -1, "direct": 0, "tile": 1, "shared": 2}
IGNORE = -100
DIRECT_ROWS = 16  # up to here a layer takes no workspace, whatever its sizes (asking the library for it is most of a microsecond)
_uint8 = torch.uint8


class Packed:
    """Weights of rows x n in 4 bits: `data` holds their bytes (on the GPU, private layout; see pack and unpack), with scales of scale_type
    for every `group` elements of a row and, if `zeros` is true, zero points."""
    __slots__ = ("data", "rows", "n", "group", "zeros", "scale_type", "kind")

    def __init__(self, data: torch.Tensor, rows: int, n: int, group: int, zeros: bool, scale_type: torch.dtype):
        if not (data.is_cuda and data.dtype is _uint8 and data.dim() == 1 and data.is_contiguous()):
            raise ValueError("packed data is a contiguous 1-D uint8 tensor on the GPU")
        if data.numel() < packed_bytes(rows, n, group, zeros):
            raise ValueError(f"{data.numel()} bytes for packed weights of {rows} x {n}, which take {packed_bytes(rows, n, group, zeros)}")
        self.data, self.rows, self.n, self.group, self.zeros = data, rows, n, group, bool(zeros)
        self.scale_type, self.kind = scale_type, _scale_kind(scale_type)

    @property
    def shape(self) -> Tuple[int, int]:
        return self.rows, self.n


def _scale_kind(scale_type) -> int:
    if scale_type not in SCALE_TYPES:
        raise ValueError(f"scales are bfloat16 or float16, got {scale_type}")
    return mx.TYPES[scale_type]


def packed_bytes(rows: int, n: int, group: int, zeros: bool) -> int:
    if group not in GROUPS:
        raise ValueError(f"groups are of 32, 64 or 128 elements, got {group}")
    return int(_lib.ozimmu_lm_bytes(rows, n, group, bool(zeros)))


def _empty(rows: int, n: int, group: int, zeros: bool, scale_type, like: torch.Tensor) -> Packed:
    P = Packed.__new__(Packed)
    P.kind = _scale_kind(scale_type)
    P.data = like.new_empty(packed_bytes(rows, n, group, zeros), dtype=_uint8)
    P.rows, P.n, P.group, P.zeros, P.scale_type = rows, n, group, bool(zeros), scale_type
    return P


def _packed(P: Packed, what: str) -> Packed:
    if not isinstance(P, Packed):
        raise ValueError(f"{what} has to be packed 4-bit weights (see quantize and pack), got {type(P).__name__}")
    if mx._several_devices:
        _on_current_device(P.data)
    return P


def _check(status: int) -> None:
    if status:
        raise OzimmuError(status)


def quantize(W: torch.Tensor, group: int = 128, zeros: bool = False, scale_type: torch.dtype = torch.float16) -> Packed:
    """W quantised to 4 bits, a scale (and, if `zeros` says so, a zero point) for every `group` elements of a row."""
    p, n, ldw, kind = _matrix(W)
    P = _empty(p, n, group, zeros, scale_type, W)
    _check(_lib.ozimmu_lm_quantize(kind, p, n, W.data_ptr(), ldw, group, P.zeros, P.kind, P.data.data_ptr(), ozimmu._stream()))
    return P


def dequantize(P: Packed, dtype=None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The values of packed weights (in float32, or the type of `out`, unless said otherwise)."""
    data = _packed(P, "the matrix").data
    W, ldw, kind = _output(out, data, P.rows, P.n, dtype, torch.float32, 0.0)
    _check(_lib.ozimmu_lm_dequantize(kind, P.rows, P.n, P.group, P.zeros, P.kind, data.data_ptr(), W.data_ptr(), ldw, ozimmu._stream()))
    return W


def _plain(t: torch.Tensor, rows: int, width: int, dtypes, what: str) -> int:
    if not t.is_cuda or t.dtype not in dtypes or t.dim() != 2 or tuple(t.shape) != (rows, width):
        raise ValueError(f"{what}: expected {' or '.join(map(str, dtypes))} of {rows} x {width} on the GPU, got {t.dtype} of {tuple(t.shape)}")
    if mx._several_devices:
        _on_current_device(t)
    if width > 1 and t.stride(1) != 1 or rows > 1 and t.stride(0) < width:
        raise ValueError(f"{what}: expected unit stride along rows that do not overlap")
    return t.stride(0) if rows > 1 else max(width, 1)


def pack(codes: torch.Tensor, scales: torch.Tensor, zeros: Optional[torch.Tensor] = None, n: Optional[int] = None, group: int = 128) -> Packed:
    """Weights of n columns (default: two for every byte of codes) from the plain layout: per row ceil(n / 2) bytes of two codes each, the
    first in the lower half, ceil(n / group) scales in bfloat16 or float16 and, if there are zero points, as many of those in uint8."""
    if codes.dim() != 2:
        raise ValueError("codes: expected a 2-D tensor")
    rows = codes.shape[0]
    n = 2 * codes.shape[1] if n is None else n
    P = _empty(rows, n, group, zeros is not None, scales.dtype, codes)
    groups = -(-n // group)
    ldc, lds = _plain(codes, rows, -(-n // 2), (_uint8,), "codes"), _plain(scales, rows, groups, SCALE_TYPES, "scales")
    ldz = 0 if zeros is None else _plain(zeros, rows, groups, (_uint8,), "zeros")
    _check(_lib.ozimmu_lm_pack(rows, n, group, codes.data_ptr(), ldc, scales.data_ptr(), lds, None if zeros is None else zeros.data_ptr(), ldz,
                               P.data.data_ptr(), ozimmu._stream()))
    return P


def unpack(P: Packed) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
    """Codes, scales and zero points (None: without) of packed weights in the plain layout."""
    data = _packed(P, "the matrix").data
    groups = -(-P.n // P.group)
    codes = data.new_empty((P.rows, -(-P.n // 2)), dtype=_uint8)
    scales = data.new_empty((P.rows, groups), dtype=P.scale_type)
    zeros = data.new_empty((P.rows, groups), dtype=_uint8) if P.zeros else None
    _check(_lib.ozimmu_lm_unpack(P.rows, P.n, P.group, data.data_ptr(), codes.data_ptr(), max(codes.shape[1], 1), scales.data_ptr(), max(groups, 1),
                                 zeros.data_ptr() if P.zeros else None, max(groups, 1), ozimmu._stream()))
    return codes, scales, zeros


def linear_workspace_bytes(m: int, n: int, p: int, way: str = "auto") -> int:
    return int(_lib.ozimmu_lm_linear_way_workspace_bytes(WAYS[way], m, n, p))


def linear(X: torch.Tensor, W: Packed, dtype=None, alpha: float = 1.0, beta: float = 0.0, D: Optional[torch.Tensor] = None,
           workspace: Optional[torch.Tensor] = None, way: str = "auto") -> torch.Tensor:
    """D <- alpha X W^T + beta D for rows X in 16 bits and packed weights W (a new D in the type of X unless said otherwise); `way` forces how
    it is run (see ozimmu_lm_linear_way in the header)."""
    m, n, ldx, xkind = _matrix(X)
    if not xkind:
        raise ValueError("X: expected bfloat16 or float16, got torch.float32")
    _not_recorded(X, "X")
    if _packed(W, "W").n != n:
        raise ValueError("inner dimensions differ")
    p, number = W.rows, WAYS[way]
    D, ldd, dkind = _output(D, X, m, p, dtype, X.dtype, beta)
    if workspace is None and (number == 0 or (number < 0 and m <= DIRECT_ROWS)):
        room, size = None, 0
    else:
        nbytes = _lib.ozimmu_lm_linear_way_workspace_bytes(number, m, n, p) if workspace is None else 0
        workspace, room, size = _workspace(workspace, nbytes, X)
    status = _lib.ozimmu_lm_linear_way(number, m, n, p, alpha, xkind, X.data_ptr(), ldx, W.group, W.zeros, W.kind, W.data.data_ptr(), beta, dkind,
                                       D.data_ptr(), ldd, room, size, ozimmu._stream())
    if status:
        raise OzimmuError(status)
    return D


def _vector(t: torch.Tensor, m: int, dtype, what: str) -> int:
    """The stride of a 1-D tensor of m numbers."""
    if not t.is_cuda or t.dtype is not dtype or t.dim() != 1 or t.shape[0] != m:
        raise ValueError(f"{what}: expected {dtype} of {m} on the GPU, got {t.dtype} of {tuple(t.shape)}")
    if mx._several_devices:
        _on_current_device(t)
    return t.stride(0) if m > 1 else 1


def _layer(X: torch.Tensor, W: torch.Tensor, y: torch.Tensor):
    """Sizes, leading dimensions, type number and the targets' stride of a layer with its loss."""
    m, n, ldx, kind = _matrix(X)
    p, nw, ldw, wkind = _matrix(W)
    if not kind or not wkind:
        raise ValueError(f"X and W: expected bfloat16 or float16, got {X.dtype} and {W.dtype}")
    if wkind != kind:
        raise ValueError("X and W have to be of one type")
    if nw != n:
        raise ValueError("inner dimensions differ")
    return m, n, p, ldx, ldw, kind, _vector(y, m, torch.int64, "targets")


def _dense(t: Optional[torch.Tensor], m: int, like: torch.Tensor, what: str) -> torch.Tensor:
    if t is None:
        return like.new_empty(m, dtype=torch.float32)
    if _vector(t, m, torch.float32, what) != 1:
        raise ValueError(f"{what}: expected unit stride")
    return t


def cross_entropy_workspace_bytes(m: int, n: int, p: int, backward: bool = False) -> int:
    """Workspace of cross_entropy, or of cross_entropy_backward, for m tokens of n elements and p words."""
    return int((_lib.ozimmu_lm_cross_entropy_backward_workspace_bytes if backward else _lib.ozimmu_lm_cross_entropy_workspace_bytes)(m, n, p))


def cross_entropy(X: torch.Tensor, W: torch.Tensor, y: torch.Tensor, ignore: int = IGNORE, loss: Optional[torch.Tensor] = None,
                  lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Per row of X the cross entropy of its logits X W^T against the target in y (0 where that is `ignore`), and the logarithm of the sum of
    their exponentials, which cross_entropy_backward takes."""
    m, n, p, ldx, ldw, kind, stride = _layer(X, W, y)
    _not_recorded(X, "X")
    _not_recorded(W, "W")
    loss, lse = _dense(loss, m, X, "loss"), _dense(lse, m, X, "lse")
    nbytes = _lib.ozimmu_lm_cross_entropy_workspace_bytes(m, n, p) if workspace is None else 0
    workspace, room, size = _workspace(workspace, nbytes, X)
    status = _lib.ozimmu_lm_cross_entropy(kind, m, n, p, X.data_ptr(), ldx, W.data_ptr(), ldw, y.data_ptr(), stride, ignore, loss.data_ptr(),
                                          lse.data_ptr(), room, size, ozimmu._stream())
    if status:
        raise OzimmuError(status)
    return loss, lse


def cross_entropy_backward(g: torch.Tensor, X: torch.Tensor, W: torch.Tensor, y: torch.Tensor, lse: torch.Tensor, ignore: int = IGNORE,
                           dx_type=None, dw_type=None, beta: float = 0.0, dX: Optional[torch.Tensor] = None, dW: Optional[torch.Tensor] = None,
                           need_dx: bool = True, need_dw: bool = True,
                           workspace: Optional[torch.Tensor] = None) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
    """Gradients of cross_entropy from the gradient g of its losses: dX, and dW + beta times the dW that is handed over.  Unless said
    otherwise they come in the types of X and W; need_dx, need_dw: whether they are wanted (None comes for one that is not)."""
    m, n, p, ldx, ldw, kind, stride = _layer(X, W, y)
    for t, what in ((X, "X"), (W, "W"), (g, "g")):
        _not_recorded(t, what)
    if not need_dx and not need_dw:
        raise ValueError("neither dX nor dW asked for")
    if (dX is not None and not need_dx) or (dW is not None and not need_dw):
        raise ValueError("an output for a gradient that is not asked for")
    g_stride = _vector(g, m, torch.float32, "g")
    if _vector(lse, m, torch.float32, "lse") != 1:
        raise ValueError("lse: expected unit stride")
    lddx = lddw = dxkind = dwkind = 0
    if need_dx:
        dX, lddx, dxkind = _output(dX, X, m, n, dx_type, X.dtype, 0.0)
    if need_dw:
        dW, lddw, dwkind = _output(dW, W, p, n, dw_type, W.dtype, beta)
    nbytes = _lib.ozimmu_lm_cross_entropy_backward_workspace_bytes(m, n, p) if workspace is None else 0
    workspace, room, size = _workspace(workspace, nbytes, X)
    status = _lib.ozimmu_lm_cross_entropy_backward(kind, m, n, p, g.data_ptr(), g_stride, X.data_ptr(), ldx, W.data_ptr(), ldw, y.data_ptr(), stride,
                                                   ignore, lse.data_ptr(), dxkind, dX.data_ptr() if need_dx else None, lddx, beta, dwkind,
                                                   dW.data_ptr() if need_dw else None, lddw, room, size, ozimmu._stream())
    if status:
        raise OzimmuError(status)
    return (dX if need_dx else None), (dW if need_dw else None)
