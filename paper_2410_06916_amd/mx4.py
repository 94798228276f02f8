"""MXFP4 matrices and the products with them (swift_mx4_* of include/swift.h): argument checks and marshalling only.

    w = mx4_quantize(weight)                      # [rows, depth] fp32 or bf16 -> 4.25 bits a weight
    y = mx4_linear(x, w, residual=r)              # x W^T + r
    gu = mx4_quantize_gated(gate, up)
    h = mx4_swiglu(x, gu)                         # silu(x gate^T) * (x up^T)

Work goes to torch's current stream of the tensors' device, which has to be the stream they are ready on; results are new tensors
unless `out` is given.  There is no gradient: the weights are frozen, and tensors that require one are refused while gradients are enabled.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional

import torch

from .binding import BF16, F32, _chk, lib

_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}
_F32 = torch.float32


class Mx4Weight:
    """A packed matrix [rows][depth] (gated: a gate and an up matrix of that size each).  `data`: the packed bytes, a uint8 tensor."""

    __slots__ = ("rows", "depth", "gated", "data", "device")

    def __init__(self, rows: int, depth: int, gated: bool, data: torch.Tensor):
        if data.dtype != torch.uint8 or data.dim() != 1 or not data.is_contiguous() or data.numel() != packed_bytes(rows, depth, gated):
            raise ValueError("data must be the packed bytes of such a matrix: a contiguous uint8 vector")
        self.rows, self.depth, self.gated, self.data, self.device = rows, depth, bool(gated), data, data.device

    def to(self, device) -> "Mx4Weight":
        return Mx4Weight(self.rows, self.depth, self.gated, self.data.to(device))


def packed_bytes(rows: int, depth: int, gated: bool = False) -> int:
    n = C.c_uint64()
    _chk(lib().swift_mx4_bytes(rows, depth, gated, C.byref(n)), "swift_mx4_bytes")
    return n.value


def _check(t: torch.Tensor, what: str, device=None) -> int:
    """The library's code for t's type, once t is something a kernel can read or write by rows."""
    dt = _DTYPES.get(t.dtype)
    if dt is None:
        raise TypeError(f"{what} must be float32 or bfloat16, not {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{what} must be on the GPU")
    if device is not None and t.device != device:
        raise ValueError(f"{what} is on {t.device}, the weight on {device}")
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{what} requires a gradient, which these operators do not have")
    return dt


def _rows_of(t: torch.Tensor, what: str) -> int:
    """Elements from one row of a matrix to the next."""
    if t.dim() != 2:
        raise ValueError(f"{what} must be a matrix, not of shape {tuple(t.shape)}")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"the elements of a row of {what} must be contiguous")
    ld = t.stride(0) if t.shape[0] > 1 else t.shape[1]
    if ld < t.shape[1]:
        raise ValueError(f"the rows of {what} overlap")
    return ld


def _on(device, f, *args):
    """f(*args, stream) with `device` current."""
    if device.index != torch.cuda.current_device():
        with torch.cuda.device(device):
            return f(*args, torch.cuda.current_stream(device).cuda_stream)
    return f(*args, torch.cuda.current_stream(device).cuda_stream)


def mx4_quantize(w: torch.Tensor) -> Mx4Weight:
    """The matrix w [rows, depth] in MXFP4."""
    dt, ld = _check(w, "w"), _rows_of(w, "w")
    rows, depth = w.shape
    data = torch.empty(packed_bytes(rows, depth), dtype=torch.uint8, device=w.device)
    _chk(_on(w.device, lib().swift_mx4_quantize, data.data_ptr(), w.data_ptr(), ld, None, 0, dt, rows, depth), "swift_mx4_quantize")
    return Mx4Weight(rows, depth, False, data)


def mx4_quantize_gated(gate: torch.Tensor, up: torch.Tensor) -> Mx4Weight:
    """gate and up [rows, depth] in MXFP4, as one packed matrix for mx4_swiglu."""
    dt, ld, ld_up = _check(gate, "gate"), _rows_of(gate, "gate"), _rows_of(up, "up")
    if _check(up, "up", gate.device) != dt or up.shape != gate.shape:
        raise ValueError("gate and up must be of one type and shape")
    rows, depth = gate.shape
    data = torch.empty(packed_bytes(rows, depth, True), dtype=torch.uint8, device=gate.device)
    _chk(_on(gate.device, lib().swift_mx4_quantize, data.data_ptr(), gate.data_ptr(), ld, up.data_ptr(), ld_up, dt, rows, depth), "swift_mx4_quantize")
    return Mx4Weight(rows, depth, True, data)


def _output(out: Optional[torch.Tensor], shape, dtype, device, what: str):
    """(the result as a matrix, its type's code, its row pitch)."""
    if out is None:
        t = torch.empty(shape, dtype=dtype, device=device)
        return t, _DTYPES[dtype], shape[1]
    dt = _check(out, what, device)
    if out.dtype != dtype or tuple(out.shape) != tuple(shape):
        raise ValueError(f"{what} must be {dtype} of shape {tuple(shape)}")
    return out, dt, _rows_of(out, what)


def _out_dtype(dtype: Optional[torch.dtype], out: Optional[torch.Tensor], default: torch.dtype) -> torch.dtype:
    dtype = dtype or (out.dtype if out is not None else default)
    if dtype not in _DTYPES:
        raise TypeError(f"results are float32 or bfloat16, not {dtype}")
    return dtype


def mx4_dequantize(w: Mx4Weight, dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The numbers w stands for, [rows, depth], or [2 * rows, depth] of a gated one (gate rows first); exact in either type."""
    y, dt, ld = _output(out, (w.rows * (2 if w.gated else 1), w.depth), _out_dtype(dtype, None, _F32), w.device, "out")
    _chk(_on(w.device, lib().swift_mx4_dequantize, y.data_ptr(), ld, dt, w.data.data_ptr(), w.rows, w.depth, w.gated), "swift_mx4_dequantize")
    return y


def _activations(x: torch.Tensor, w: Mx4Weight):
    """(x as rows, their number, type's code, pitch, workspace and its size)."""
    dt = _check(x, "x", w.device)
    if x.dim() < 1 or x.shape[-1] != w.depth:
        raise ValueError(f"x must be [..., {w.depth}], not {tuple(x.shape)}")
    rows = x if x.dim() == 2 else x.reshape(-1, w.depth)
    ld, n = _rows_of(rows, "x"), rows.shape[0]
    need = C.c_uint64()
    _chk(lib().swift_mx4_workspace(w.rows, w.depth, w.gated, n, dt, C.byref(need)), "swift_mx4_workspace")
    ws = torch.empty(need.value, dtype=torch.uint8, device=w.device)
    return rows, n, dt, ld, ws, need.value


def mx4_linear(x: torch.Tensor, w: Mx4Weight, residual: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
               out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [..., depth] times w transposed, plus residual [..., rows]: [..., rows], of x's type unless out_dtype or out say otherwise.
    out may be the residual."""
    if w.gated:
        raise ValueError("a gated weight goes through mx4_swiglu")
    rows, n, x_dt, ld_x, ws, need = _activations(x, w)
    shape = (*x.shape[:-1], w.rows)
    dtype = _out_dtype(out_dtype, out, x.dtype)
    y, y_dt, ld_y = _output(None if out is None else _as_rows(out, shape, "out"), (n, w.rows), dtype, w.device, "out")
    r_ptr, ld_r = None, 0
    if residual is not None:
        if residual.dtype != dtype:
            raise ValueError(f"residual must be of the result's type, {dtype}")
        _check(residual, "residual", w.device)
        r = _as_rows(residual, shape, "residual")
        r_ptr, ld_r = r.data_ptr(), _rows_of(r, "residual")
    _chk(_on(w.device, lib().swift_mx4_linear, y.data_ptr(), ld_y, y_dt, rows.data_ptr(), ld_x, x_dt, n, w.data.data_ptr(), w.rows, w.depth, r_ptr, ld_r,
             ws.data_ptr(), need), "swift_mx4_linear")
    return out if out is not None else y.view(shape)


def mx4_swiglu(x: torch.Tensor, w: Mx4Weight, out_dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """silu(x gate^T) * (x up^T) for x [..., depth] and a gated w: [..., rows], of x's type unless out_dtype or out say otherwise."""
    if not w.gated:
        raise ValueError("mx4_swiglu takes a weight of mx4_quantize_gated")
    rows, n, x_dt, ld_x, ws, need = _activations(x, w)
    shape = (*x.shape[:-1], w.rows)
    dtype = _out_dtype(out_dtype, out, x.dtype)
    y, y_dt, ld_y = _output(None if out is None else _as_rows(out, shape, "out"), (n, w.rows), dtype, w.device, "out")
    _chk(_on(w.device, lib().swift_mx4_swiglu, y.data_ptr(), ld_y, y_dt, rows.data_ptr(), ld_x, x_dt, n, w.data.data_ptr(), w.rows, w.depth, ws.data_ptr(), need),
         "swift_mx4_swiglu")
    return out if out is not None else y.view(shape)


def _as_rows(t: torch.Tensor, shape, what: str) -> torch.Tensor:
    """t, of shape [..., rows], as a matrix over the same memory."""
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what} must be of shape {tuple(shape)}, not {tuple(t.shape)}")
    if t.dim() == 2:
        return t
    try:
        return t.view(-1, shape[-1])
    except RuntimeError:
        raise ValueError(f"the rows of {what} must lie at one distance from each other") from None
