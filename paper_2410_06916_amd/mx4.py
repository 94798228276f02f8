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
import functools
from typing import Optional

import torch

from .binding import BF16, F32, _chk, lib

_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}
_F32 = torch.float32
_INT_MAX = (1 << 31) - 1  # (what lies beyond would be cut to 32 bits on its way into the library)


class Mx4Weight:
    """A packed matrix [rows][depth] (gated: a gate and an up matrix of that size each).  `data`: the packed bytes, a uint8 tensor."""

    __slots__ = ("rows", "depth", "gated", "data", "device", "address", "_workspace")

    def __init__(self, rows: int, depth: int, gated: bool, data: torch.Tensor):
        if data.dtype != torch.uint8 or data.dim() != 1 or not data.is_contiguous() or data.numel() != packed_bytes(rows, depth, gated):
            raise ValueError("data must be the packed bytes of such a matrix: a contiguous uint8 vector")
        self._set(rows, depth, bool(gated), data)

    def _set(self, rows, depth, gated, data):
        self.rows, self.depth, self.gated, self.data, self.device = rows, depth, gated, data, data.device
        self.address = data.data_ptr()
        self._workspace = {}  # bytes that a product needs, by rows and type of x

    def to(self, device) -> "Mx4Weight":
        return Mx4Weight(self.rows, self.depth, self.gated, self.data.to(device))

    def workspace_bytes(self, n: int, x_dtype: int) -> int:
        need = self._workspace.get((n, x_dtype))
        if need is None:
            size = C.c_uint64()
            _chk(lib().swift_mx4_workspace(self.rows, self.depth, self.gated, n, x_dtype, C.byref(size)), "swift_mx4_workspace")
            if len(self._workspace) >= 256:
                self._workspace.clear()
            need = self._workspace[n, x_dtype] = size.value
        return need


@functools.lru_cache(maxsize=1024)
def packed_bytes(rows: int, depth: int, gated: bool = False) -> int:
    if max(rows, depth) > _INT_MAX:
        raise ValueError("a packed matrix has at most 2^22 rows and a depth of at most 2^22")
    n = C.c_uint64()
    _chk(lib().swift_mx4_bytes(rows, depth, gated, C.byref(n)), "swift_mx4_bytes")
    return n.value


def _packed(rows: int, depth: int, gated: bool, device) -> Mx4Weight:
    w = Mx4Weight.__new__(Mx4Weight)
    w._set(rows, depth, gated, torch.empty(packed_bytes(rows, depth, gated), dtype=torch.uint8, device=device))
    return w


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
    shape = t.shape
    if len(shape) != 2:
        raise ValueError(f"{what} must be a matrix, not of shape {tuple(shape)}")
    rows, width = shape
    ld, step = t.stride()
    if step != 1 and width > 1:
        raise ValueError(f"the elements of a row of {what} must be contiguous")
    if rows <= 1:
        return width
    if ld < width:
        raise ValueError(f"the rows of {what} overlap")
    return ld


_current_device, _raw_stream = torch.cuda.current_device, torch._C._cuda_getCurrentRawStream
_functions = {}  # the library's, by name


def _call(name: str, device, *args):
    """The C call with torch's current stream of `device` as its last argument, `device` being current."""
    f = _functions.get(name)
    if f is None:
        f = _functions[name] = getattr(lib(), name)
    index = device.index
    if index != _current_device():
        with torch.cuda.device(device):
            rc = f(*args, _raw_stream(index))
    else:
        rc = f(*args, _raw_stream(index))
    if rc:
        _chk(rc, name)


def mx4_quantize(w: torch.Tensor) -> Mx4Weight:
    """The matrix w [rows, depth] in MXFP4."""
    dt, ld = _check(w, "w"), _rows_of(w, "w")
    rows, depth = w.shape
    m = _packed(rows, depth, False, w.device)
    _call("swift_mx4_quantize", w.device, m.address, w.data_ptr(), ld, None, 0, dt, rows, depth)
    return m


def mx4_quantize_gated(gate: torch.Tensor, up: torch.Tensor) -> Mx4Weight:
    """gate and up [rows, depth] in MXFP4, as one packed matrix for mx4_swiglu."""
    dt, ld, ld_up = _check(gate, "gate"), _rows_of(gate, "gate"), _rows_of(up, "up")
    if _check(up, "up", gate.device) != dt or up.shape != gate.shape:
        raise ValueError("gate and up must be of one type and shape")
    rows, depth = gate.shape
    m = _packed(rows, depth, True, gate.device)
    _call("swift_mx4_quantize", gate.device, m.address, gate.data_ptr(), ld, up.data_ptr(), ld_up, dt, rows, depth)
    return m


def _out_dtype(dtype: Optional[torch.dtype], out: Optional[torch.Tensor], default: torch.dtype) -> torch.dtype:
    dtype = dtype or (out.dtype if out is not None else default)
    if dtype not in _DTYPES:
        raise TypeError(f"results are float32 or bfloat16, not {dtype}")
    return dtype


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


def _output(out: Optional[torch.Tensor], shape, width: int, dtype, device, x=None):
    """(the result, its address, row pitch and type's code); shape: as the caller sees it, rows of `width`; x: what it is made from."""
    if out is None:
        t = torch.empty(shape, dtype=dtype, device=device)
        return t, t.data_ptr(), width, _DTYPES[dtype]
    dt = _check(out, "out", device)
    if out.dtype != dtype:
        raise ValueError(f"out must be {dtype}, not {out.dtype}")
    m = _as_rows(out, shape, "out")
    if x is not None and m.data_ptr() == x.data_ptr() and m.numel():
        raise ValueError("out may not be x, whose rows are read while results are written")
    return out, m.data_ptr(), _rows_of(m, "out"), dt


def mx4_dequantize(w: Mx4Weight, dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The numbers w stands for, [rows, depth], or [2 * rows, depth] of a gated one (gate rows first), as float32 unless dtype or out say
    otherwise; exact in either type."""
    dtype = _out_dtype(dtype, out, _F32)
    if not w.data.is_cuda:
        raise ValueError("the weight must be on the GPU")
    rows = w.rows * (2 if w.gated else 1)
    y, ptr, ld, dt = _output(out, (rows, w.depth), w.depth, dtype, w.device)
    _call("swift_mx4_dequantize", w.device, ptr, ld, dt, w.address, w.rows, w.depth, w.gated)
    return y


def _activations(x: torch.Tensor, w: Mx4Weight):
    """(x's rows as a matrix, their number, pitch, type's code, the result's shape, the workspace that a product needs, its address and size)."""
    dt, shape = _check(x, "x", w.device), x.shape
    if not shape or shape[-1] != w.depth:
        raise ValueError(f"x must be [..., {w.depth}], not {tuple(shape)}")
    if len(shape) == 2:
        m, n = x, shape[0]
        y_shape = (n, w.rows)
    else:
        m = x.reshape(-1, w.depth)
        n, y_shape = m.shape[0], (*shape[:-1], w.rows)
    if n > _INT_MAX:
        raise ValueError("x has more than 2^31 - 1 rows")
    need = w.workspace_bytes(n, dt)
    if not need:
        return m, n, _rows_of(m, "x"), dt, y_shape, None, None, 0
    ws = torch.empty(need, dtype=torch.uint8, device=w.device)
    return m, n, _rows_of(m, "x"), dt, y_shape, ws, ws.data_ptr(), need


def mx4_linear(x: torch.Tensor, w: Mx4Weight, residual: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
               out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [..., depth] times w transposed, plus residual [..., rows]: [..., rows], of x's type unless out_dtype or out say otherwise.
    out may be the residual, and overlaps no other tensor of the call."""
    if w.gated:
        raise ValueError("a gated weight goes through mx4_swiglu")
    m, n, ld_x, x_dt, shape, ws, ws_ptr, need = _activations(x, w)
    dtype = x.dtype if out_dtype is None and out is None else _out_dtype(out_dtype, out, x.dtype)
    y, y_ptr, ld_y, y_dt = _output(out, shape, w.rows, dtype, w.device, m)
    r_ptr, ld_r = None, 0
    if residual is not None:
        if residual.dtype != dtype:
            raise ValueError(f"residual must be of the result's type, {dtype}")
        _check(residual, "residual", w.device)
        r = _as_rows(residual, shape, "residual")
        r_ptr, ld_r = r.data_ptr(), _rows_of(r, "residual")
        if r_ptr == y_ptr and ld_r != ld_y and n > 1:
            raise ValueError("out and residual overlap: their rows lie at different distances")
    _call("swift_mx4_linear", w.device, y_ptr, ld_y, y_dt, m.data_ptr(), ld_x, x_dt, n, w.address, w.rows, w.depth, r_ptr, ld_r, ws_ptr, need)
    return y


def mx4_swiglu(x: torch.Tensor, w: Mx4Weight, out_dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """silu(x gate^T) * (x up^T) for x [..., depth] and a gated w: [..., rows], of x's type unless out_dtype or out say otherwise.
    out overlaps no other tensor of the call."""
    if not w.gated:
        raise ValueError("mx4_swiglu takes a gated weight, as mx4_quantize_gated makes it")
    m, n, ld_x, x_dt, shape, ws, ws_ptr, need = _activations(x, w)
    dtype = x.dtype if out_dtype is None and out is None else _out_dtype(out_dtype, out, x.dtype)
    y, y_ptr, ld_y, y_dt = _output(out, shape, w.rows, dtype, w.device, m)
    _call("swift_mx4_swiglu", w.device, y_ptr, ld_y, y_dt, m.data_ptr(), ld_x, x_dt, n, w.address, w.rows, w.depth, ws_ptr, need)
    return y
