"""MXFP4 and the products with it in 64 bits, written from the format's definition: what the tests compare with."""
import numpy as np
import torch

BLOCK = 32
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def values(w: torch.Tensor) -> torch.Tensor:
    """What w [rows, depth] stands for once quantised, as float64 on the CPU (blocks with an infinity or a NaN: NaN)."""
    v = w.detach().cpu().to(torch.float64).numpy()
    rows, depth = v.shape
    out = np.empty_like(v)
    for k in range(0, depth, BLOCK):
        b = v[:, k:k + BLOCK]
        top = np.abs(b).max(axis=1)
        ok = np.isfinite(b).all(axis=1)
        _, p = np.frexp(np.where(ok, top, 1.0))            # top = f 2^p, f in [1/2, 1): floor(log2 top) = p - 1
        scale = np.ldexp(1.0, np.where(top > 0, np.maximum(p - 3, -127), -127))[:, None]
        q = np.abs(np.where(ok[:, None], b, 0.0)) / scale
        # nearest grid point; of two equally near ones the one at an even place of the grid
        d = np.abs(q[..., None] - GRID)
        near = d == d.min(axis=-1, keepdims=True)
        first, last = near.argmax(axis=-1), len(GRID) - 1 - near[..., ::-1].argmax(axis=-1)
        code = np.where(first % 2 == 0, first, last)
        out[:, k:k + BLOCK] = np.where(ok[:, None], np.copysign(GRID[code], b) * scale, np.nan)
    return torch.from_numpy(out)


def linear(x, w, residual=None):
    """(x w^T + residual, sum of |products|): w as float64 values."""
    xd, wd = x.detach().cpu().double(), w.double()
    y = xd @ wd.t()
    return (y if residual is None else y + residual.detach().cpu().double()), xd.abs() @ wd.abs().t()


def linear_bound(y, size, depth, terms, out_dtype):
    """How far a product may be off: at most depth * terms additions in fp32, each off by at most a step (2^-23: the matrix cores may cut off)
    of a partial sum that is no larger than the sum of the magnitudes, with signs that do not agree: their root, four times over; then
    the result's own rounding (half a step) and the residual's addition."""
    acc = 4.0 * (depth * terms + 16) ** 0.5 * 2.0 ** -23 * size + 2.0 ** -24 * y.abs()
    return acc + (2.0 ** -8 * (y.abs() + acc) if out_dtype == torch.bfloat16 else 0.0)


def swiglu(x, gate, up):
    """(h, g, u, sums of the magnitudes of both)."""
    g, gs = linear(x, gate)
    u, us = linear(x, up)
    return g / (1.0 + torch.exp(-g)) * u, g, u, gs, us


def swiglu_bound(h, g, u, gs, us, depth, terms, out_dtype):
    """The products' errors through silu(g) u (silu is 1.1-Lipschitz), and the arithmetic of silu in fp32: an exponential of an argument
    below 100 in magnitude wherever the result counts (its rounding moves the exponential by |g| 2^-24), an addition, a division, a
    product, each off by a few steps."""
    dg, du = linear_bound(g, gs, depth, terms, torch.float32), linear_bound(u, us, depth, terms, torch.float32)
    s = g / (1.0 + torch.exp(-g))
    acc = 1.1 * dg * (u.abs() + du) + s.abs() * du + h.abs() * (g.abs().clamp(max=100.0) + 16.0) * 2.0 ** -23
    return acc + (2.0 ** -8 * (h.abs() + acc) if out_dtype == torch.bfloat16 else 0.0) + 1e-37
