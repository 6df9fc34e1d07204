"""Plain forms of a sublayer's norm and gated product in 64 bits, and the error each output may have.

Beside the bounds of tests/dense_util.py (F = 2^-24, a rounding is half a step):

* a sum of squares over `width` columns goes in runs of at most max(32, width / 256) in a lane, then through at most 12
  additions of partial sums; its terms are positive, so its relative error is at most that many F, half of it in a
  root, and the formation of s, the root, the division and the products with rstd and w add fewer than 12 F: `near(width)`;
* a value in e4m3 is off by 2^-4 of itself, or 2^-10 below the smallest normal one, in units of its scale;
* the dot product of the gradient has the same runs, each term off by near(width) and its own products' roundings.
"""
import torch

from tests import dense_util as du

F = 2.0 ** -24
U = {**du.U, torch.float8_e4m3fn: 2.0 ** -4}


def near(width):
    return (max(32, width / 256) / 2 + 18) * F


def norm64(x, w, residual=None, eps=1e-5):
    """(y, s) in 64 bits."""
    s = du.rows2(du.d64(x))
    if residual is not None:
        s = s + du.rows2(du.d64(residual))
    return s / torch.sqrt((s * s).mean(1, keepdim=True) + eps) * du.d64(w), s


def norm_bounds(x, w, residual=None, eps=1e-5, out_dtype=torch.float32):
    """((y, tol), (s, tol)): s in the residual's type.  Rounding x + residual to fp32 is off by F of s, in y as well."""
    y, s = norm64(x, w, residual, eps)
    e = near(s.shape[1])
    sum_tol = (F + U[residual.dtype]) * s.abs() + 1e-37 if residual is not None else None
    return (y, (e + U[out_dtype]) * y.abs() + 1e-37), (s, sum_tol)


def scales64(y, block):
    step = block or y.shape[1]
    top = torch.stack([c.abs().max(1).values for c in y.split(step, 1)], 1)
    return torch.where(top > 0, top / 448, 1.0)


def norm_grad64(dy, s, w, dsum=None, eps=1e-5, ds_dtype=torch.float32):
    """((ds, tol), (dw, tol))."""
    dy, s, w = du.rows2(du.d64(dy)), du.rows2(du.d64(s)), du.d64(w)
    m, width = s.shape
    rstd = 1 / torch.sqrt((s * s).mean(1, keepdim=True) + eps)
    n, dn = s * rstd, dy * w
    dot = (n * dn).mean(1, keepdim=True)
    ds = rstd * (dn - n * dot)
    e = near(width)
    e_dot = (2 * e + (max(32, width / 256) + 16) * F) * (n * dn).abs().mean(1, keepdim=True)
    tol = rstd * ((2 * e + 4 * F) * (dn.abs() + (n * dot).abs()) + n.abs() * e_dot)
    if dsum is not None:
        ds = ds + du.rows2(du.d64(dsum))
        tol = tol + F * ds.abs()
    dw = (dy * n).sum(0)
    tol_w = (e + (m + 24) * F) * (dy * n).abs().sum(0)
    return (ds, tol + U[ds_dtype] * (ds.abs() + tol) + 1e-37), (dw, tol_w + F * dw.abs() + 1e-37)
