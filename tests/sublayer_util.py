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


def gated64(x, w_gate, w_up, bias_gate=None, bias_up=None, act=None, out_dtype=None):
    """((out, tol), (gate, tol), (up, tol)): the products as tests/dense_util.py bounds them; out from the unrounded ones,
    the activation within 16 steps of fp32 at the size of its argument."""
    ty, ot = x.dtype, out_dtype or x.dtype
    x = du.rows2(du.d64(x))
    k = x.shape[1]
    got = []
    for w, b in ((w_gate, bias_gate), (w_up, bias_up)):
        w, b = du.d64(w), du.d64(b)
        z, mag = x @ w.t(), x.abs() @ w.abs().t()
        if b is not None:
            z, mag = z + b, mag + b.abs()
        got.append((z, (k + 8) * F * mag))
    (g, eg), (u, eu) = got
    a = du.act64(g, act)
    ea = eg if act in (None, "none") else 1.13 * eg + 16 * F * g.abs()
    out = a * u
    eo = ea * u.abs() + (a.abs() + ea) * eu + 2 * F * out.abs()
    return ((out, eo + U[ot] * (out.abs() + eo) + 1e-37), (g, eg + U[ty] * (g.abs() + eg) + 1e-37),
            (u, eu + U[ty] * (u.abs() + eu) + 1e-37))


def gated_backward64(dh, x, w_gate, w_up, gate, up, act=None):
    """((dx, tol), (dw_gate, tol), (dw_up, tol), (db_gate, tol), (db_up, tol))."""
    ty = x.dtype
    dh, x, gate, up = (du.rows2(du.d64(t)) for t in (dh, x, gate, up))
    wg, wu = du.d64(w_gate), du.d64(w_up)
    m, n = dh.shape
    plain = act in (None, "none")
    dg = dh * up * (1.0 if plain else du.slope64(gate, act))
    d_up = dh * du.act64(gate, act)
    sg = (dh * up).abs() * (1.0 if plain else 1.13)
    s_up = (dh * gate).abs()
    rnd = U[ty] if ty == torch.bfloat16 else 0.0
    eg, e_up = 18 * F * sg + rnd * dg.abs(), 18 * F * s_up + rnd * d_up.abs()
    dx = dg @ wg + d_up @ wu
    ex = (eg + (2 * n + 8) * F * sg) @ wg.abs() + (e_up + (2 * n + 8) * F * s_up) @ wu.abs()
    out = [(dx, ex + U[ty] * (dx.abs() + ex) + 1e-37)]
    for d, e, s in ((dg, eg, sg), (d_up, e_up, s_up)):
        dw, ew = d.t() @ x, (e + (m + 8) * F * s).t() @ x.abs()
        out.append((dw, ew + U[ty] * (dw.abs() + ew) + 1e-37))
    for d, s in ((dg, sg), (d_up, s_up)):
        db, eb = d.sum(0), ((m + 26) * F * s).sum(0)
        out.append((db, eb + F * db.abs() + 1e-37))
    return out
