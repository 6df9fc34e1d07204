"""Plain forms of the dense operators in 64 bits, and the error each output may have.

Bounds are derived from the operators' arithmetic, element by element, before any comparison:

* a stored value is rounded once: half a step, ``eps(dtype) / 2`` of its size (bf16 2^-8, fp32
  2^-24);
* a product's sum over K indices in fp32 is off by at most ``(K + 8) 2^-24`` of the sum of the
  absolute products, whatever the order (bf16 operands multiply exactly; fp32 ones as three
  terms each leave out less than 2^-24 of every product, which the 8 holds with the joins);
* an activation changes an error of its argument by its slope, at most 1.13, and is itself
  evaluated within 16 steps of fp32 at the size of its argument;
* with bf16 inputs a gradient's first operand (dz, or the logits' gradients P) is rounded to bf16,
  half a step of each element;
* the logits' error is carried by a softmax without being enlarged, and exp of an argument d is
  off by (4 + |d|) 2^-23 of itself.
"""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
F = 2.0 ** -24


def act64(z, act):
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    return z


def slope64(z, act):
    if act == "silu":
        s = torch.sigmoid(z)
        return s + z * s * (1 - s)
    if act == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return torch.ones_like(z)


def d64(t):
    return None if t is None else t.detach().double().cpu()


def rows2(t):
    return t.reshape(-1, t.shape[-1])


def projection64(x, w, bias=None, act=None, residual=None, out_dtype=None):
    """(out, pre) with their bounds, as ((out, tol), (pre, tol))."""
    ty, ot = x.dtype, out_dtype or x.dtype
    x, w, bias, residual = rows2(d64(x)), d64(w), d64(bias), d64(residual)
    k = x.shape[1]
    z = x @ w.t()
    mag = x.abs() @ w.abs().t()
    if bias is not None:
        z = z + bias
        mag = mag + bias.abs()
    e = (k + 8) * F * mag
    out = act64(z, act)
    eo = e if act in (None, "none") else 1.13 * e + 16 * F * z.abs()
    if residual is not None:
        out = out + rows2(residual)
        eo = eo + F * (out.abs() + rows2(residual).abs())
    return (out, eo + U[ot] * (out.abs() + eo) + 1e-37), (z, e + U[ty] * (z.abs() + e) + 1e-37)


def projection_backward64(dy, x, w, pre=None, act=None):
    ty = x.dtype
    dy, x, w, pre = rows2(d64(dy)), rows2(d64(x)), d64(w), d64(pre)
    dz = dy if pre is None or act in (None, "none") else dy * slope64(rows2(pre), act)
    size = dy.abs() if pre is None or act in (None, "none") else dy.abs() * 1.13
    e = 16 * F * size + (U[ty] * dz.abs() if ty == torch.bfloat16 else 0.0)
    m, n = dz.shape
    dx, dw, db = dz @ w, dz.t() @ x, dz.sum(0)
    ex = (e + (n + 8) * F * size) @ w.abs()
    ew = (e + (m + 8) * F * size).t() @ x.abs()
    eb = ((m + 24) * F * size).sum(0)
    return ((dx, ex + U[ty] * (dx.abs() + ex) + 1e-37), (dw, ew + U[ty] * (dw.abs() + ew) + 1e-37),
            (db, eb + F * db.abs() + 1e-37))


def head64(x, w, exclude=-1):
    """Logits in 64 bits (excluded ones -inf) and the bound of a logit of each row."""
    x, w = rows2(d64(x)), d64(w)
    k = x.shape[1]
    l = x @ w.t()
    e = ((k + 8) * F * (x.abs() @ w.abs().t())).max(1, keepdim=True).values
    if 0 <= exclude < w.shape[0]:
        l[:, exclude] = -math.inf
    return l, e


def counted(labels, vocab, exclude):
    labels = labels.reshape(-1).cpu()
    return (labels >= 0) & (labels < vocab) & (labels != exclude)


def head_loss64(x, w, labels, exclude=-1):
    l, e = head64(x, w, exclude)
    ok = counted(labels, w.shape[0], exclude)
    lab = torch.where(ok, labels.reshape(-1).cpu(), 0)
    lse = torch.logsumexp(l, 1)
    loss = lse - l.gather(1, lab[:, None])[:, 0]
    loss = torch.where(ok, loss, 0.0)
    lse = torch.where(ok, lse, 0.0)
    d = (l.max(1).values - torch.where(l.isinf(), math.inf, l).min(1).values)
    n = l.shape[1]
    tol = 2 * e[:, 0] + (8 + d + math.sqrt(n)) * 2 * F + 4 * F * (loss.abs() + lse.abs() + l.max(1).values.abs())
    return (loss, tol), (lse, tol)


def head_loss_backward64(dloss, x, w, labels, exclude=-1):
    ty = x.dtype
    l, e = head64(x, w, exclude)
    ok = counted(labels, w.shape[0], exclude)
    lab = torch.where(ok, labels.reshape(-1).cpu(), 0)
    p = torch.softmax(l, 1)
    hot = torch.zeros_like(p).scatter_(1, lab[:, None], 1.0)
    g = torch.where(ok, d64(dloss).reshape(-1), 0.0)[:, None]
    # a logit's error moves its probability by that share of it; the label's is 1 - p of the same
    (_, tl), _ = head_loss64(x, w, labels, exclude)
    far = torch.where(l.isinf(), 0.0, (l - torch.logsumexp(l, 1, keepdim=True)).abs())
    size = torch.where(hot > 0, 1 - p, p) * g.abs()
    P = (p - hot) * g
    dp = p * g.abs() * (e + tl[:, None] + (8 + far) * 2 * F) + 8 * F * size
    if ty == torch.bfloat16:
        dp = dp + U[ty] * (P.abs() + dp)
    x, w = rows2(d64(x)), d64(w)
    m, n = P.shape
    dpw = dp
    if ty == torch.bfloat16 and m > 64:
        # dw's product is of P / h and h x, h the label's entry, each rounded to half a step u: together
        # (1 + u)^2 - 1 = 2 u + u^2 of a product (the label's own, of 1 and h x, less), u of it is in dp
        dpw = dp + (U[ty] + U[ty] ** 2) * (P.abs() + dp)
    dx, dw = P @ w, P.t() @ x
    ex = (dp + (n + 8) * F * P.abs()) @ w.abs()
    ew = (dpw + (m + 8) * F * P.abs()).t() @ x.abs()
    return (dx, ex + U[ty] * (dx.abs() + ex) + 1e-37), (dw, ew + U[ty] * (dw.abs() + ew) + 1e-37)


def worst(got, want):
    """The largest error of ``got`` as a share of its bound; infinite where one side is not finite."""
    ref, tol = want
    g = got.detach().double().cpu().reshape(ref.shape)
    if g.numel() == 0:
        return 0.0
    if not bool(torch.isfinite(g).all()):
        return math.inf
    return float(((g - ref).abs() / tol).max())
