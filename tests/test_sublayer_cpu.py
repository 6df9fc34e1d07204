"""Refusals of a sublayer's operators, on the host: the checks run before anything is enqueued, so every
error path is reached without a GPU (the pointers here are never read)."""
import ctypes

import pytest
import torch

import paper_2607_02805_amd as bd

A = 1 << 40          # made-up addresses, 1 TiB apart
X, RES, SUM, W, OUT, SCALE, DY, DT, DS, DW, WS = (A * i for i in range(1, 12))
BIG = 1 << 38
F32, BF, E4 = bd.DTYPE_F32, bd.DTYPE_BF16, bd.DTYPE_E4M3


def norm(rows=100, n=200, xt=BF, x=X, ldx=200, rt=BF, res=RES, ldr=200, sum_=SUM, lds=200, w=W, eps=1e-5, ot=BF, out=OUT,
         ldo=200, scale=None, block=0):
    return bd.lib().bdlm_check_add_rmsnorm(rows, n, xt, x, ldx, rt, res, ldr, sum_, lds, w, eps, ot, out, ldo, scale, block)


def grad(rows=100, n=200, yt=BF, dy=DY, ldy=200, st=BF, s=X, lds=200, w=W, eps=1e-5, dt=BF, dsum=DT, ldt=200, ds=DS,
         ldd=200, dw=DW, ws=WS, size=BIG):
    return bd.lib().bdlm_check_add_rmsnorm_backward(rows, n, yt, dy, ldy, st, s, lds, w, eps, dt, dsum, ldt, ds, ldd, dw, ws,
                                                    size)


@pytest.mark.parametrize("call", [norm, grad])
def test_norm_sizes(call):
    assert call() == bd.OK
    for bad in (dict(rows=-1), dict(n=0), dict(n=-3), dict(rows=(1 << 22) + 1), dict(n=(1 << 22) + 1), dict(eps=-1e-9),
                dict(eps=float("nan")), dict(eps=float("inf"))):
        assert call(**bad) == bd.E_SHAPE, bad
    assert call(w=None) == bd.E_NULL and call(w=W + 4) == bd.E_ALIGN


def test_norm_arguments():
    assert norm(xt=2) == bd.E_DTYPE and norm(rt=7) == bd.E_DTYPE and norm(ot=3) == bd.E_DTYPE and norm(ot=-1) == bd.E_DTYPE
    assert norm(rt=7, res=None, sum_=None) == bd.OK            # not read
    assert norm(x=None) == bd.E_NULL and norm(out=None) == bd.E_NULL and norm(res=None) == bd.E_NULL
    for p in ("x", "res", "sum_", "out"):
        assert norm(**{p: dict(x=X, res=RES, sum_=SUM, out=OUT)[p] + 8}) == bd.E_ALIGN, p
    for ld in ("ldx", "ldr", "lds", "ldo"):
        assert norm(**{ld: -1}) == bd.E_SHAPE and norm(**{ld: (1 << 40) + 1}) == bd.E_SHAPE, ld
    assert norm(ldo=199) == bd.E_SHAPE and norm(lds=199) == bd.E_SHAPE and norm(ldx=0, ldr=0) == bd.OK
    assert norm(rows=0, x=None, res=None, sum_=None, out=None, w=None) == bd.OK
    # 8 bits
    assert norm(ot=E4) == bd.E_NULL and norm(ot=E4, scale=SCALE) == bd.OK and norm(ot=E4, scale=SCALE, block=128) == bd.OK
    assert norm(ot=E4, scale=SCALE, block=64) == bd.E_SHAPE and norm(block=128) == bd.E_SHAPE
    assert norm(ot=E4, scale=SCALE + 2) == bd.E_ALIGN
    # in place, and overlaps
    assert norm(out=X) == bd.OK and norm(sum_=RES) == bd.OK
    assert norm(out=X, ldo=208) == bd.E_SHAPE and norm(out=X, xt=F32) == bd.E_SHAPE and norm(out=X + 16) == bd.E_SHAPE
    assert norm(out=X, ldx=0, ldo=0) == bd.E_SHAPE
    assert norm(sum_=RES, lds=208) == bd.E_SHAPE and norm(sum_=RES + 32) == bd.E_SHAPE
    for p in (RES, SUM, W):
        assert norm(out=p) == bd.E_SHAPE
    assert norm(sum_=X) == bd.E_SHAPE and norm(sum_=W) == bd.E_SHAPE
    for p in (X, RES, SUM, W, OUT):
        assert norm(ot=E4, scale=p) == bd.E_SHAPE
    # column slices of one matrix
    assert norm(ldx=400, out=X + 400, ldo=400) == bd.OK and norm(ldx=400, out=X + 384, ldo=400) == bd.E_SHAPE


def test_norm_backward_arguments():
    for t in ("yt", "st", "dt"):
        assert grad(**{t: E4}) == bd.E_DTYPE
    assert grad(dy=None) == bd.E_NULL and grad(s=None) == bd.E_NULL and grad(dsum=None) == bd.OK
    assert grad(ds=None, dw=None, ws=None, size=0) == bd.OK and grad(dw=None, ws=None, size=0) == bd.OK
    for p, at in (("dy", DY), ("s", X), ("dsum", DT), ("ds", DS)):
        assert grad(**{p: at + 8}) == bd.E_ALIGN, p
    assert grad(dw=DW + 2) == bd.E_ALIGN
    assert grad(ldd=199) == bd.E_SHAPE and grad(ldy=-1) == bd.E_SHAPE and grad(ldt=-1) == bd.E_SHAPE
    assert grad(ws=None) == bd.E_WORKSPACE and grad(size=99) == bd.E_WORKSPACE and grad(ws=WS + 64) == bd.E_ALIGN
    assert grad(ds=DT) == bd.OK and grad(ds=DT, ldd=208) == bd.E_SHAPE and grad(ds=DY) == bd.E_SHAPE
    for p in (X, W, DW):
        assert grad(ds=p) == bd.E_SHAPE
    for p in (X, DY, DT, W):
        assert grad(dw=p) == bd.E_SHAPE
    for p in (X, DY, DT, W, DS, DW):
        assert grad(ws=p) == bd.E_WORKSPACE
    n = ctypes.c_int64(-1)
    f = bd.lib().bdlm_add_rmsnorm_backward_workspace
    assert f(100, 200, None) == bd.E_NULL and f(-1, 200, ctypes.byref(n)) == bd.E_SHAPE and f(1, 0, ctypes.byref(n)) == bd.E_SHAPE
    assert f(100, 200, ctypes.byref(n)) == bd.OK and grad(size=n.value) == bd.OK and grad(size=n.value - 1) == bd.E_WORKSPACE
    assert f(0, 200, ctypes.byref(n)) == bd.OK and n.value == 0


def test_norm_binding_refuses():
    x, w = torch.zeros(4, 8), torch.ones(8)
    for call in (lambda: bd.add_rmsnorm(x, w), lambda: bd.add_rmsnorm_backward(x, x, w)):
        with pytest.raises(ValueError, match="GPU"):
            call()
