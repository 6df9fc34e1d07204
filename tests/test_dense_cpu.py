"""Refusals and plans of the dense operators, on the host: the checks run before anything is
enqueued, so every error path is reached without a GPU (the pointers here are never read)."""
import ctypes

import pytest
import torch

import paper_2607_02805_amd as bd

A = 1 << 40          # made-up addresses, 1 TiB apart
X, W, OUT, RES, PRE, BIAS, WS, LAB, LOSS, LSE, GRAD, DX, DW, DB, DY = (A * i for i in range(1, 16))
BIG = 1 << 38


def desc(rows=100, k=72, n=130, dtype=bd.DTYPE_BF16, **kw):
    d = bd.DenseDesc()
    assert bd.lib().bdlm_dense_desc_init(ctypes.byref(d), rows, k, n, dtype) == 0
    for name, v in kw.items():
        setattr(d, name, v)
    return d


def projection(d, act=0, odt=1, x=X, w=W, bias=BIAS, res=RES, ldr=None, out=OUT, ldo=None, pre=PRE, ldp=None,
               ws=WS, size=BIG):
    n = d.out_features
    return bd.lib().bdlm_check_projection(ctypes.byref(d), act, odt, x, w, bias, res, n if ldr is None else ldr, out,
                                          n if ldo is None else ldo, pre, n if ldp is None else ldp, ws, size)


def backward(d, act=0, ydt=1, dy=DY, ldy=None, x=X, w=W, pre=PRE, ldp=None, dx=DX, ldx=None, dw=DW, ldw=None, db=DB,
             ws=WS, size=BIG):
    n, k = d.out_features, d.in_features
    return bd.lib().bdlm_check_projection_backward(
        ctypes.byref(d), act, ydt, dy, n if ldy is None else ldy, x, w, pre, n if ldp is None else ldp, dx,
        k if ldx is None else ldx, dw, k if ldw is None else ldw, db, ws, size)


def loss(d, labels=LAB, exclude=-1, x=X, w=W, out=LOSS, lse=LSE, ws=WS, size=BIG):
    return bd.lib().bdlm_check_head_loss(ctypes.byref(d), labels, exclude, x, w, out, lse, ws, size)


def loss_grad(d, labels=LAB, exclude=-1, x=X, w=W, out=LOSS, lse=LSE, dloss=GRAD, dx=DX, ldx=None, dw=DW, ldw=None,
              ws=WS, size=BIG):
    k = d.in_features
    return bd.lib().bdlm_check_head_loss_backward(ctypes.byref(d), labels, exclude, x, w, out, lse, dloss, dx,
                                                  k if ldx is None else ldx, dw, k if ldw is None else ldw, ws, size)


def select(d, exclude=-1, x=X, w=W, token=LAB, logprob=LOSS, ws=WS, size=BIG):
    return bd.lib().bdlm_check_head_select(ctypes.byref(d), exclude, x, w, token, logprob, ws, size)


CALLS = (projection, backward, loss, loss_grad, select)


@pytest.mark.parametrize("call", CALLS)
def test_descriptor(call):
    assert call(desc()) == bd.OK
    assert call(desc(rows=0)) == bd.OK
    for bad in (dict(rows=-1), dict(k=0), dict(n=0), dict(k=-4), dict(rows=(1 << 22) + 1), dict(k=(1 << 22) + 1),
                dict(n=(1 << 22) + 1), dict(x_stride=-1), dict(w_stride=-1), dict(x_stride=(1 << 40) + 1)):
        assert call(desc(**bad)) == bd.E_SHAPE, bad
    for bad in (dict(dtype=2), dict(dtype=-1), dict(reserved=1)):
        assert call(desc(**bad)) == bd.E_DTYPE, bad


@pytest.mark.parametrize("call", CALLS)
def test_missing_and_misaligned_inputs(call):
    d = desc()
    assert call(d, x=None) == bd.E_NULL
    assert call(d, w=None) == bd.E_NULL
    assert call(d, x=X + 8) == bd.E_ALIGN
    assert call(d, w=W + 2) == bd.E_ALIGN
    assert call(desc(rows=0), x=None) == bd.OK       # an empty tensor can have no storage
    assert call(desc(rows=200), ws=None) == bd.E_WORKSPACE
    assert call(desc(rows=200), size=255) == bd.E_WORKSPACE
    assert call(desc(rows=200), ws=WS + 128) == bd.E_ALIGN


def test_null_descriptor():
    L = bd.lib()
    n = ctypes.c_int64(0)
    assert L.bdlm_dense_desc_init(None, 1, 1, 1, 0) == bd.E_NULL
    for name in ("projection", "projection_backward", "head_loss", "head_loss_backward", "head_select"):
        f = getattr(L, f"bdlm_{name}_workspace")
        assert f(None, ctypes.byref(n)) == bd.E_NULL
        assert f(ctypes.byref(desc()), None) == bd.E_NULL
        assert f(ctypes.byref(desc(n=0)), ctypes.byref(n)) == bd.E_SHAPE


def test_projection_arguments():
    d = desc()
    n = 130
    assert projection(d, act=3) == bd.E_SHAPE and projection(d, act=-1) == bd.E_SHAPE
    assert projection(d, odt=2) == bd.E_DTYPE
    assert projection(d, out=None) == bd.E_NULL
    assert projection(d, out=OUT + 4) == bd.E_ALIGN and projection(d, res=RES + 2) == bd.E_ALIGN
    assert projection(d, pre=PRE + 8) == bd.E_ALIGN and projection(d, bias=BIAS + 2) == bd.E_ALIGN
    assert projection(d, ldo=n - 1) == bd.E_SHAPE and projection(d, ldp=n - 1) == bd.E_SHAPE
    assert projection(d, ldr=-1) == bd.E_SHAPE and projection(d, ldr=0) == bd.OK    # one row for all
    assert projection(desc(rows=1), ldo=0) == bd.OK                                  # a row has no stride
    assert projection(d, bias=None, res=None, pre=None) == bd.OK
    # overlaps
    assert projection(d, res=OUT) == bd.OK                                           # in place
    assert projection(d, res=OUT, ldr=n + 8) == bd.E_SHAPE
    assert projection(d, res=OUT + 16) == bd.E_SHAPE
    for what in ("x", "w", "bias", "pre"):
        assert projection(d, **{what: OUT}) == bd.E_SHAPE, what
    assert projection(d, pre=RES) == bd.E_SHAPE and projection(d, pre=X) == bd.E_SHAPE
    for p in (X, W, OUT, RES, PRE, BIAS):
        assert projection(d, ws=p) == bd.E_WORKSPACE
    # column slices of one matrix
    wide = desc(x_stride=400)
    assert projection(wide, out=X + 72 * 2, ldo=400, res=None, pre=None) == bd.OK
    assert projection(wide, out=X + 64 * 2, ldo=400, res=None, pre=None) == bd.E_SHAPE
    assert projection(wide, out=X + 272 * 2, ldo=400, res=None, pre=None) == bd.E_SHAPE      # into the next row
    assert projection(wide, out=X + 264 * 2, ldo=400, res=None, pre=None) == bd.OK
    # few rows need no workspace
    need = ctypes.c_int64(-1)
    assert bd.lib().bdlm_projection_workspace(ctypes.byref(desc(rows=32)), ctypes.byref(need)) == 0
    assert need.value == 0 and projection(desc(rows=32), ws=None, size=0) == bd.OK
    fp32 = desc(rows=64, dtype=bd.DTYPE_F32)
    assert bd.lib().bdlm_projection_workspace(ctypes.byref(fp32), ctypes.byref(need)) == 0 and need.value == 0


def test_backward_arguments():
    d = desc()
    assert backward(d, act=3) == bd.E_SHAPE and backward(d, ydt=7) == bd.E_DTYPE
    assert backward(d, dy=None) == bd.E_NULL and backward(d, dy=DY + 2) == bd.E_ALIGN
    assert backward(d, pre=None) == bd.OK and backward(d, act=1, pre=None) == bd.E_NULL
    assert backward(d, act=2, pre=PRE + 4) == bd.E_ALIGN
    assert backward(d, ldy=-1) == bd.E_SHAPE and backward(d, ldx=71) == bd.E_SHAPE and backward(d, ldw=71) == bd.E_SHAPE
    assert backward(d, dx=None, dw=None, db=None) == bd.OK
    assert backward(d, x=None, dw=None) == bd.OK and backward(d, w=None, dx=None) == bd.OK
    assert backward(d, db=DB + 2) == bd.E_ALIGN
    for what in ("x", "w", "dy", "dw", "db"):
        assert backward(d, **{what: DX}) == bd.E_SHAPE, what
    assert backward(d, act=1, pre=DX) == bd.E_SHAPE and backward(d, db=DY) == bd.E_SHAPE
    for p in (X, W, DY, DX, DW, DB):
        assert backward(d, ws=p) == bd.E_WORKSPACE


def test_head_arguments():
    d = desc()
    for call in (loss, loss_grad):
        assert call(d, labels=None) == bd.E_NULL and call(d, out=None) == bd.E_NULL and call(d, lse=None) == bd.E_NULL
        assert call(d, labels=LAB + 4) == bd.E_ALIGN and call(d, lse=LSE + 2) == bd.E_ALIGN
    assert loss_grad(d, dloss=None) == bd.E_NULL and loss_grad(d, ldx=71) == bd.E_SHAPE
    assert loss_grad(d, dx=None, dw=None) == bd.OK
    assert select(d, token=None) == bd.E_NULL and select(d, logprob=None) == bd.E_NULL
    assert select(d, token=LAB + 4) == bd.E_ALIGN
    one = desc(n=1)
    for call in (loss, loss_grad, select):
        assert call(one) == bd.OK and call(one, exclude=1) == bd.OK and call(one, exclude=0) == bd.E_SHAPE
    assert loss(d, out=LAB) == bd.E_SHAPE and loss(d, lse=LOSS) == bd.E_SHAPE
    assert loss_grad(d, dx=DW) == bd.E_SHAPE and loss_grad(d, dw=LAB) == bd.E_SHAPE
    assert select(d, token=X) == bd.E_SHAPE and select(d, logprob=LAB) == bd.E_SHAPE


@pytest.mark.parametrize("dtype", [bd.DTYPE_F32, bd.DTYPE_BF16])
def test_workspace_sizes(dtype):
    """Sizes are non-negative multiples of 256, and none overflows at the largest sizes."""
    need = ctypes.c_int64(0)
    top = 1 << 22
    for rows in (0, 1, 64, 65, 4096, top):
        for k in (1, 72, 1024, top):
            for n in (1, 130, 50257, top):
                d = desc(rows, k, n, dtype)
                for name in ("projection", "projection_backward", "head_loss", "head_loss_backward", "head_select"):
                    assert getattr(bd.lib(), f"bdlm_{name}_workspace")(ctypes.byref(d), ctypes.byref(need)) == 0
                    assert need.value >= 0 and need.value % 256 == 0, (name, rows, k, n, need.value)


def test_products_that_fit_no_launch():
    """2^23 large tiles are 2^32 threads, one more than a launch holds."""
    edge = (1 << 23) // (1 << 14)          # 2^22 rows are 2^14 tiles; this many tiles of columns are too many
    wide = desc(rows=1 << 22, k=64, n=256 * edge)
    for call in (projection, loss, select):
        assert call(wide, size=1 << 39) == bd.E_SHAPE
        assert call(desc(rows=1 << 22, k=64, n=256 * (edge - 1)), size=1 << 39) == bd.OK


def test_python_refusals():
    x, w = torch.zeros(3, 8), torch.zeros(5, 8)
    with pytest.raises(ValueError, match="GPU"):
        bd.projection(x, w)
    for call, match in ((lambda: bd.projection(x, w.bfloat16()), "dtype"), (lambda: bd.projection(x, w[:, :4]), "shape"),
                        (lambda: bd.projection(x.half(), w.half()), "bfloat16 or float32"),
                        (lambda: bd.projection(x, w, act="relu"), "act must"),
                        (lambda: bd.projection(x, w.t().contiguous().t()), "unit stride"),
                        (lambda: bd.projection(x, w, torch.zeros(4)), "bias"),
                        (lambda: bd.projection(x, w, residual=torch.zeros(3, 4)), "residual"),
                        (lambda: bd.projection(x, w, out=torch.zeros(3, 5), residual=torch.zeros(3, 5).bfloat16()),
                         "residual"),
                        (lambda: bd.projection_backward(torch.zeros(3, 5), x, w, act="silu"), "pre is needed"),
                        (lambda: bd.projection_backward(torch.zeros(3, 4), x, w), "dy"),
                        (lambda: bd.projection_backward(torch.zeros(3, 5), x, w, dx=torch.zeros(3, 9)), "dx"),
                        (lambda: bd.head_loss(x, w, torch.zeros(3)), "labels"),
                        (lambda: bd.head_loss(x, w, torch.zeros(4, dtype=torch.int64)), "labels"),
                        (lambda: bd.head_select(x, w, token=torch.zeros(3)), "token")):
        with pytest.raises(ValueError, match=match):
            call()


def test_overlaps_of_the_widest_matrices():
    """2^22 rows 2^40 elements apart reach past 2^63 bytes: what lies between them is still seen."""
    far = desc(rows=1 << 22, k=64, n=130, dtype=bd.DTYPE_F32, x_stride=1 << 40)
    assert projection(far, x=X) == bd.E_SHAPE                             # out, pre: above x's first row
    assert projection(far, x=DY) == bd.OK                                 # all below it
    assert projection(far, x=DY, out=DY + A) == bd.E_SHAPE
    assert select(far, x=X) == bd.E_SHAPE and select(far, x=DY) == bd.OK
    assert select(far, x=DY, token=DY + A) == bd.E_SHAPE and select(far, x=DY, ws=DY + A) == bd.E_WORKSPACE
    d = desc(rows=1 << 22, k=64, n=130, dtype=bd.DTYPE_F32)
    assert projection(d, res=DY, ldr=1 << 40) == bd.OK
    assert projection(d, res=DY, ldr=1 << 40, out=DY + A) == bd.E_SHAPE


@pytest.mark.parametrize("exclude", [-1, 5, 4, 0, 2 ** 64, 2 ** 64 + 3, -2 ** 64 + 3, 2 ** 63, -2 ** 63 - 1, 2 ** 40])
def test_any_integer_may_be_excluded(monkeypatch, exclude):
    """A token past the vocabulary is none of it, however large: it does not come out as another one."""
    seen = []
    monkeypatch.setattr(bd, "_dense_call", lambda name, d, device, workspace, args: seen.append(args))
    x, w, v = torch.zeros(3, 8), torch.zeros(5, 8), torch.zeros(3)
    labels = torch.zeros(3, dtype=torch.int64)
    bd.head_select(x, w, exclude=exclude)
    bd.head_loss(x, w, labels, exclude=exclude)
    bd.head_loss_backward(v, x, w, labels, v, v, exclude=exclude)
    for args, at in zip(seen, (0, 1, 1)):
        got = ctypes.c_int64(args[at]).value
        assert got == exclude if 0 <= exclude < 5 else not 0 <= got < 5, (args, got)
