"""Refusals of a sublayer's operators and of the head's log-probabilities, on the host: the checks run before anything is enqueued, so every
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


WG, WU, BG, BU, PG, PU, DWG, DWU, DBG, DBU, DX = (A * i for i in range(20, 31))


def desc(rows=100, k=72, n=130, dtype=BF, **kw):
    d = bd.DenseDesc()
    assert bd.lib().bdlm_dense_desc_init(ctypes.byref(d), rows, k, n, dtype) == 0
    for name, v in kw.items():
        setattr(d, name, v)
    return d


def gated(d, act=1, ot=BF, x=X, wg=WG, wu=WU, bg=BG, bu=BU, out=OUT, ldo=None, pg=PG, pu=PU, ldp=None, ws=WS, size=BIG):
    n = d.out_features
    return bd.lib().bdlm_check_gated_projection(ctypes.byref(d), act, ot, x, wg, wu, bg, bu, out, n if ldo is None else ldo,
                                                pg, pu, n if ldp is None else ldp, ws, size)


def gated_grad(d, act=1, ht=BF, dh=DY, ldh=None, x=X, wg=WG, wu=WU, pg=PG, pu=PU, ldp=None, dx=DX, ldx=None, dwg=DWG,
               dwu=DWU, ldw=None, dbg=DBG, dbu=DBU, ws=WS, size=BIG):
    n, k = d.out_features, d.in_features
    return bd.lib().bdlm_check_gated_projection_backward(
        ctypes.byref(d), act, ht, dh, n if ldh is None else ldh, x, wg, wu, pg, pu, n if ldp is None else ldp, dx,
        k if ldx is None else ldx, dwg, dwu, k if ldw is None else ldw, dbg, dbu, ws, size)


@pytest.mark.parametrize("call", [gated, gated_grad])
def test_gated_descriptor(call):
    assert call(desc()) == bd.OK and call(desc(rows=0), x=None) == bd.OK
    for bad in (dict(rows=-1), dict(k=0), dict(n=0), dict(rows=(1 << 22) + 1), dict(k=(1 << 22) + 1), dict(n=(1 << 22) + 1),
                dict(x_stride=-1), dict(w_stride=-1), dict(w_stride=(1 << 40) + 1)):
        assert call(desc(**bad)) == bd.E_SHAPE, bad
    for bad in (dict(dtype=2), dict(reserved=1)):
        assert call(desc(**bad)) == bd.E_DTYPE, bad
    d = desc(rows=200)
    for p in ("x", "wg", "wu"):
        assert call(d, **{p: None}) == bd.E_NULL and call(d, **{p: X * 40 + 8}) == bd.E_ALIGN, p
    assert call(d, act=3) == bd.E_SHAPE and call(d, act=-1) == bd.E_SHAPE
    assert call(d, ws=None) == bd.E_WORKSPACE and call(d, size=255) == bd.E_WORKSPACE and call(d, ws=WS + 64) == bd.E_ALIGN
    # more threads than a launch holds
    assert call(desc(rows=1 << 22, k=64, n=1 << 22), size=1 << 62) == bd.E_SHAPE


def test_gated_arguments():
    d = desc()
    assert gated(d, ot=2) == bd.E_DTYPE and gated(d, out=None) == bd.E_NULL and gated(d, out=OUT + 8) == bd.E_ALIGN
    assert gated(d, pg=None) == bd.E_NULL and gated(d, pu=None) == bd.E_NULL and gated(d, pg=None, pu=None) == bd.OK
    assert gated(d, bg=None, bu=None) == bd.OK and gated(d, bg=BG + 2) == bd.E_ALIGN and gated(d, bu=BU + 1) == bd.E_ALIGN
    assert gated(d, ldo=129) == bd.E_SHAPE and gated(d, ldp=129) == bd.E_SHAPE
    assert gated(d, wu=WG) == bd.OK                             # the same weights twice
    for p in (X, WG, WU, BG, BU, PG, PU):
        assert gated(d, out=p) == bd.E_SHAPE
    assert gated(d, pg=PU) == bd.E_SHAPE and gated(d, pu=X) == bd.E_SHAPE
    assert gated(d, pu=PG + 130 * 2 + 12, ldp=400) == bd.OK and gated(d, pu=PG + 96 * 2, ldp=400) == bd.E_SHAPE
    for p in (X, WG, WU, BG, BU, PG, PU, OUT):
        assert gated(d, ws=p) == bd.E_WORKSPACE
    need = ctypes.c_int64(-1)
    f = bd.lib().bdlm_gated_projection_workspace
    assert f(ctypes.byref(desc(rows=32)), ctypes.byref(need)) == 0 and need.value == 0
    assert gated(desc(rows=32), ws=None, size=0) == bd.OK
    assert f(None, ctypes.byref(need)) == bd.E_NULL and f(ctypes.byref(d), None) == bd.E_NULL
    assert f(ctypes.byref(d), ctypes.byref(need)) == 0
    assert gated(d, size=need.value) == bd.OK and gated(d, size=need.value - 1) == bd.E_WORKSPACE


def test_gated_backward_arguments():
    d = desc()
    assert gated_grad(d, ht=2) == bd.E_DTYPE
    for p in ("dh", "pg", "pu"):
        assert gated_grad(d, **{p: None}) == bd.E_NULL and gated_grad(d, **{p: A * 50 + 8}) == bd.E_ALIGN, p
    assert gated_grad(d, act=0, pg=None) == bd.E_NULL           # the product needs them without an activation too
    assert gated_grad(d, x=None, dwg=None, dwu=None) == bd.OK and gated_grad(d, wg=None, wu=None, dx=None) == bd.OK
    assert gated_grad(d, dx=None, dwg=None, dwu=None, dbg=None, dbu=None) == bd.OK
    assert gated_grad(d, ldx=71) == bd.E_SHAPE and gated_grad(d, ldw=71) == bd.E_SHAPE and gated_grad(d, ldh=-1) == bd.E_SHAPE
    assert gated_grad(d, dbg=DBG + 2) == bd.E_ALIGN and gated_grad(d, dwu=DWU + 8) == bd.E_ALIGN
    outs = ("dx", "dwg", "dwu", "dbg", "dbu")
    at = dict(dx=DX, dwg=DWG, dwu=DWU, dbg=DBG, dbu=DBU)
    for o in outs:
        for p in (X, WG, WU, DY, PG, PU):
            assert gated_grad(d, **{o: p}) == bd.E_SHAPE, o
        for other in outs:
            if other != o:
                assert gated_grad(d, **{o: at[other]}) == bd.E_SHAPE, (o, other)
        assert gated_grad(d, ws=at[o]) == bd.E_WORKSPACE


def test_gated_binding_refuses():
    x, w = torch.zeros(4, 8), torch.ones(6, 8)
    pre = (torch.zeros(4, 6), torch.zeros(4, 6))
    for call in (lambda: bd.gated_projection(x, w, w), lambda: bd.gated_projection_backward(pre[0], x, w, w, pre)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    wide = torch.ones(6, 16)[:, :8]
    for bad in (lambda: bd.gated_projection(x, w, wide), lambda: bd.gated_projection(x, w, w[:5]),
                lambda: bd.gated_projection(x, w, w.bfloat16()), lambda: bd.gated_projection(x, w, w, act="relu"),
                lambda: bd.gated_projection(x, w, w, pre=pre[0]), lambda: bd.gated_projection(x, w, w, pre=(pre[0], True)),
                lambda: bd.gated_projection(x, w, w, pre=(pre[0], torch.zeros(4, 9)[:, :6])),
                lambda: bd.gated_projection_backward(pre[0], x, w, w, None),
                lambda: bd.gated_projection_backward(pre[0], x, w, w, pre, dw_gate=torch.zeros(6, 9)[:, :8])):
        with pytest.raises(ValueError):
            bad()


TOK, LP, ENT, TT, TL = (A * i for i in range(40, 45))


def logprobs(d, tokens=TOK, exclude=-1, top=4, x=X, w=W, lp=LP, ent=ENT, tt=TT, tl=TL, ws=WS, size=BIG):
    return bd.lib().bdlm_check_head_logprobs(ctypes.byref(d), tokens, exclude, top, x, w, lp, ent, tt, tl, ws, size)


def test_logprobs_arguments():
    d = desc()
    assert logprobs(d) == bd.OK and logprobs(desc(rows=0), tokens=None, lp=None, tt=None, tl=None, x=None) == bd.OK
    for bad in (dict(rows=-1), dict(k=0), dict(n=0), dict(rows=(1 << 22) + 1), dict(n=(1 << 22) + 1), dict(x_stride=-1)):
        assert logprobs(desc(**bad), top=0) == bd.E_SHAPE, bad
    assert logprobs(desc(dtype=2)) == bd.E_DTYPE
    assert logprobs(d, x=None) == bd.E_NULL and logprobs(d, w=W + 2) == bd.E_ALIGN
    assert logprobs(d, tokens=None) == bd.E_NULL and logprobs(d, lp=None) == bd.E_NULL
    assert logprobs(d, tokens=None, lp=None) == bd.OK and logprobs(d, ent=None) == bd.OK
    assert logprobs(d, tt=None) == bd.E_NULL and logprobs(d, tl=None) == bd.E_NULL
    assert logprobs(d, top=0, tt=None, tl=None) == bd.OK
    assert logprobs(d, top=-1) == bd.E_SHAPE and logprobs(d, top=17) == bd.E_SHAPE and logprobs(d, top=16) == bd.OK
    few = desc(n=5)
    assert logprobs(few, top=5) == bd.OK and logprobs(few, top=6) == bd.E_SHAPE and logprobs(few, top=5, exclude=1) == bd.E_SHAPE
    assert logprobs(few, top=5, exclude=5) == bd.OK and logprobs(desc(n=1), exclude=0, top=0) == bd.E_SHAPE
    for p, at in (("tokens", TOK + 4), ("lp", LP + 2), ("ent", ENT + 1), ("tt", TT + 4), ("tl", TL + 2)):
        assert logprobs(d, **{p: at}) == bd.E_ALIGN, p
    ins, outs = dict(x=X, w=W, tokens=TOK), dict(lp=LP, ent=ENT, tt=TT, tl=TL)
    for o in outs:
        for p in ins.values():
            assert logprobs(d, **{o: p}) == bd.E_SHAPE, o
        for other, p in outs.items():
            if other != o:
                assert logprobs(d, **{o: p}) == bd.E_SHAPE, (o, other)
    for p in (*ins.values(), *outs.values()):
        assert logprobs(d, ws=p) == bd.E_WORKSPACE
    need = ctypes.c_int64(-1)
    f = bd.lib().bdlm_head_logprobs_workspace
    assert f(None, 1, ctypes.byref(need)) == bd.E_NULL and f(ctypes.byref(d), 1, None) == bd.E_NULL
    assert f(ctypes.byref(d), 17, ctypes.byref(need)) == bd.E_SHAPE and f(ctypes.byref(few), 6, ctypes.byref(need)) == bd.E_SHAPE
    for rows in (3, 100):
        for top in (0, 4):
            d = desc(rows=rows)
            assert f(ctypes.byref(d), top, ctypes.byref(need)) == bd.OK
            assert logprobs(d, top=top, size=need.value) == bd.OK
            assert logprobs(d, top=top, size=need.value - 1) == bd.E_WORKSPACE and logprobs(d, top=top, ws=None) == bd.E_WORKSPACE
            assert logprobs(d, top=top, ws=WS + 64) == bd.E_ALIGN


def test_logprobs_binding_refuses():
    x, w, t = torch.zeros(4, 8), torch.ones(6, 8), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="GPU"):
        bd.head_logprobs(x, w, t, top=2)
    for bad in (dict(top=17), dict(top=-1), dict(tokens=t[:3]), dict(tokens=t.int()), dict(logprob=torch.zeros(4)),
                dict(top_token=t), dict(top=2, top_token=t), dict(tokens=t, logprob=torch.zeros(5))):
        with pytest.raises(ValueError):
            bd.head_logprobs(x, w, **bad)
