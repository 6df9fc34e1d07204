"""GPU tests of the norm at a sublayer's entry (residual's addition, 8-bit outputs with scales) and of its gradient,
against plain forms in 64 bits within the bounds that tests/sublayer_util.py derives."""
import sys

import pytest
import torch

from tests import dense_util as du
from tests import sublayer_util as su

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32, E4 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


def say(*a):
    print("[gpu-addnorm]", *a, flush=True)
    sys.stdout.flush()


def gen(seed):
    g = torch.Generator().manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g)


def near(got, want, what):
    share = du.worst(got, want)
    say("   ", what, "error / bound %.3g" % share)
    assert share <= 1.0, (what, share)


def eight_bits(q, scale, y, block):
    """8-bit values and scales of y (64 bits) within their bounds."""
    width = y.shape[1]
    want = su.scales64(y, block)
    e = su.near(width) + 8 * su.F
    near(scale, (want, e * want), "scale")
    sc = du.rows2(du.d64(scale))
    each = sc if not block else sc.repeat_interleave(block, 1)[:, :width]
    got = du.rows2(q.float().double().cpu()) * each
    near(got, (y, 2.0 ** -4 * y.abs() + 2.0 ** -10 * each + 2 * e * y.abs()), "values")
    # the largest of those that share a scale is the largest number there is
    step = block or width
    top = torch.stack([c.abs().max(1).values for c in du.rows2(q.float().cpu()).split(step, 1)], 1)
    assert bool(((top == 448) | (du.rows2(want) == 1.0)).all())


# both sides of every width rule (512, 1,024, 2,048, 4,096, 8,192), odd ones; rows past one turn of the grid
SIZES = [(1, 1), (3, 7), (5, 64), (2, 127), (130, 448), (7, 512), (9, 513), (3, 1000), (1, 1024), (6, 1025), (3, 2048),
         (5, 2049), (2, 4096), (3, 4101), (2, 8192), (3, 8193), (2, 20001), (8300, 40), (2100, 1100), (530, 8200)]


@pytest.mark.parametrize("out", [BF, F32, E4])
@pytest.mark.parametrize("size", SIZES)
def test_norm(size, out):
    import paper_2607_02805_amd as bd
    m, n = size
    r = gen(1)
    x, w = r(m, n).to(BF), 1 + 0.3 * r(n)
    stream = 3 * r(m, n) * (1 + 9 * (torch.rand(n) < 0.02))
    for xt, rt in ((BF, None), (BF, BF), (BF, F32), (F32, None), (F32, BF), (F32, F32)):
        xd = x.to(xt).to(DEV)
        rd = None if rt is None else stream.to(rt).to(DEV)
        for block in (0, 128) if out == E4 else (0,):
            say("add_rmsnorm", size, xt, rt, out, block)
            got, total, scale = bd.add_rmsnorm(xd, w.to(DEV), rd, out_dtype=out, scale_block=block)
            torch.cuda.synchronize()
            assert got.dtype == out and (total is None) == (rt is None) and (scale is None) == (out != E4)
            y, s = su.norm_bounds(xd, w, rd, out_dtype=out)
            if out == E4:
                eight_bits(got, scale, y[0], block)
            else:
                near(got, y, "out")
            if total is not None:
                assert total.dtype == rt
                near(total, s, "sum")


@pytest.mark.parametrize("types", [(a, b, c) for a in (BF, F32) for b in (BF, F32) for c in (None, BF, F32)])
@pytest.mark.parametrize("size", SIZES)
def test_norm_backward(size, types):
    import paper_2607_02805_amd as bd
    m, n = size
    yt, st, tt = types
    r = gen(2)
    s, w, dy = (3 * r(m, n)).to(st).to(DEV), (1 + 0.3 * r(n)).to(DEV), r(m, n).to(yt).to(DEV)
    dsum = None if tt is None else r(m, n).to(tt).to(DEV)
    say("add_rmsnorm_backward", size, types)
    ds, dw = bd.add_rmsnorm_backward(dy, s, w, dsum)
    torch.cuda.synchronize()
    assert ds.dtype == (tt or st)
    want = su.norm_grad64(dy, s, w, dsum, ds_dtype=ds.dtype)
    near(ds, want[0], "ds")
    near(dw, want[1], "dw")
    if n in (1025, 8193, 64):
        # one of the two alone, and in place
        only, none = bd.add_rmsnorm_backward(dy, s, w, dsum, dw=None)
        assert none is None and torch.equal(only, ds)
        none, only = bd.add_rmsnorm_backward(dy, s, w, dsum, ds=None)
        assert none is None and torch.equal(only, dw)
        if tt is not None:
            own = dsum.clone()
            got, _ = bd.add_rmsnorm_backward(dy, s, w, own, ds=own)
            assert got is own and torch.equal(own, ds)


def test_gradient_against_differences():
    """Of sum(out g) + sum(s h): the directional derivative by central differences of the forward call in fp32, whose
    outputs are off by near(width) of themselves."""
    import paper_2607_02805_amd as bd
    m, n, h = 5, 600, 2.0 ** -6
    r = gen(3)
    x, res, w, g, hb = (r(m, n).to(DEV) for _ in range(5))
    w = w[0].contiguous()
    d, dv = r(m, n).to(DEV), r(n).to(DEV)

    def value(x, w):
        out, total, _ = bd.add_rmsnorm(x, w, res, eps=1e-3)
        return float((out.double() * g.double()).sum() + (total.double() * hb.double()).sum()), \
            float((out.double() * g.double()).abs().sum() + (total.double() * hb.double()).abs().sum())

    _, s, _ = bd.add_rmsnorm(x, w, res, eps=1e-3)
    ds, dw = bd.add_rmsnorm_backward(g, s, w, hb, eps=1e-3)
    for want, (up, size), (down, _) in (
            (float((ds.double() * d.double()).sum()), value(x + h * d, w), value(x - h * d, w)),
            (float((dw.double() * dv.double()).sum()), value(x, w + h * dv), value(x, w - h * dv))):
        got = (up - down) / (2 * h)
        # the third derivative of s / |s| along d, of unit size per column, times h^2 / 6, is below h^2 of the terms
        assert abs(got - want) <= size * (2 * su.near(n) / h + h * h), (got, want)


@pytest.mark.parametrize("n", [40, 700, 1100, 9000])
def test_layouts(n):
    """Column slices at odd strides, rows of stride 0, leading dimensions, outputs inside larger ones left alone."""
    import paper_2607_02805_amd as bd
    r = gen(4)
    big = r(6, 2, n + 37).to(BF).to(DEV)
    x = big[:, :, 8:8 + n]
    stream = r(6, 2, n + 3).to(DEV)[..., :n]
    w = r(n).to(DEV)
    hold = torch.full((12, n + 5), 7.0, dtype=BF, device=DEV)
    total = torch.full((12, n + 9), 7.0, device=DEV)
    out = hold.view(6, 2, n + 5)[..., :n]
    got, kept, _ = bd.add_rmsnorm(x, w, stream, out=out, sum=total.view(6, 2, n + 9)[..., :n])
    y, s = su.norm_bounds(x, w, stream, out_dtype=BF)
    near(got, y, "out")
    near(kept, s, "sum")
    assert bool((hold[:, n:] == 7).all()) and bool((total[:, n:] == 7).all())
    one = r(n).to(DEV)
    got, _, _ = bd.add_rmsnorm(one.expand(4, n), w)
    near(got, su.norm_bounds(one.expand(4, n), w)[0], "stride 0")
    # 8 bits into a slice
    hold = torch.zeros((12, n + 3), dtype=torch.uint8, device=DEV).view(E4)
    q, _, scale = bd.add_rmsnorm(x.reshape(12, n).contiguous(), w, out=hold[:, :n], scale_block=128)
    eight_bits(q, scale, su.norm64(x, w)[0], 128)
    assert bool((hold.view(torch.uint8)[:, n:] == 0).all())
    dy = r(6, 2, n + 1).to(DEV)[..., :n]
    grad = torch.full((6, 2, n + 7), 7.0, dtype=BF, device=DEV)
    ds, dw = bd.add_rmsnorm_backward(dy, x, w, x, ds=grad[..., :n])
    a, b = su.norm_grad64(dy, x, w, x, ds_dtype=BF)
    near(ds, a, "ds")
    near(dw, b, "dw")
    assert bool((grad[..., n:] == 7).all())


@pytest.mark.parametrize("n", [40, 1100, 9000])
def test_in_place(n):
    import paper_2607_02805_amd as bd
    r = gen(5)
    x, stream, w = r(9, n).to(BF).to(DEV), r(9, n).to(BF).to(DEV), r(n).to(DEV)
    want, total, _ = bd.add_rmsnorm(x, w, stream)
    a, b = x.clone(), stream.clone()
    got, kept, _ = bd.add_rmsnorm(a, w, b, out=a, sum=b)
    assert got is a and kept is b and torch.equal(a, want) and torch.equal(b, total)
    got, none, _ = bd.add_rmsnorm(x, w, stream, sum=False)
    assert none is None and torch.equal(got, want)


@pytest.mark.parametrize("n", [33, 900, 1500, 9000])
def test_range(n):
    """Rows whose squares overflow or vanish in fp32, rows of zeros, and rows with an infinity or NaN; none disturbs another."""
    import paper_2607_02805_amd as bd
    r = gen(6)
    x = r(8, n)
    size = torch.tensor([1.0, 2.0 ** 100, 2.0 ** 125, 2.0 ** -90, 0.0, 1.0, 1.0, 2.0 ** -120])[:, None]
    x = (x.clamp(-3, 3) * size).to(BF)
    x[5, n // 2] = float("inf")
    x[6, 3] = float("nan")
    xd, w = x.to(DEV), (1 + 0.1 * r(n)).to(DEV)
    fine = [0, 1, 2, 3, 4, 7]
    for eps in (1e-5, 1e-30):
        for out in (F32, BF):
            got, _, _ = bd.add_rmsnorm(xd, w, eps=eps, out_dtype=out)
            y, _ = su.norm_bounds(xd[fine], w, eps=eps, out_dtype=out)
            near(got[fine], y, ("out", eps, out))
            got = got.cpu()
            assert bool(got[6].isnan().all())
            assert bool(got[5, n // 2].isnan()) and bool((got[5][torch.arange(n) != n // 2] == 0).all())
        q, _, scale = bd.add_rmsnorm(xd, w, eps=eps, out_dtype=E4)
        scale = scale.cpu()
        assert bool(scale[[5, 6]].isnan().all()) and float(scale[4]) == 1.0
        assert bool((q[4].float() == 0).all())
        rows = fine[:4] + [7]
        eight_bits(q[rows], scale[rows], su.norm64(xd[rows], w, eps=eps)[0], 0)
        dy = r(8, n).to(DEV)
        ds, _ = bd.add_rmsnorm_backward(dy, xd, w, eps=eps, ds=torch.empty(8, n, device=DEV))
        near(ds[fine], su.norm_grad64(dy[fine], xd[fine], w, eps=eps)[0], ("ds", eps))
        assert bool(ds[6].isnan().all())


def test_e4m3_rounds_to_nearest_even():
    """Values on, beside and between e4m3's numbers: with a largest |x| of 448 and w = 1 the scale is rstd, so that what is
    rounded is x itself; torch's own conversion rounds to nearest even."""
    import paper_2607_02805_amd as bd
    n = 512
    grid = torch.arange(0, 127, dtype=torch.uint8).view(E4).float()
    mid = (grid[1:] + grid[:-1]) / 2
    v = torch.cat([grid, mid, mid * (1 + 2.0 ** -12), mid * (1 - 2.0 ** -12)])
    x = torch.zeros(2, n)
    x[0, :v.numel()], x[1, :v.numel()] = v, -v
    x[:, -1] = 448
    xd, w = x.to(DEV), torch.ones(n, device=DEV)
    q, _, _ = bd.add_rmsnorm(xd, w, out_dtype=E4)
    # (products with rstd and its inverse are off by a few F)
    away = (x.abs()[..., None] - mid).abs().min(-1).values > 1e-4 * x.abs()
    assert bool((q.float().cpu()[away] == x.to(E4).float()[away]).all())


def test_empty_and_streams():
    import paper_2607_02805_amd as bd
    w = torch.ones(64, device=DEV)
    out, total, _ = bd.add_rmsnorm(torch.empty(0, 64, device=DEV), w, torch.empty(0, 64, device=DEV))
    assert out.shape == (0, 64) and total.shape == (0, 64)
    ds, dw = bd.add_rmsnorm_backward(torch.empty(0, 64, device=DEV), torch.empty(0, 64, device=DEV), w)
    assert ds.shape == (0, 64) and bool((dw == 0).all())
    r = gen(7)
    x, res, w = r(300, 1024).to(BF).to(DEV), r(300, 1024).to(DEV), r(1024).to(DEV)
    want = bd.add_rmsnorm(x, w, res)
    grads = bd.add_rmsnorm_backward(x, want[1], w, res)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = bd.add_rmsnorm(x, w, res, stream=side)
    more = bd.add_rmsnorm_backward(x, got[1], w, res, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got[:2] + more, want[:2] + grads))


@pytest.mark.parametrize("n", [1024, 9000])
def test_graph(n):
    """Captured calls, replayed with other inputs in place and eager work in between."""
    import paper_2607_02805_amd as bd
    r = gen(8)
    x, res, w = r(70, n).to(BF).to(DEV), r(70, n).to(DEV), r(n).to(DEV)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        bd.add_rmsnorm(x, w, res)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, total, _ = bd.add_rmsnorm(x, w, res)
        q, _, scale = bd.add_rmsnorm(x, w, out_dtype=E4, scale_block=128)
        ds, dw = bd.add_rmsnorm_backward(out, total, w, res)
    for k in range(3):
        x.copy_(r(70, n).to(BF))
        res.mul_(1.5)
        g.replay()
        torch.cuda.synchronize()
        a, b, _ = bd.add_rmsnorm(x, w, res)
        c, _, e = bd.add_rmsnorm(x, w, out_dtype=E4, scale_block=128)
        f = bd.add_rmsnorm_backward(a, b, w, res)
        for got, want in ((out, a), (total, b), (scale, e), (ds, f[0]), (dw, f[1])):
            assert torch.equal(got, want), k
        assert torch.equal(q.view(torch.uint8), c.view(torch.uint8))
