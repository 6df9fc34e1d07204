"""GPU tests of the gated product and its gradients against plain forms in 64 bits, within the bounds that
tests/sublayer_util.py derives."""
import sys

import pytest
import torch

from tests import dense_util as du
from tests import sublayer_util as su

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def say(*a):
    print("[gpu-gated]", *a, flush=True)
    sys.stdout.flush()


def gen(seed):
    g = torch.Generator().manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g)


def near(got, want, what):
    share = du.worst(got, want)
    say("   ", what, "error / bound %.3g" % share)
    assert share <= 1.0, (what, share)


# rows, in, out: one token to several tiles; outputs beside multiples of 16, 32 and 64; split contractions; large tiles
SIZES = [(1, 1, 1), (1, 64, 32), (3, 129, 65), (16, 256, 96), (17, 100, 33), (32, 1024, 50), (33, 384, 130), (64, 200, 47),
         (65, 64, 64), (66, 2100, 31), (70, 7, 9), (128, 64, 128), (129, 200, 257), (300, 129, 515), (100, 4096, 70),
         (513, 448, 130), (1030, 192, 1100)]


def inputs(m, k, n, dtype, seed):
    r = gen(seed)
    x = r(m, k).to(dtype).to(DEV)
    w = [(r(n, k) / k ** 0.5).to(dtype).to(DEV) for _ in range(2)]
    return x, w[0], w[1], r


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", SIZES)
def test_gated(size, dtype):
    import paper_2607_02805_amd as bd
    m, k, n = size
    x, wg, wu, r = inputs(m, k, n, dtype, 1)
    bg, bu = r(n).to(DEV), r(n).to(DEV)
    for act, biases in (("silu", (None, None)), ("gelu", (bg, bu)), (None, (bg, None)), ("silu", (None, bu))):
        say("gated_projection", size, dtype, act, [b is not None for b in biases])
        out, pre = bd.gated_projection(x, wg, wu, *biases, act=act, pre=True)
        only = bd.gated_projection(x, wg, wu, *biases, act=act)
        torch.cuda.synchronize()
        for got, want, what in zip((out, *pre), su.gated64(x, wg, wu, *biases, act=act), ("out", "gate", "up")):
            near(got, want, what)
        assert torch.equal(only, out)
    other = torch.empty(m, n, dtype=F32 if dtype == BF else BF, device=DEV)
    near(bd.gated_projection(x, wg, wu, out=other), su.gated64(x, wg, wu, act="silu", out_dtype=other.dtype)[0], "other type")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", SIZES)
def test_gated_backward(size, dtype):
    import paper_2607_02805_amd as bd
    m, k, n = size
    x, wg, wu, r = inputs(m, k, n, dtype, 2)
    pre = ((2 * r(m, n)).to(dtype).to(DEV), r(m, n).to(dtype).to(DEV))
    for act, ht in ((None, dtype), ("silu", dtype), ("gelu", F32 if dtype == BF else BF)):
        dh = r(m, n).to(ht).to(DEV)
        say("gated_projection_backward", size, dtype, act, ht)
        got = bd.gated_projection_backward(dh, x, wg, wu, pre, act=act, dbg=True, dbu=True)
        torch.cuda.synchronize()
        want = su.gated_backward64(dh, x, wg, wu, *pre, act=act)
        names = ("dx", "dw_gate", "dw_up", "dbg", "dbu")
        for g, w, what in zip(got, want, names):
            near(g, w, what)
        # one of them alone
        for i, what in enumerate(names):
            alone = bd.gated_projection_backward(dh, x, wg, wu, pre, act=act, **{
                name: (True if name == what else None) for name in names})
            assert [a is not None for a in alone] == [j == i for j in range(5)]
            near(alone[i], want[i], what + " alone")


def test_gradient_against_differences():
    """Directional derivatives of sum(out g) by central differences of the forward call in fp32."""
    import paper_2607_02805_amd as bd
    m, k, n, h = 70, 33, 40, 2.0 ** -7
    x, wg, wu, r = inputs(m, k, n, F32, 3)
    bg, bu, g = r(n).to(DEV), r(n).to(DEV), r(m, n).to(DEV)
    for act in (None, "silu", "gelu"):
        _, pre = bd.gated_projection(x, wg, wu, bg, bu, act=act, pre=True)
        grads = bd.gated_projection_backward(g, x, wg, wu, pre, act=act, dbg=True, dbu=True)
        at = (x, wg, wu, bg, bu)
        for i, grad in enumerate(grads):
            d = r(*at[i].shape).to(DEV)

            def value(step):
                t = [v + step * d if j == i else v for j, v in enumerate(at)]
                out = bd.gated_projection(*t, act=act).double()
                return float((out * g).sum()), float((out * g).abs().sum())

            (up, size), (down, _) = value(h), value(-h)
            got, want = (up - down) / (2 * h), float((grad.double() * d.double()).sum())
            # an output is off by (k + 40) F of its factors' size, about its own; the third derivative in h is below 8 |d z|^3
            # of an output, |d z| up to 3 k^0.5 (x, of weights of size k^-0.5: 3)
            move = 3 * (k ** 0.5 if i in (1, 2) else 1)
            tol = size * ((k + 40) * su.F * 4 / h) + float(g.abs().sum()) * h * h * move ** 3 / 6
            assert abs(got - want) <= tol, (act, i, got, want, tol)


@pytest.mark.parametrize("rows", [5, 200])
def test_layouts(rows):
    """Both weights as slices of one matrix and as alternate rows of one, x and outputs inside larger tensors, leading
    dimensions, w_up before w_gate in memory."""
    import paper_2607_02805_amd as bd
    k, n = 96, 72
    r = gen(4)
    x = r(rows, 2, k + 8).to(BF).to(DEV)[..., :k]
    both = (r(2 * n, k + 3) / k ** 0.5).to(BF).to(DEV)
    for wg, wu in ((both[:n, :k], both[n:, :k]), (both[n:, :k], both[:n, :k]), (both[::2, :k], both[1::2, :k]),
                   (both[:n, :k].contiguous(),) * 2):
        if wg.data_ptr() % 16 or wu.data_ptr() % 16:
            wide = torch.zeros(2 * n, k + 8, dtype=BF, device=DEV)
            wide[:, :k] = both[:, :k]
            at = [(w.data_ptr() - both.data_ptr()) // (2 * (k + 3)) for w in (wg, wu)]
            step = wg.stride(0) // (k + 3)
            wg, wu = (wide[a::step][:n, :k] for a in at)
        hold = torch.full((rows, 2, n + 8), 7.0, dtype=F32, device=DEV)
        keep = torch.full((2, rows, 2, n + 8), 7.0, dtype=BF, device=DEV)
        out, pre = bd.gated_projection(x, wg, wu, out=hold[..., :n], pre=(keep[0, ..., :n], keep[1, ..., :n]))
        for got, want, what in zip((out, *pre), su.gated64(x, wg, wu, act="silu", out_dtype=F32), ("out", "gate", "up")):
            near(got, want, what)
        assert bool((hold[..., n:] == 7).all()) and bool((keep[..., n:] == 7).all())
        dh = r(rows, 2, n + 1).to(DEV)[..., :n]
        dw = torch.full((2, n, k + 8), 7.0, dtype=BF, device=DEV)
        dx = torch.full((rows, 2, k + 8), 7.0, dtype=BF, device=DEV)
        got = bd.gated_projection_backward(dh, x, wg, wu, pre, dx=dx[..., :k], dw_gate=dw[0, :, :k], dw_up=dw[1, :, :k])
        for g, w, what in zip(got, su.gated_backward64(dh, x, wg, wu, *pre, act="silu"), ("dx", "dw_gate", "dw_up")):
            near(g, w, what)
        assert bool((dx[..., k:] == 7).all()) and bool((dw[..., k:] == 7).all())


def test_empty_and_zero_rows():
    import paper_2607_02805_amd as bd
    w = torch.ones(24, 64, dtype=BF, device=DEV)
    x = torch.empty(0, 64, dtype=BF, device=DEV)
    assert bd.gated_projection(x, w, w).shape == (0, 24)
    e = torch.empty(0, 24, dtype=BF, device=DEV)
    got = bd.gated_projection_backward(e, x, w, w, (e, e), dbg=True, dbu=True)
    assert got[0].shape == (0, 64) and all(bool((g == 0).all()) and g.numel() for g in got[1:])


@pytest.mark.parametrize("rows", [3, 300])
def test_not_finite(rows):
    """A NaN or infinity of bf16 inputs stays in its row of the outputs, or its column."""
    import paper_2607_02805_amd as bd
    x, wg, wu, r = inputs(rows, 128, 100, BF, 5)
    clean = bd.gated_projection(x, wg, wu)
    x[1, 5], wu[7, 9] = float("nan"), float("inf")
    out = bd.gated_projection(x, wg, wu)
    rest = torch.ones_like(out, dtype=torch.bool)
    rest[1], rest[:, 7] = False, False
    assert bool(out[1].isnan().all()) and not bool(out[:, 7].isfinite().any())
    assert torch.equal(out[rest], clean[rest])


@pytest.mark.parametrize("rows", [4, 130])
def test_streams_and_graphs(rows):
    """A call on a given stream, and a captured forward and backward pass replayed with other inputs and eager work between."""
    import paper_2607_02805_amd as bd
    x, wg, wu, r = inputs(rows, 200, 136, BF, 6)
    dh = r(rows, 136).to(BF).to(DEV)

    def both():
        h, pre = bd.gated_projection(x, wg, wu, pre=True)
        return (h, *pre, *bd.gated_projection_backward(dh, x, wg, wu, pre, dbg=True, dbu=True))

    want = both()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = bd.gated_projection(x, wg, wu, stream=side)
    more = bd.gated_projection_backward(dh, x, wg, wu, want[1:3], stream=side)
    side.synchronize()
    assert torch.equal(got, want[0]) and all(torch.equal(a, b) for a, b in zip(more[:3], want[3:6]))
    with torch.cuda.stream(side):
        both()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = both()
    for k in range(3):
        x.copy_(r(rows, 200).to(BF))
        dh.mul_(0.5)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, both())), k
