"""GPU parity of the dense operators (projection, head_loss, head_select and the gradients)
against plain forms in 64 bits, within the bounds that tests/dense_util.py derives."""
import sys

import pytest
import torch

from tests import dense_util as du

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def say(*a):
    print("[gpu-dense]", *a, flush=True)
    sys.stdout.flush()


def gen(seed):
    g = torch.Generator().manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g)


def near(got, want, what):
    share = du.worst(got, want)
    say("   ", what, "error / bound %.3g" % share)
    assert share <= 1.0, (what, share)


# rows, in, out: one token to several tiles, odd sizes, both sides of every size rule
SIZES = [(1, 64, 32), (1, 1, 1), (3, 129, 65), (16, 256, 96), (17, 100, 33), (33, 1024, 50), (64, 384, 130),
         (65, 64, 64), (70, 7, 9), (128, 64, 128), (129, 200, 257), (300, 129, 515), (513, 448, 130)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", SIZES)
def test_projection(size, dtype):
    import paper_2607_02805_amd as bd
    m, k, n = size
    r = gen(1)
    x, w, b = r(m, k).to(dtype).to(DEV), (r(n, k) / k ** 0.5).to(dtype).to(DEV), r(n).to(DEV)
    res = r(m, n).to(dtype).to(DEV)
    for act, bias, residual in ((None, None, None), ("silu", b, None), ("gelu", b, res), (None, None, res)):
        say("projection", size, dtype, act, bias is not None, residual is not None)
        out, pre = bd.projection(x, w, bias, act=act, residual=residual, pre=True)
        torch.cuda.synchronize()
        want, keep = du.projection64(x, w, bias, act, residual)
        near(out, want, "out")
        near(pre, keep, "pre")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", SIZES)
def test_projection_backward(size, dtype):
    import paper_2607_02805_amd as bd
    m, k, n = size
    r = gen(2)
    x, w = r(m, k).to(dtype).to(DEV), (r(n, k) / k ** 0.5).to(dtype).to(DEV)
    dy, pre = r(m, n).to(dtype).to(DEV), (2 * r(m, n)).to(dtype).to(DEV)
    for act in (None, "silu", "gelu"):
        say("projection_backward", size, dtype, act)
        got = bd.projection_backward(dy, x, w, pre=pre, act=act, db=True)
        torch.cuda.synchronize()
        for g, want, what in zip(got, du.projection_backward64(dy, x, w, pre, act), ("dx", "dw", "db")):
            near(g, want, what)


HEADS = [(1, 64, 2), (1, 128, 1000), (5, 72, 333), (20, 64, 515), (40, 200, 1037), (64, 64, 130), (65, 64, 257),
         (130, 136, 1025), (300, 448, 4100), (700, 65, 1031)]


def head_inputs(m, k, n, dtype, seed, left_out=0.3, exclude=-1):
    r = gen(seed)
    g = torch.Generator().manual_seed(seed + 1)
    w = (r(n, k) / k ** 0.5).to(dtype)
    lean = torch.randint(0, n, (m,), generator=g)
    x = (r(m, k) + 6 * torch.rand(m, 1, generator=g) * w[lean].float()).to(dtype)
    labels = torch.where(torch.rand(m, generator=g) < left_out, -100, lean)
    if m > 3:
        labels[1], labels[2] = n, exclude
    dloss = torch.rand(m, generator=g) + 0.1
    return x.to(DEV), w.to(DEV), labels.to(DEV), dloss.to(DEV)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", HEADS)
def test_head_select(size, dtype):
    import paper_2607_02805_amd as bd
    m, k, n = size
    for exclude in (-1, n - 1, 0):
        say("head_select", size, dtype, exclude)
        x, w, _, _ = head_inputs(m, k, n, dtype, 3)
        token, logprob = bd.head_select(x, w, exclude=exclude)
        torch.cuda.synchronize()
        l, e = du.head64(x, w, exclude)
        token = token.cpu()
        assert bool(((token >= 0) & (token < n) & (token != exclude)).all())
        # the token's logit is the largest, within twice a logit's bound
        picked = l.gather(1, token[:, None])[:, 0]
        assert bool((l.max(1).values - picked <= 2 * e[:, 0]).all())
        lse = torch.logsumexp(l, 1)
        (_, tol), _ = du.head_loss64(x, w, token, exclude)
        near(logprob, (picked - lse, tol), "logprob")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", HEADS)
def test_head_loss(size, dtype):
    import paper_2607_02805_amd as bd
    m, k, n = size
    for exclude in (-1, n - 1):
        say("head_loss", size, dtype, exclude)
        x, w, labels, dloss = head_inputs(m, k, n, dtype, 4, exclude=exclude)
        loss, lse = bd.head_loss(x, w, labels, exclude=exclude)
        dx, dw = bd.head_loss_backward(dloss, x, w, labels, loss, lse, exclude=exclude)
        torch.cuda.synchronize()
        want_loss, want_lse = du.head_loss64(x, w, labels, exclude)
        near(loss, want_loss, "loss")
        near(lse, want_lse, "lse")
        out = ~du.counted(labels, n, exclude)
        assert bool((loss.cpu()[out] == 0).all()) and bool((lse.cpu()[out] == 0).all())
        assert bool((dx.cpu()[out] == 0).all())
        want_dx, want_dw = du.head_loss_backward64(dloss, x, w, labels, exclude)
        near(dx, want_dx, "dx")
        near(dw, want_dw, "dw")
