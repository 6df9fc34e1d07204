"""The dense operators together with the scan, as a layer and a head use them (GPU).

Decoding: the mixer's input projection, whose columns the scan reads as views; the block step; the
gated normalisation; the output projection onto the residual stream; the head.  Training: two
projections, the masked loss, and all their gradients.  Every stage is compared with its plain
form in 64 bits on the inputs that it had, within its bound; the gradients also with differences
of the whole chain's loss.
"""
import numpy as np
import pytest
import torch

import oracle
from tests import dense_util as du
from tests.gpu_util import REL_TOL, from_pool, rel_err, to_host

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def near(got, want, what):
    share = du.worst(got, want)
    print("[gpu-chain]", what, "error / bound %.3g" % share, flush=True)
    assert share <= 1.0, (what, share)


@pytest.mark.parametrize("batch,L,H,N", [(2, 16, 4, 16), (3, 32, 14, 64)])
def test_a_denoising_step_of_a_layer_and_the_head(batch, L, H, N):
    import paper_2607_02805_amd as bd
    g = torch.Generator().manual_seed(H)

    def r(*s):
        return torch.randn(*s, generator=g)
    d, inner, vocab = 32 * H, 64 * H, 1009
    cols = 2 * inner + 2 * N                                     # z, x, B, C
    x = r(batch, L, d).to(BF).to(DEV)
    w_in = (r(cols, d) / d ** 0.5).to(BF).to(DEV)
    w_dt = (0.3 * r(H, d) / d ** 0.5).to(BF).to(DEV)
    w_out = (r(d, inner) / inner ** 0.5).to(BF).to(DEV)
    w_head = (r(vocab, d) / d ** 0.5).to(BF).to(DEV)
    A, D = -torch.exp(r(H).abs()).to(DEV), r(H).to(DEV)
    norm_w = (1 + 0.1 * r(inner)).to(DEV)
    h = (0.1 * r(batch, H, N // 4, 64, 4)).to(DEV)

    proj = bd.projection(x, w_in)
    z = proj[..., :inner]
    xs = proj[..., inner:2 * inner].unflatten(2, (H, 64))
    Bm = proj[..., 2 * inner:2 * inner + N].unflatten(2, (1, N))
    Cm = proj[..., 2 * inner + N:].unflatten(2, (1, N))
    dt = torch.nn.functional.softplus(bd.projection(x, w_dt).float() - 4.6).to(BF)
    y = bd.scan_block_step(xs, dt, A, Bm, Cm, D, D, h)
    n = bd.gated_rmsnorm(y, z, norm_w)
    n16 = n.reshape(batch, L, inner).to(BF)
    stream = x.float().clone()
    before = stream.clone()
    bd.projection(n16, w_out, residual=stream, out=stream)       # onto the fp32 residual stream
    last = stream.to(BF)
    token, logprob = bd.head_select(last, w_head, exclude=vocab - 1)
    torch.cuda.synchronize()

    near(proj, du.projection64(x, w_in)[0], "in")
    v = {"x": to_host(xs), "dt": to_host(dt), "B": to_host(Bm), "C": to_host(Cm), "A": A.cpu().numpy(),
         "D": D.cpu().numpy(), "D_rev": D.cpu().numpy()}
    assert rel_err(y, oracle.block_step(v, from_pool(h).astype(np.float64))) <= REL_TOL
    near(stream, du.projection64(n16, w_out, residual=before, out_dtype=torch.float32)[0], "out")
    l, e = du.head64(last, w_head, vocab - 1)
    picked = l.gather(1, token.reshape(-1).cpu()[:, None])[:, 0]
    assert bool((l.max(1).values - picked <= 2 * e[:, 0]).all())
    (_, tol), _ = du.head_loss64(last, w_head, token, vocab - 1)
    near(logprob, (picked - torch.logsumexp(l, 1), tol), "logprob")


@pytest.mark.parametrize("m,d,f,vocab,dtype", [(150, 64, 136, 700, torch.float32), (20, 40, 72, 130, torch.float32),
                                               (150, 64, 192, 700, BF)])
def test_training_chain_and_its_gradients(m, d, f, vocab, dtype):
    import paper_2607_02805_amd as bd
    g = torch.Generator().manual_seed(m + f)

    def r(*s):
        return torch.randn(*s, generator=g)
    x = r(m, d).to(dtype).to(DEV)
    w1, b1 = (r(f, d) / d ** 0.5).to(dtype).to(DEV), (0.1 * r(f)).to(DEV)
    w2, b2 = (r(d, f) / f ** 0.5).to(dtype).to(DEV), (0.1 * r(d)).to(DEV)
    wv = (r(vocab, d) / d ** 0.5).to(dtype).to(DEV)
    labels = torch.where(torch.rand(m, generator=g) < 0.4, -100, torch.randint(0, vocab - 1, (m,), generator=g)).to(DEV)
    weight = (torch.rand(m, generator=g) + 0.2).to(DEV)

    h, pre = bd.projection(x, w1, b1, act="gelu", pre=True)
    s = bd.projection(h, w2, b2, residual=x)
    loss, lse = bd.head_loss(s, wv, labels, exclude=vocab - 1)
    ds, dwv = bd.head_loss_backward(weight, s, wv, labels, loss, lse, exclude=vocab - 1)
    dh, dw2, db2 = bd.projection_backward(ds, h, w2, db=True)
    dx, dw1, db1 = bd.projection_backward(dh, x, w1, pre=pre, act="gelu", db=True)
    torch.cuda.synchronize()

    (want_h, want_pre) = du.projection64(x, w1, b1, "gelu")
    near(h, want_h, "h")
    near(pre, want_pre, "pre")
    near(s, du.projection64(h, w2, b2, residual=x)[0], "s")
    near(loss, du.head_loss64(s, wv, labels, vocab - 1)[0], "loss")
    for got, want, what in zip((ds, dwv), du.head_loss_backward64(weight, s, wv, labels, vocab - 1), ("ds", "dwv")):
        near(got, want, what)
    for got, want, what in zip((dh, dw2, db2), du.projection_backward64(ds, h, w2), ("dh", "dw2", "db2")):
        near(got, want, what)
    for got, want, what in zip((dx, dw1, db1), du.projection_backward64(dh, x, w1, pre, "gelu"), ("dx", "dw1", "db1")):
        near(got, want, what)
    if dtype == BF:
        return

    # differences of the chain's loss in 64 bits, along random directions
    leaves = [t.double().cpu() for t in (x, w1, b1, w2, b2, wv)]
    lab, wt = labels.cpu(), weight.double().cpu()
    ok = du.counted(lab, vocab, vocab - 1)

    def total(x, w1, b1, w2, b2, wv):
        h = du.act64(x @ w1.t() + b1, "gelu")
        l = (h @ w2.t() + b2 + x) @ wv.t()
        l[:, vocab - 1] = float("-inf")
        each = torch.logsumexp(l, 1) - l.gather(1, torch.where(ok, lab, 0)[:, None])[:, 0]
        return float((torch.where(ok, each, 0.0) * wt).sum())
    grads = [dx.double().cpu() + ds.double().cpu(), dw1, db1, dw2, db2, dwv]     # x also through the residual
    for i, grad in enumerate(grads):
        v = torch.randn(leaves[i].shape, generator=g, dtype=torch.float64)
        v /= v.norm()
        eps = 1e-4
        hi = total(*[t + eps * v if j == i else t for j, t in enumerate(leaves)])
        lo = total(*[t - eps * v if j == i else t for j, t in enumerate(leaves)])
        slope = (hi - lo) / (2 * eps)
        got = float((grad.double().cpu() * v).sum())
        # the difference's own error is eps^2 times the third derivative; fp32's is 2^-24 of the norm
        assert abs(got - slope) <= 1e-5 * float(grad.double().norm()) + 1e-7, (i, got, slope)
