"""GPU tests of the head's log-probabilities, entropies and most probable tokens against plain forms in 64 bits.

Inputs lie on a grid (x in multiples of 2^-4, w of 2^-8), so that every logit is exact in fp32 in any order of its sum and
the order of the tokens, ties among them, is the same everywhere.  What is left is the softmax: with d = logit - largest,
exp(d) is off by (4 + |d|) 2^-23 of itself, of which |d| exp(d) <= 1 counts at most 1; sums of n positive terms by at most
(n / 64 + 20) 2^-24 of themselves (64 or fewer in a run, then pairs or runs of records); log1p, the quotient and the last
sums by a few 2^-24 of their terms.
"""
import sys

import pytest
import torch

from tests import dense_util as du

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
F = 2.0 ** -24


def say(*a):
    print("[gpu-logprobs]", *a, flush=True)
    sys.stdout.flush()


def inputs(m, k, n, dtype, seed, spread=6.0, step=2.0 ** -8):
    g = torch.Generator().manual_seed(seed)
    w = (torch.randn(n, k, generator=g) / k ** 0.5 / step).round().clamp(-255, 255) * step
    lean = torch.randint(0, n, (m,), generator=g)
    x = torch.randn(m, k, generator=g) + spread * torch.rand(m, 1, generator=g) * w[lean]
    x = (x * 16).round().clamp(-127, 127) / 16
    tokens = torch.where(torch.rand(m, generator=g) < 0.5, lean, torch.randint(0, n, (m,), generator=g))
    if m > 3:
        tokens[1], tokens[2] = n, -100
    return x.to(dtype).to(DEV), w.to(dtype).to(DEV), tokens.to(DEV)


def want64(x, w, exclude):
    l = du.rows2(du.d64(x)) @ du.d64(w).t()
    if 0 <= exclude < l.shape[1]:
        l[:, exclude] = -float("inf")
    return l


def close(got, want, tol, what):
    share = float(((got.double().cpu().reshape(want.shape) - want).abs() / tol).max()) if want.numel() else 0.0
    say("   ", what, "error / bound %.3g" % share)
    assert share <= 1.0, (what, share)


def check(got, x, w, tokens, top, exclude):
    logprob, entropy, token, listed = got
    l = want64(x, w, exclude)
    n = l.shape[1]
    lse = torch.logsumexp(l, 1)
    p = (l - lse[:, None]).exp()
    terms = (n / 64 + 20) * F + 16 * F           # of a sum of exponentials
    if tokens is None:
        assert logprob is None
    else:
        t = tokens.reshape(-1).cpu()
        here = (t >= 0) & (t < n)
        want = torch.where(here, l.gather(1, t.clamp(0, n - 1)[:, None])[:, 0] - lse, 0.0)
        gone = here & (t == exclude)
        assert bool((logprob.reshape(-1).cpu()[gone] == -float("inf")).all())
        keep = ~gone
        close(logprob.reshape(-1)[keep.to(DEV)], want[keep], (terms + 8 * F * (1 + want.abs()))[keep], "logprob")
    if entropy is not None:
        d = l - l.max(1, keepdim=True).values
        e = d.exp()
        slope = torch.where(e > 0, -e * d, 0.0).sum(1) / e.sum(1)
        close(entropy, torch.special.entr(p).sum(1), terms * (1 + 2 * slope) + 8 * F * (1 + slope), "entropy")
    if top == 0:
        assert token is None and listed is None
        return
    order = torch.sort(l, dim=1, descending=True, stable=True)
    assert torch.equal(token.reshape(-1, top).cpu(), order.indices[:, :top])
    want = order.values[:, :top] - lse[:, None]
    close(listed, want, (terms + 8 * F * (1 + want.abs())), "top")


# rows, in, vocabulary: few rows with 16 and 32 columns a workgroup, small and large tiles, past the end of groups and tiles
SIZES = [(1, 64, 2), (1, 128, 1000), (5, 72, 333), (20, 64, 515), (32, 96, 16401), (40, 200, 1037), (64, 64, 130), (65, 64, 257),
         (130, 136, 1025), (300, 448, 4100), (700, 65, 1031), (2, 64, 40000), (260, 64, 33000)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", SIZES)
def test_logprobs(size, dtype):
    import paper_2607_02805_amd as bd
    m, k, n = size
    for top, exclude, given in ((0, -1, True), (1, n - 1, True), (5, 0, False), (16, n // 2, True), (2, -1, False)):
        if top > n - (exclude >= 0):
            continue
        say("head_logprobs", size, dtype, top, exclude, given)
        x, w, tokens = inputs(m, k, n, dtype, 1)
        if given and m > 4:
            tokens[4] = exclude
        got = bd.head_logprobs(x, w, tokens if given else None, top=top, exclude=exclude)
        torch.cuda.synchronize()
        check(got, x, w, tokens if given else None, top, exclude)


# few rows, tiles, and tiles of a split contraction whose logits are joined
@pytest.mark.parametrize("rows,k", [(3, 64), (200, 64), (200, 1536)])
def test_ties(rows, k):
    """Equal logits throughout a group, a tile and over several: the lowest tokens, in order."""
    import paper_2607_02805_amd as bd
    n = 1500
    x = torch.ones(rows, k, dtype=BF, device=DEV)
    w = torch.zeros(n, k, dtype=BF, device=DEV)
    got = bd.head_logprobs(x, w, top=16)
    assert torch.equal(got[2].cpu(), torch.arange(16).expand(rows, 16))
    w[700:] = 0.5
    w[1400] = 1.0
    for exclude, want in ((-1, [1400, *range(700, 715)]), (1400, [*range(700, 716)]), (703, [1400, 700, 701, 702, *range(704, 716)])):
        got = bd.head_logprobs(x, w, top=16, exclude=exclude)
        assert torch.equal(got[2].cpu(), torch.tensor(want).expand(rows, 16)), exclude
        check(got, x, w, None, 16, exclude)
    # more groups, and more values, than are gathered before they are counted
    for many in (10000, 40000):
        v = torch.zeros(many, k, dtype=BF, device=DEV)
        for first in (0, many - 700):
            v.zero_()
            v[first:] = 0.5
            assert torch.equal(bd.head_logprobs(x, v, top=16)[2].cpu(), torch.arange(first, first + 16).expand(rows, 16)), (many, first)
            assert torch.equal(bd.head_logprobs(x, v, top=3, exclude=first + 1)[2].cpu(),
                               torch.tensor([first, first + 2, first + 3]).expand(rows, 3))
    # far apart, and equal: in every group of columns one
    w.zero_()
    w[5::37] = 1.0
    got = bd.head_logprobs(x, w, top=16)
    assert torch.equal(got[2].cpu(), torch.arange(5, n, 37)[:16].expand(rows, 16))
    # all of a row's largest in one group of columns
    w.zero_()
    w[320:352] = torch.arange(32, 0, -1, device=DEV)[:, None].to(BF) / 64
    got = bd.head_logprobs(x, w, top=16)
    assert torch.equal(got[2].cpu(), torch.arange(320, 336).expand(rows, 16))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_sure_rows(dtype):
    """Nearly certain tokens: log-probabilities and entropies near 0 keep their digits."""
    import paper_2607_02805_amd as bd
    for m in (4, 150):
        x, w, _ = inputs(m, 256, 2000, dtype, 2, spread=0.0)
        lean = torch.arange(m) % 2000
        x = ((x.float().cpu() * 0.25 + 24 * w.float().cpu()[lean]) * 16).round().clamp(-127, 127) / 16
        x, t = x.to(dtype).to(DEV), lean.to(DEV)
        got = bd.head_logprobs(x, w, t, top=3)
        check(got, x, w, t, 3, -1)
        l = want64(x, w, -1)
        d = l - l.max(1, keepdim=True).values
        rest = d.exp().scatter(1, l.argmax(1, keepdim=True), 0.0).sum(1)
        exact = -torch.log1p(rest)
        assert bool((exact > -1e-4).all())
        # the others' sum is of terms exp(d), each off by (4 + |d|) 2^-23 of itself
        far = d.abs().max(1).values
        close(got[0], exact, ((8 + far) * 2 + 60) * F * exact.abs(), "sure logprob")
        slope = torch.where(d < 0, -d.exp() * d, 0.0).sum(1)
        close(got[1], torch.log1p(rest) + slope / (1 + rest), ((8 + far) * 2 + 80) * F * (slope + rest), "sure entropy")


@pytest.mark.parametrize("rows,k", [(4, 64), (200, 64), (200, 1536)])
def test_not_finite(rows, k):
    """NaN and infinite logits stay in their rows; what is left of a row is listed, and then nothing."""
    import paper_2607_02805_amd as bd
    n, top = 300, 8
    x, w, tokens = inputs(rows, k, n, BF, 3)
    tokens[:] = 7
    clean = bd.head_logprobs(x, w, tokens, top=top)
    a, b = x.clone(), w.clone()
    a[:, 0], b[:, 0] = 0, 0
    a[0, 0] = 1.0
    b[3:, 0] = float("-inf")          # row 0: three finite logits; the others' 0 * -inf is NaN there
    got = bd.head_logprobs(a, b, tokens, top=top)
    ids, lp = got[2].cpu(), got[3].cpu()
    first = (a[0].float().cpu() @ b[:3].float().cpu().t()).sort(descending=True, stable=True).indices
    assert ids[0].tolist() == [*first.tolist(), *[-1] * 5] and bool((lp[0, 3:] == -float("inf")).all())
    assert bool(lp[0, :3].isfinite().all()) and float(got[0][0]) == -float("inf") and bool(got[1][0].isfinite())
    assert bool(got[0][1:].isnan().all()) and bool(got[1][1:].isnan().all())
    assert bool(((ids[1:, :3] >= 0) & (ids[1:, :3] < 3)).all()) and bool((ids[1:, 3:] == -1).all())
    x[1, 0] = float("nan")
    got = bd.head_logprobs(x, w, tokens, top=top)
    rest = [r for r in range(rows) if r != 1]
    assert all(torch.equal(g[rest], c[rest]) for g, c in zip(got, clean))
    assert bool(got[0][1].isnan()) and bool(got[1][1].isnan()) and bool((got[2][1] == -1).all())
    assert bool((got[3][1] == -float("inf")).all())
    # w's row of the excluded token may hold anything
    w2 = w.clone()
    w2[9] = float("nan")
    x[1, 0] = 0.0
    for g, c in zip(bd.head_logprobs(x, w2, tokens, top=top, exclude=9), bd.head_logprobs(x, w, tokens, top=top, exclude=9)):
        assert torch.equal(g, c)


@pytest.mark.parametrize("rows,k", [(6, 72), (90, 72), (90, 1000)])
def test_layouts_streams_graphs(rows, k):
    import paper_2607_02805_amd as bd
    n = 900
    x, w, tokens = inputs(rows, k, n, BF, 4)
    want = bd.head_logprobs(x, w, tokens, top=4, exclude=5)
    wide = torch.zeros(rows, k + 16, dtype=BF, device=DEV)
    wide[:, 8:8 + k] = x
    got = bd.head_logprobs(wide[:, 8:8 + k], w, tokens, top=4, exclude=5)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    got = bd.head_logprobs(x.view(2, rows // 2, k), w, tokens.view(2, -1), top=4, exclude=5)
    assert got[2].shape == (2, rows // 2, 4) and all(torch.equal(a.reshape(b.shape), b) for a, b in zip(got, want))
    only = bd.head_logprobs(x, w, tokens, entropy=False)
    assert only[1] is None and torch.equal(only[0], bd.head_logprobs(x, w, tokens)[0])
    assert bd.head_logprobs(x[:0], w, tokens[:0], top=4)[2].shape == (0, 4)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = bd.head_logprobs(x, w, tokens, top=4, exclude=5, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with torch.cuda.stream(side):
        bd.head_logprobs(x, w, tokens, top=4, exclude=5)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = bd.head_logprobs(x, w, tokens, top=4, exclude=5)
    for s in range(3):
        other, _, t = inputs(rows, k, n, BF, 10 + s)
        x.copy_(other)
        tokens.copy_(t)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, bd.head_logprobs(x, w, tokens, top=4, exclude=5))), s


def test_agrees_with_select_and_loss():
    """The best alternative is the token that head_select picks, and a token's log-probability the loss's negative."""
    import paper_2607_02805_amd as bd
    for m in (7, 150):
        x, w, tokens = inputs(m, 96, 2100, BF, 5)
        logprob, _, token, listed = bd.head_logprobs(x, w, tokens, top=1, exclude=2)
        pick, lp = bd.head_select(x, w, exclude=2)
        assert torch.equal(token[:, 0], pick) and float((listed[:, 0] - lp).abs().max()) <= 2e-6
        loss, _ = bd.head_loss(x, w, tokens, exclude=2)
        assert float((logprob + loss)[logprob.isfinite()].abs().max()) <= 4e-6
