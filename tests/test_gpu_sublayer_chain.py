"""A sublayer's operators together, as a model runs them, and at the sizes that reach every kind of launch
(tests/test_sublayer_plans.py holds that they do)."""
import sys

import pytest
import torch

from tests import dense_util as du
from tests import sublayer_util as su
from tests.test_gpu_logprobs import check as check_logprobs
from tests.test_gpu_logprobs import inputs as logprob_inputs
from tests.test_sublayer_plans import GATED_SIZES, GRAD_SIZES, TOP_SIZES

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def say(*a):
    print("[gpu-sublayer]", *a, flush=True)
    sys.stdout.flush()


def near(got, want, what):
    share = du.worst(got, want)
    say("   ", what, "error / bound %.3g" % share)
    assert share <= 1.0, (what, share)


def gen(seed):
    g = torch.Generator().manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g)


@pytest.mark.parametrize("size", GATED_SIZES)
def test_gated_launches(size):
    import paper_2607_02805_amd as bd
    m, k, n = size
    r = gen(1)
    x, wg, wu = r(m, k).to(BF).to(DEV), (r(n, k) / k ** 0.5).to(BF).to(DEV), (r(n, k) / k ** 0.5).to(BF).to(DEV)
    bg, bu = r(n).to(DEV), r(n).to(DEV)
    say("gated_projection", size)
    out, pre = bd.gated_projection(x, wg, wu, bg, bu, act="gelu", pre=True)
    for got, want, what in zip((out, *pre), su.gated64(x, wg, wu, bg, bu, act="gelu"), ("out", "gate", "up")):
        near(got, want, what)


@pytest.mark.parametrize("size", GRAD_SIZES)
def test_gated_backward_launches(size):
    import paper_2607_02805_amd as bd
    m, k, n = size
    r = gen(2)
    x, wg, wu = r(m, k).to(BF).to(DEV), (r(n, k) / k ** 0.5).to(BF).to(DEV), (r(n, k) / k ** 0.5).to(BF).to(DEV)
    pre = (r(m, n).to(BF).to(DEV), r(m, n).to(BF).to(DEV))
    dh = r(m, n).to(BF).to(DEV)
    say("gated_projection_backward", size)
    got = bd.gated_projection_backward(dh, x, wg, wu, pre, dbg=True, dbu=True)
    for g, want, what in zip(got, su.gated_backward64(dh, x, wg, wu, *pre, act="silu"), ("dx", "dw_gate", "dw_up", "dbg", "dbu")):
        near(g, want, what)


@pytest.mark.parametrize("size", TOP_SIZES)
def test_logprobs_launches(size):
    import paper_2607_02805_amd as bd
    m, k, n = size
    x, w, tokens = logprob_inputs(m, k, n, BF, 3)
    for top, exclude in ((16, n - 1), (3, -1), (0, 5)):
        say("head_logprobs", size, top, exclude)
        check_logprobs(bd.head_logprobs(x, w, tokens, top=top, exclude=exclude), x, w, tokens, top, exclude)


class Sublayer:
    """add_rmsnorm -> gated_projection -> projection onto the stream -> add_rmsnorm -> head."""

    def __init__(self, width, hidden, vocab, dtype):
        r = gen(4)
        self.n1, self.n2 = (1 + 0.1 * r(width)).to(DEV), (1 + 0.1 * r(width)).to(DEV)
        self.wg, self.wu = ((r(hidden, width) / width ** 0.5).to(dtype).to(DEV) for _ in range(2))
        self.wd = (r(width, hidden) / hidden ** 0.5).to(dtype).to(DEV)
        self.head = (r(vocab, width) / width ** 0.5).to(dtype).to(DEV)

    def forward(self, bd, x, stream, keep=None):
        a, s, _ = bd.add_rmsnorm(x, self.n1, stream)
        h, pre = bd.gated_projection(a, self.wg, self.wu, pre=True)
        y = bd.projection(h, self.wd)
        z, s2, _ = bd.add_rmsnorm(y, self.n2, s, out_dtype=a.dtype)
        return a, s, h, pre, y, z, s2

    def backward(self, bd, dz, kept):
        a, s, h, pre, _, _, s2 = kept
        ds2, dn2 = bd.add_rmsnorm_backward(dz, s2, self.n2)
        dh, dwd, _ = bd.projection_backward(ds2, h, self.wd)
        da, dwg, dwu, _, _ = bd.gated_projection_backward(dh, a, self.wg, self.wu, pre)
        ds, dn1 = bd.add_rmsnorm_backward(da, s, self.n1, ds2)
        return ds, dn1, dn2, dwd, dwg, dwu

    def loss64(self, x, stream, g, weights):
        n1, n2, wg, wu, wd = weights
        s = x + stream
        a = s * torch.rsqrt((s * s).mean(1, keepdim=True) + 1e-5) * n1
        h = torch.nn.functional.silu(a @ wg.t()) * (a @ wu.t())
        s2 = s + h @ wd.t()
        z = s2 * torch.rsqrt((s2 * s2).mean(1, keepdim=True) + 1e-5) * n2
        return (z * g).sum(), z


@pytest.mark.parametrize("rows", [3, 70, 300])
def test_chain_in_fp32_has_the_gradients_of_its_formula(rows):
    """In fp32 every operator is right to a few 2^-24 of its terms' sizes; through five of them, with sums of up to `hidden`
    terms of random sign, less than 2^-24 * 1,000 of an output's norm is left."""
    import paper_2607_02805_amd as bd
    layer = Sublayer(96, 160, 500, F32)
    r = gen(5)
    x, stream, g = r(rows, 96).to(DEV), r(rows, 96).to(DEV), r(rows, 96).to(DEV)
    kept = layer.forward(bd, x, stream)
    got = layer.backward(bd, g, kept)
    leaves = [t.double().cpu().requires_grad_() for t in (stream, layer.n1, layer.n2, layer.wd, layer.wg, layer.wu)]
    s, n1, n2, wd, wg, wu = leaves
    loss, z = layer.loss64(x.double().cpu(), s, g.double().cpu(), (n1, n2, wg, wu, wd))
    z = z.detach()
    assert float((kept[5].double().cpu() - z).norm() / z.norm()) < 1000 * 2.0 ** -24
    for have, want in zip(got, torch.autograd.grad(loss, leaves)):
        off = float((have.double().cpu() - want).norm() / want.norm())
        say("   ", tuple(have.shape), "%.3g" % off)
        assert off < 1000 * 2.0 ** -24


def test_chain_captured_and_replayed():
    """Forward, head and backward in one graph, replayed with other inputs, eager calls of the same layer in between; and two
    graphs on two streams, each with its own workspaces."""
    import paper_2607_02805_amd as bd
    layer = Sublayer(128, 192, 700, BF)
    r = gen(6)
    rows = 160
    sets = []
    for _ in range(2):
        x, stream, g = r(rows, 128).to(BF).to(DEV), r(rows, 128).to(DEV), r(rows, 128).to(BF).to(DEV)
        tokens = torch.randint(0, 700, (rows,), generator=torch.Generator().manual_seed(1)).to(DEV)
        sets.append((x, stream, g, tokens))

    def run(x, stream, g, tokens):
        kept = layer.forward(bd, x, stream)
        return (*kept[:3], *kept[3], *kept[4:], *layer.backward(bd, g, kept),
                *bd.head_logprobs(kept[5], layer.head, tokens, top=4, exclude=1))

    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    graphs, held = [], []
    for k in range(2):
        with torch.cuda.stream(side[k]):
            run(*sets[k])
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[k], stream=side[k]):
            held.append(run(*sets[k]))
    for turn in range(3):
        for x, stream, g, tokens in sets:
            x.copy_(r(rows, 128).to(BF))
            g.copy_(r(rows, 128).to(BF))
        torch.cuda.synchronize()
        for k in range(2):
            with torch.cuda.stream(side[k]):
                graphs[k].replay()
        torch.cuda.synchronize()
        for k in range(2):
            for a, b in zip(held[k], run(*sets[k])):
                assert torch.equal(a, b), (turn, k)


def test_repeated_calls_agree():
    """Sums are taken in a fixed order, whatever the timing."""
    import paper_2607_02805_amd as bd
    layer = Sublayer(448, 900, 5000, BF)
    r = gen(7)
    x, stream, g = r(400, 448).to(BF).to(DEV), r(400, 448).to(DEV), r(400, 448).to(BF).to(DEV)
    first = None
    for _ in range(4):
        kept = layer.forward(bd, x, stream)
        got = (kept[2], kept[5], *layer.backward(bd, g, kept), *bd.head_logprobs(kept[5], layer.head, top=16)[1:])
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(got, first))


def test_another_stream_than_the_tensors():
    """A given stream that waits for the tensors' own: outputs and workspaces are allocated on it."""
    import paper_2607_02805_amd as bd
    layer = Sublayer(128, 192, 700, BF)
    r = gen(8)
    side = torch.cuda.Stream()
    for rows in (5, 200):
        x, stream = r(rows, 128).to(BF).to(DEV), r(rows, 128).to(DEV)
        side.wait_stream(torch.cuda.current_stream())
        a, s, _ = bd.add_rmsnorm(x, layer.n1, stream, stream=side)
        h, pre = bd.gated_projection(a, layer.wg, layer.wu, pre=True, stream=side)
        lp = bd.head_logprobs(a, layer.head, top=3, stream=side)
        grads = bd.gated_projection_backward(h, a, layer.wg, layer.wu, pre, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        b, t, _ = bd.add_rmsnorm(x, layer.n1, stream)
        h2, pre2 = bd.gated_projection(b, layer.wg, layer.wu, pre=True)
        torch.cuda.synchronize()
        assert torch.equal(a, b) and torch.equal(s, t) and torch.equal(h, h2)
        for u, v in zip(lp[1:], bd.head_logprobs(b, layer.head, top=3)[1:]):
            assert torch.equal(u, v)
        for u, v in zip(grads[:3], bd.gated_projection_backward(h2, b, layer.wg, layer.wu, pre2)[:3]):
            assert torch.equal(u, v)
