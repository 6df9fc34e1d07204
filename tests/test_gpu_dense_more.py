"""More of the dense operators on the GPU, against 64 bits: activations relative to their own value; every tile
kernel that a plan can choose, at ragged sizes and over several stages; gradients over several pieces of the
vocabulary; workspaces of exactly the size asked for."""
import ctypes
import sys

import pytest
import torch

from tests import dense_util as du
from tests.test_gpu_dense import head_inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def say(*a):
    print("[gpu-dense-more]", *a, flush=True)
    sys.stdout.flush()


def gen(seed):
    g = torch.Generator().manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g)


def near(got, want, what):
    share = du.worst(got, want)
    say("   ", what, "error / bound %.3g" % share)
    assert share <= 1.0, (what, share)


# rows, in, out, type.  Together with the gradients' and the losses' own products these run each combination of tile,
# buffers, layout, output and term pairs that a plan can choose (tests/test_dense_plans.py holds them to that), over
# several stages and with tiles that end inside the matrix; the last ones several rounds of large tiles.
PROJECTIONS = [(83, 6772, 23, F32), (3968, 4238, 2, F32), (905, 258, 758, BF), (166, 133, 16963, BF), (39, 902, 151, BF),
               (1, 4845, 1740, F32), (27004, 511, 2, F32), (12399, 4332, 2, BF), (16705, 129, 411, BF), (1, 6781, 5215, BF),
               (16590, 74, 141, F32), (27686, 73, 386, F32), (1324, 5910, 148, BF), (158, 471, 16801, F32),
               (129, 4284, 18851, BF), (1417, 2702, 3061, F32), (4111, 328, 4101, BF), (4111, 328, 4101, F32)]
HEADS = [(21780, 85, 2, F32), (68, 70, 44473, F32), (416, 262, 3015, BF), (42, 132, 36521, BF), (33, 67, 66687, BF), (412, 129, 28991, F32),
         (143, 292, 40837, BF), (6102, 5869, 2, BF), (777, 136, 32003, BF)]


@pytest.mark.parametrize("m,k,n,dtype", PROJECTIONS)
def test_projections_on_every_tile(m, k, n, dtype):
    import paper_2607_02805_amd as bd
    r = gen(51)
    say("projection", m, k, n, dtype)
    x, w, b = r(m, k).to(dtype).to(DEV), (r(n, k) / k ** 0.5).to(dtype).to(DEV), r(n).to(DEV)
    res, dy, pre = r(m, n).to(dtype).to(DEV), r(m, n).to(dtype).to(DEV), (2 * r(m, n)).to(dtype).to(DEV)
    out, kept = bd.projection(x, w, b, act="gelu", residual=res, pre=True)
    grads = bd.projection_backward(dy, x, w, pre=pre, act="gelu", db=True)
    torch.cuda.synchronize()
    want, keep = du.projection64(x, w, b, "gelu", res)
    near(out, want, "out")
    near(kept, keep, "pre")
    for g, ref, what in zip(grads, du.projection_backward64(dy, x, w, pre, "gelu"), ("dx", "dw", "db")):
        near(g, ref, what)


@pytest.mark.parametrize("m,k,n,dtype", HEADS)
def test_heads_on_every_tile(m, k, n, dtype):
    import paper_2607_02805_amd as bd
    say("head", m, k, n, dtype)
    exclude = n // 2 if n > 2 else -1
    x, w, labels, dloss = head_inputs(m, k, n, dtype, 52, exclude=exclude)
    loss, lse = bd.head_loss(x, w, labels, exclude=exclude)
    dx, dw = bd.head_loss_backward(dloss, x, w, labels, loss, lse, exclude=exclude)
    token, logprob = bd.head_select(x, w, exclude=exclude)
    torch.cuda.synchronize()
    want_loss, want_lse = du.head_loss64(x, w, labels, exclude)
    near(loss, want_loss, "loss")
    near(lse, want_lse, "lse")
    out = ~du.counted(labels, n, exclude)
    assert bool((loss.cpu()[out] == 0).all()) and bool((dx.cpu()[out] == 0).all())
    want_dx, want_dw = du.head_loss_backward64(dloss, x, w, labels, exclude)
    near(dx, want_dx, "dx")
    near(dw, want_dw, "dw")
    l, e = du.head64(x, w, exclude)
    token = token.cpu()
    picked = l.gather(1, token[:, None])[:, 0]
    assert bool((token != exclude).all()) and bool((l.max(1).values - picked <= 2 * e[:, 0]).all())
    (_, tol), _ = du.head_loss64(x, w, token, exclude)
    near(logprob, (picked - torch.logsumexp(l, 1), tol), "logprob")


# ------------------------------------------------------------------ several pieces of the vocabulary
# (rows, in, vocabulary, type, excluded, columns of a piece): P of a piece stays within 512 MB, so that both go in three
PIECES = [(9000, 72, 20001, F32, 6911, 6912), (9000, 72, 20001, F32, 20000, 6912), (9001, 136, 70001, BF, 23551, 23552)]


@pytest.mark.parametrize("m,k,n,dtype,exclude,piece", PIECES)
def test_gradients_over_pieces_of_the_vocabulary(m, k, n, dtype, exclude, piece):
    """On sampled rows and tokens, those beside the pieces' ends and the excluded one among them; what w holds for
    the excluded token has no part."""
    import paper_2607_02805_amd as bd
    g = torch.Generator(device=DEV).manual_seed(53)
    x = torch.randn(m, k, generator=g, device=DEV).to(dtype)
    w = (torch.randn(n, k, generator=g, device=DEV) / k ** 0.5).to(dtype)
    labels = torch.randint(0, n, (m,), generator=g, device=DEV)
    labels[::3] = -100
    labels[7] = exclude
    dloss = torch.rand(m, generator=g, device=DEV) + 0.1
    w[exclude] = float("nan")
    say("pieces", m, k, n, dtype, exclude)
    loss, lse = bd.head_loss(x, w, labels, exclude=exclude)
    dx, dw = bd.head_loss_backward(dloss, x, w, labels, loss, lse, exclude=exclude)
    torch.cuda.synchronize()
    w[exclude] = 0
    rows = torch.tensor([0, 1, 2, 7, 127, 128, 255, 256, 4094, 4095, 4096, m - 2, m - 1], device=DEV)
    near(loss[rows], du.head_loss64(x[rows], w, labels[rows], exclude)[0], "loss")
    near(dx[rows], du.head_loss_backward64(dloss[rows], x[rows], w, labels[rows], exclude)[0], "dx")
    ends = [v + d for v in (piece, 2 * piece) for d in (-257, -256, -1, 0, 1, 255, 256)]
    at = [t for t in {*ends, 0, 1, n - 1, n - 2, exclude - 1, exclude, exclude + 1, int(labels[5])} if 0 <= t < n]
    at = torch.tensor(sorted(at), device=DEV)
    x64, w64 = x.double(), w.double().t().contiguous()
    ref = torch.zeros(len(at), k, dtype=torch.float64, device=DEV)
    tol = torch.zeros_like(ref)
    u = du.U[dtype]
    for r0 in range(0, m, 1000):
        xs, lab = x64[r0:r0 + 1000], labels[r0:r0 + 1000]
        l = torch.mm(xs, w64)
        l[:, exclude] = -torch.inf
        top = torch.logsumexp(l, 1, keepdim=True)
        gw = torch.where((lab >= 0) & (lab != exclude), dloss[r0:r0 + 1000].double(), 0.0)[:, None]
        far = (l - top).abs()
        e = (k + 8) * du.F * torch.mm(xs.abs(), w64.abs()).max(1, keepdim=True).values
        p = torch.exp(l[:, at] - top)
        hot = (lab[:, None] == at).double()
        far = torch.where(torch.isinf(far[:, at]), 0.0, far[:, at])
        # as tests/dense_util.py derives them: the logit's error e and the loss' (2 e and its sums) in P
        own = l.gather(1, lab.clamp(min=0)[:, None])
        most = l.max(1, keepdim=True).values
        span = most - torch.where(l.isinf(), torch.inf, l).min(1, keepdim=True).values
        tl = 2 * e + (8 + span + n ** 0.5) * 2 * du.F + 4 * du.F * ((top - own).abs() + top.abs() + most.abs())
        P = (p - hot) * gw
        size = torch.where(hot > 0, 1 - p, p) * gw
        dp = p * gw * (e + torch.where(torch.isfinite(tl), tl, 0.0) + (8 + far) * 2 * du.F) + 8 * du.F * size
        if dtype == BF:
            dp = dp + u * (P.abs() + dp)
            dp = dp + (u + u * u) * (P.abs() + dp)
        ref += torch.mm(P.t().contiguous(), xs)
        tol += torch.mm((dp + (m + 8) * du.F * P.abs()).t().contiguous(), xs.abs())
    tol = tol + u * (ref.abs() + tol) + 1e-37
    share = float(((dw[at].double() - ref).abs() / tol).max())
    say("    dw error / bound %.3g" % share)
    assert share <= 1.0
    assert bool((dw[exclude] == 0).all()) and bool((dx[7] == 0).all()) and bool(torch.isfinite(dw).all())


# ------------------------------------------------------------------ workspaces
@pytest.mark.parametrize("m,k,n,dtype", [(40, 72, 130, BF), (40, 72, 1100, F32), (64, 129, 1100, BF), (300, 448, 1100, BF),
                                         (300, 130, 1100, F32), (9000, 72, 20001, F32), (9001, 72, 40001, BF)])
def test_workspaces_of_the_size_asked_for(m, k, n, dtype):
    """Nothing is written past them, whatever the terms, the copies and the pieces of the vocabulary."""
    import paper_2607_02805_amd as bd
    x, w, labels, dloss = head_inputs(m, k, n, dtype, 54)
    d, _ = bd._dense(x, w)
    loss, lse = bd.head_loss(x, w, labels)
    calls = [("head_loss", lambda ws: bd.head_loss(x, w, labels, workspace=ws)),
             ("head_loss_backward", lambda ws: bd.head_loss_backward(dloss, x, w, labels, loss, lse, workspace=ws)),
             ("head_select", lambda ws: bd.head_select(x, w, workspace=ws))]
    if m * n < 1 << 24:
        dy = torch.randn(m, n, device=DEV)
        calls += [("projection", lambda ws: bd.projection(x, w, act="gelu", pre=True, workspace=ws)),
                  ("projection_backward", lambda ws: bd.projection_backward(dy, x, w, workspace=ws, db=True))]
    for name, call in calls:
        need = ctypes.c_int64(0)
        assert getattr(bd.lib(), f"bdlm_{name}_workspace")(ctypes.byref(d), ctypes.byref(need)) == 0
        buf = torch.full((need.value + (1 << 20),), 0xA5, dtype=torch.uint8, device=DEV)
        say("canary", name, m, k, n, dtype, need.value)
        want = call(None)
        got = call(buf[:need.value])
        torch.cuda.synchronize()
        assert bool((buf[need.value:] == 0xA5).all())
        for a, b in zip(want, got):
            assert torch.equal(a, b)


# ------------------------------------------------------------------ a captured loss
@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_captured_loss_serves_any_labels(dtype):
    """The rows that count are found on the device: a replay follows the labels, from none of them to all."""
    import paper_2607_02805_amd as bd
    m, k, n = 700, 136, 2100
    x, w, labels, dloss = head_inputs(m, k, n, dtype, 55)

    def run():
        loss, lse = bd.head_loss(x, w, labels)
        return (loss, lse, *bd.head_loss_backward(dloss, x, w, labels, loss, lse))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    every = torch.arange(m, device=DEV) % n
    for count in (0, 1, 64, 65, 300, m):
        labels.copy_(torch.where(torch.arange(m, device=DEV) < count, every, -1))
        for t in got:
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, run()):
            assert torch.equal(a, b), count


# ------------------------------------------------------------------ activations
# Steps of fp32 (2^-24 of the value) that an activation of an exact fp32 argument may be off by.
#   GELU, fp32: t = 1 / (1 + p a) 3 (product and sum 1, reciprocal after its Newton step 2), which R(t) takes over
#     with a sensitivity below 1; the polynomial's last two fused operations and the product with t 4; its
#     fit 1; exp2 2, what y lacks 1; products with e and z 2: 13 in all, 16 taken.
#   SiLU: exp2's argument is rounded, and its constant is: 1.5 |z|; exp2 2, sum 1, reciprocal 2, product 1: 6 + 1.5 |z|,
#     12 + 2 |z| taken.
# A slope is a sum of two terms, each off by as much of itself, and two more roundings.  At a bf16 argument, which
#   is itself half a step from what it stands for (GELU's tail moves by z^2 2^-8 with it), GELU's slope may be off by 2^-11
#   of the terms.
def phi64(z):
    return 0.5 * torch.special.erfc(-z / 2 ** 0.5)      # (torch's own ndtr is 1 + erf: no digits in the tail)


def value64(z, act):
    return z * torch.sigmoid(z) if act == "silu" else z * phi64(z)


def steps(z, act):
    return 16.0 if act == "gelu" else 12 + 2 * z.abs()


@pytest.mark.parametrize("m", [1, 70])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_activations_keep_their_digits_in_the_tail(act, m):
    """Arguments from -12 to 12: an fp32 value within some steps of itself, however small, a bf16 value
    within half a bf16 step and 2^-11 of itself; slopes (as a bias gradient of one row) likewise."""
    import paper_2607_02805_amd as bd
    z = torch.cat([torch.linspace(-12, 12, 1501), -torch.logspace(-6, 0, 200), torch.logspace(-6, 0, 200)])
    n, z64 = len(z), z.double()
    x, w, bias = torch.zeros(m, 8), torch.zeros(n, 8), z.to(DEV)
    want = value64(z64, act)
    for dtype, out_dtype in ((F32, F32), (BF, F32), (F32, BF), (BF, BF)):
        out = torch.empty(m, n, dtype=out_dtype, device=DEV)
        bd.projection(x.to(dtype).to(DEV), w.to(dtype).to(DEV), bias, act=act, out=out)
        got = out.cpu().double()
        share = steps(z64, act) * du.F if out_dtype == F32 else 2.0 ** -8 + 2.0 ** -11
        off = ((got - want).abs() / (share * want.abs() + 1e-37)).max(1).values
        say(act, m, dtype, out_dtype, "error / bound %.3g" % float(off.max()))
        assert float(off.max()) <= 1.0
        assert torch.equal(got, got[:1].expand(m, n))
    dy = torch.zeros(m, n, device=DEV)
    dy[m // 2] = 1.0                                  # one row: its slopes are the bias gradient
    for dtype in (F32, BF):
        pre = z.to(dtype)
        p64 = pre.double()
        _, _, db = bd.projection_backward(dy, x.to(dtype).to(DEV), w.to(dtype).to(DEV),
                                          pre=pre.expand(m, n).contiguous().to(DEV), act=act, dx=None, dw=None, db=True)
        if act == "gelu":
            first, second = phi64(p64), p64 * torch.exp(-p64 * p64 / 2) / (2 * torch.pi) ** 0.5
        else:
            s = torch.sigmoid(p64)
            first, second = s, p64 * s * torch.sigmoid(-p64)
        slope, size = first + second, first + second.abs()
        share = (steps(p64, act) + 4) * du.F + (2.0 ** -11 if act == "gelu" and dtype == BF else 0.0)
        off = (db.cpu().double() - slope).abs() / (share * size + 1e-37)
        say(act, m, dtype, "slope: error / bound %.3g" % float(off.max()))
        assert float(off.max()) <= 1.0


@pytest.mark.parametrize("m", [1, 70])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_activations_far_out_in_bf16(act, m):
    """Where squares overflow, and at infinities: values and slopes are the limits, a NaN stays one."""
    import paper_2607_02805_amd as bd
    z = torch.tensor([-3e38, -1e30, -1e19, -200.0, -90.0, 0.0, -0.0, 90.0, 200.0, 1e19, 1e30, 3e38,
                      float("inf"), float("-inf"), float("nan")]).to(BF)
    n = len(z)
    x, w = torch.zeros(m, 8, dtype=BF, device=DEV), torch.zeros(n, 8, dtype=BF, device=DEV)
    right = torch.where(z > 0, z, torch.where(z.isnan(), z, torch.zeros_like(z)))
    for out_dtype in (BF, F32):
        out = torch.empty(m, n, dtype=out_dtype, device=DEV)
        bd.projection(x, w, z.float().to(DEV), act=act, out=out)
        got = out.cpu()
        assert torch.equal(got[:, :-1], right[:-1].to(out_dtype).expand(m, n - 1)), (out_dtype, got[0])
        assert bool(got[:, -1].isnan().all())
    dy = torch.zeros(m, n, dtype=BF, device=DEV)
    dy[0] = 1.0
    _, _, db = bd.projection_backward(dy, x, w, pre=z.expand(m, n).contiguous().to(DEV), act=act, dx=None, dw=None, db=True)
    slope = torch.where(z > 0, 1.0, torch.where(z == 0, 0.5, 0.0))
    got = db.cpu()
    # (at 0: Phi's fit, off by 1e-7)
    assert bool(((got - slope)[:-1].abs() <= 2.0 ** -22).all()), got
    # (the other rows' products of 0 with a NaN's slope, too)
    assert bool(got[-1].isnan())
