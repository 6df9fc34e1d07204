"""A sublayer's operators and the head's log-probabilities on matrices whose rows lie more than 2^32 elements from the first, with
what lies between them left alone."""
import sys

import pytest
import torch

from tests import dense_util as du
from tests import sublayer_util as su
from tests.test_gpu_logprobs import check, inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32, E4 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
SIZES = [(3, 1 << 32), (70, 1 << 26)]      # rows, and elements from one to the next


def say(*a):
    print("[gpu-sublayer-far]", *a, flush=True)
    sys.stdout.flush()


def near(got, want, what):
    share = du.worst(got, want)
    say("   ", what, "error / bound %.3g" % share)
    assert share <= 1.0, (what, share)


def far(rows, cols, step, dtype=BF, value=None):
    """[rows][cols] with a row every `step` elements, canaries of 7 beside each row; the rest is not written."""
    raw = torch.empty((rows - 1) * step + cols + 64, dtype=torch.uint8 if dtype == E4 else dtype, device=DEV)
    torch.as_strided(raw, (rows, 32), (step, 1), cols).fill_(7)
    t = torch.as_strided(raw, (rows, cols), (step, 1))
    if value is not None:
        t.copy_(value)
    return t.view(E4) if dtype == E4 else t


def alone(t):
    """The 32 elements behind each row."""
    raw = t.view(torch.uint8) if t.dtype == E4 else t
    return bool((torch.as_strided(raw, (t.shape[0], 32), t.stride(), t.shape[1]) == 7).all())


@pytest.mark.parametrize("width", [520, 1100, 8200])
@pytest.mark.parametrize("rows,step", SIZES)
def test_norm(rows, step, width):
    import paper_2607_02805_amd as bd
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g)
    say("add_rmsnorm", rows, step, width)
    x, res, w = far(rows, width, step, value=r(rows, width)), far(rows, width, step, value=r(rows, width)), r(width).to(DEV)
    out, total = far(rows, width, step), far(rows, width, step)
    bd.add_rmsnorm(x, w, res, out=out, sum=total)
    y, s = su.norm_bounds(x, w, res, out_dtype=BF)
    near(out, y, "out")
    near(total, s, "sum")
    q = far(rows, width, step, E4)
    _, _, scale = bd.add_rmsnorm(x, w, out=q, scale_block=128)
    want = su.norm64(x, w)[0]
    each = du.d64(scale).repeat_interleave(128, 1)[:, :width]
    near(q.float().double().cpu() * each, (want, 2.0 ** -4 * want.abs() + 2.0 ** -10 * each + 2 * (su.near(width) + 8 * su.F) * want.abs()), "e4m3")
    ds, dw = bd.add_rmsnorm_backward(x, total, w, res, ds=out)
    for got, want, what in zip((ds, dw), su.norm_grad64(x, total, w, res, ds_dtype=BF), ("ds", "dw")):
        near(got, want, what)
    assert alone(out) and alone(total) and alone(q)


@pytest.mark.parametrize("rows,step", SIZES)
def test_gated(rows, step):
    import paper_2607_02805_amd as bd
    k, n = 192, 70
    g = torch.Generator().manual_seed(2)
    r = lambda *s: torch.randn(*s, generator=g)
    say("gated_projection", rows, step)
    x = far(rows, k, step, value=r(rows, k))
    wide = torch.empty(n * (1 << 26), dtype=BF, device=DEV)
    wg, wu = (torch.as_strided(wide, (n, k), (1 << 26, 1), at) for at in (0, 1 << 25))
    wg.copy_(r(n, k) / k ** 0.5)
    wu.copy_(r(n, k) / k ** 0.5)
    out, gate, up = (far(rows, n, step) for _ in range(3))
    bd.gated_projection(x, wg, wu, out=out, pre=(gate, up))
    for got, want, what in zip((out, gate, up), su.gated64(x, wg, wu, act="silu"), ("out", "gate", "up")):
        near(got, want, what)
    assert alone(out) and alone(gate) and alone(up)
    dh, dx = far(rows, n, step, value=r(rows, n)), far(rows, k, step)
    got = bd.gated_projection_backward(dh, x, wg, wu, (gate, up), dx=dx, dbg=True, dbu=True)
    for a, b, what in zip(got, su.gated_backward64(dh, x, wg, wu, gate, up, act="silu"), ("dx", "dw_gate", "dw_up", "dbg", "dbu")):
        near(a, b, what)
    assert alone(dx)


@pytest.mark.parametrize("rows,step", SIZES)
def test_logprobs(rows, step):
    import paper_2607_02805_amd as bd
    k, n = 64, 90
    say("head_logprobs", rows, step)
    x, w, tokens = inputs(rows, k, n, BF, 3)
    x, w = far(rows, k, step, value=x), far(n, k, 1 << 26, value=w)
    check(bd.head_logprobs(x, w, tokens, top=5, exclude=4), x, w, tokens, 5, 4)
