"""More of the dense operators on the GPU, against 64 bits: activations relative to their own value."""
import sys

import pytest
import torch

from tests import dense_util as du

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def say(*a):
    print("[gpu-dense-more]", *a, flush=True)
    sys.stdout.flush()


def gen(seed):
    g = torch.Generator().manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g)


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
