"""The workgroups of the gradient of a sublayer's norm: few rows, wide rows, and a gradient of the stream alone."""
import ctypes
import sys

import pytest
import torch

import paper_2607_02805_amd as bd
from tests import dense_util as du
from tests import sublayer_util as su

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def say(*a):
    print("[gpu-addnorm-grids]", *a, flush=True)
    sys.stdout.flush()


@pytest.mark.parametrize("width", [1, 97, 512, 513, 1024, 1025, 4096, 4097, 8192, 8193, 32768, 1 << 22])
def test_one_workgroup_takes_no_more_than_two_short_turns(width):
    """A call whose dw one workgroup sums needs no workspace.  A turn is four rows of up to 1,024 columns, or one row: two of them
    are 8,192 elements at most, and more, or wider ones, are spread over workgroups."""
    turn = 4 if width <= 1024 else 1
    n = ctypes.c_int64(-1)
    for rows in range(1, 40):
        assert bd.lib().bdlm_add_rmsnorm_backward_workspace(rows, width, ctypes.byref(n)) == bd.OK
        if rows > turn:
            assert (n.value == 0) == (rows <= 2 * turn and width <= 4096), (rows, n.value)
            assert n.value == 0 or n.value >= 4 * width * 2
        else:
            assert n.value == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", [(8, 448), (9, 448), (8, 1024), (13, 1000), (2, 4096), (3, 4096), (2, 4100), (4, 32768), (4200, 40),
                                  (1100, 1100), (1100, 8200)])
def test_both_grids(size, dtype):
    """Both sides of each rule: the gradient of the stream is the same with dw, alone, and in place, and dw is within its bound."""
    m, n = size
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g)
    s, w, dy, dsum = (3 * r(m, n)).to(dtype).to(DEV), (1 + 0.3 * r(n)).to(DEV), r(m, n).to(dtype).to(DEV), r(m, n).to(dtype).to(DEV)
    say("add_rmsnorm_backward", size, dtype)
    ds, dw = bd.add_rmsnorm_backward(dy, s, w, dsum)
    alone, none = bd.add_rmsnorm_backward(dy, s, w, dsum, dw=None)
    none2, only = bd.add_rmsnorm_backward(dy, s, w, dsum, ds=None)
    own = dsum.clone()
    place, _ = bd.add_rmsnorm_backward(dy, s, w, own, ds=own, dw=None)
    torch.cuda.synchronize()
    assert none is None and none2 is None and place is own
    assert torch.equal(alone, ds) and torch.equal(place, ds) and torch.equal(only, dw)
    for got, want, what in zip((ds, dw), su.norm_grad64(dy, s, w, dsum, ds_dtype=ds.dtype), ("ds", "dw")):
        share = du.worst(got, want)
        say("   ", what, "error / bound %.3g" % share)
        assert share <= 1.0, (what, share)
