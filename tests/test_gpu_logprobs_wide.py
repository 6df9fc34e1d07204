"""Head's log-probabilities over vocabularies whose groups of columns are more than a row's kernel keeps in registers (past 4,096
groups of 32), with what counts on both sides of that."""
import sys

import pytest
import torch

from tests.test_gpu_logprobs import check, inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
N = 140001
KEPT = 4096 * 32


def say(*a):
    print("[gpu-logprobs-wide]", *a, flush=True)
    sys.stdout.flush()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [1, 2, 20])
def test_largest_given_and_equal_past_the_registers(rows, dtype):
    """Row 0 leans towards equal tokens on both sides, and then towards others; the rest of the rows lie as they are drawn."""
    import paper_2607_02805_amd as bd
    x, w, tokens = inputs(rows, 64, N, dtype, 1)
    lean = x[0].sign().float()
    first = [5, KEPT - 1, KEPT, N - 33, N - 1]
    second = [KEPT - 40, *range(KEPT + 1, KEPT + 15), N - 2]
    w[first], w[second] = (lean * 0.5).to(dtype), (lean * 0.375).to(dtype)
    for given in (N - 1, KEPT, KEPT - 1, KEPT + 5):
        tokens[0] = given
        for top, exclude in ((5, -1), (16, -1), (16, KEPT), (8, 5), (0, N - 1)):
            say("head_logprobs", rows, dtype, given, top, exclude)
            got = bd.head_logprobs(x, w, tokens, top=top, exclude=exclude)
            torch.cuda.synchronize()
            want = [t for t in first if t != exclude] + [t for t in second if t != exclude]
            if top:
                assert got[2][0].tolist() == want[:top]
            check(got, x, w, tokens, top, exclude)


def test_all_equal():
    """More groups reach the bound than are gathered: the list is made one value after the other."""
    import paper_2607_02805_amd as bd
    x, w = torch.ones(3, 64, dtype=BF, device=DEV), torch.zeros(N, 64, dtype=BF, device=DEV)
    assert torch.equal(bd.head_logprobs(x, w, top=16)[2].cpu(), torch.arange(16).expand(3, 16))
    for many in (10, 4000):
        w.zero_()
        w[N - many:] = 0.5
        want = [*range(N - many, N), *range(16)][:16]
        got = bd.head_logprobs(x, w, top=16)
        assert torch.equal(got[2].cpu(), torch.tensor(want).expand(3, 16)), many
        check(got, x, w, None, 16, -1)
