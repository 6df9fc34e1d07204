"""How the 8-bit outputs of a sublayer's norm round: nearest, ties to the even of two neighbours, at every number of e4m3."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32, E4 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


@pytest.mark.parametrize("block", [0, 128])
@pytest.mark.parametrize("width", [512, 1024, 2048, 4096, 8192, 16384])
def test_ties_go_to_the_even_neighbour(width, block):
    """Every step is exact: rows of ones have a mean square of 1 (their sum is a power of two), so with eps 0 the norm is w
    itself, and 448 among the values that share a scale makes that 1.  What is left is the rounding: a number of e4m3 keeps its code,
    and of the middle between two, one of whose codes is even, that one is the answer."""
    import paper_2607_02805_amd as bd
    codes = torch.arange(127)                       # 0 .. 448; 127 is NaN
    number = codes.to(torch.uint8).view(E4).float()
    middle = (number[1:] + number[:-1]) / 2
    even = torch.where(codes[:-1] % 2 == 0, codes[:-1], codes[1:])
    value, code = torch.cat([number, middle]), torch.cat([codes, even])
    value, code = torch.cat([value, -value]), torch.cat([code, code + 128])
    # 127 of them and 448 in each block of 128 columns
    pad = -len(value) % 127
    value, code = (torch.cat([t, torch.zeros(pad, dtype=t.dtype)]).view(-1, 127) for t in (value, code))
    value = torch.cat([value, torch.full((len(value), 1), 448.0)], 1).reshape(-1)
    code = torch.cat([code, torch.full((len(code), 1), 126)], 1).reshape(-1)
    w = value.repeat(width // len(value)).to(DEV)
    want = code.repeat(width // len(code)).to(torch.uint8)
    assert w.numel() == width
    one, part = torch.ones(3, width, device=DEV), torch.full((3, width), 0.25, device=DEV)
    for x, residual in ((one, None), (one.to(BF), None), (part.to(BF), 3 * part), (part, (3 * part).to(BF))):
        q, _, scale = bd.add_rmsnorm(x, w, residual, eps=0.0, out_dtype=E4, scale_block=block)
        assert bool((scale == 1).all())
        assert torch.equal(q.view(torch.uint8).cpu(), want.expand(3, width))
