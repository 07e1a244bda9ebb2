"""Edges of the operators of a model's end: small losses, rows near nothing, overflowing factors, few rows that count in a large batch."""
import math

import pytest
import torch

import ops_reference as R
from paper_2510_09103_amd import ops

pytestmark = pytest.mark.gpu
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn


def randn(*size, seed=0, dtype=F32, scale=1.0):
    g = torch.Generator("cuda").manual_seed(seed)
    return (torch.randn(*size, device="cuda", generator=g) * scale).to(dtype)


# ---- loss over the vocabulary ----------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,vocab", [(1, 40), (7, 300), (40, 700), (300, 2000)])
def test_sure_rows_keep_the_digits_of_their_loss(rows, vocab, dtype):
    """Logits that are exact (x selects a column of W): a target and one competitor below it, in the same tile or another, and nothing else.
    The loss is log(1 + exp(-gap)), whatever the size of the logits."""
    pairs = [(20.0, 12.0), (100.0, 14.0), (300.0, 14.0), (-300.0, 16.0), (1000.0, 16.0), (0.0, 15.0), (12.0, 16.0), (-20.0, 13.0)]
    W = torch.full((vocab, 16), -2048.0)
    for k, (top, gap) in enumerate(pairs):
        W[vocab - 2 - k, k], W[(vocab - 7 - k) if k % 2 else k, k] = top, top - gap
    i = torch.arange(rows) % 8
    x = torch.zeros(rows, 16)
    x[torch.arange(rows), i] = 1.0
    x, Wd, t = x.to("cuda", dtype), W.to("cuda", dtype), (vocab - 2 - i).cuda()
    assert torch.equal(Wd.float().cpu(), W)
    r = ops.head_loss(x, Wd, t)
    want = torch.tensor([math.log1p(math.exp(-gap)) for _, gap in pairs], dtype=torch.float64)[i]
    got = r.row_loss.double().cpu()
    # in the sum 1 + exp(-gap): two exponentials of one unit in the last place each (the top's and what undoes the rounding of its argument),
    # their product, the sum in the tile and the sum of two tiles with half a unit each; the logarithm adds nothing at this size
    off = 2 * 2.0 ** -23 + 3 * 2.0 ** -24
    assert float((got - want).abs().max()) <= off, (got - want).tolist()
    R.within("lse", r.lse.cpu(), torch.tensor([top for top, _ in pairs], dtype=torch.float64)[i] + want, off)
