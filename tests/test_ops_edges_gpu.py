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


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,out", [(6, 3), (40, 11), (1300, 500), (20, 20), (1300, 1300)])
@pytest.mark.parametrize("factor", [float("inf"), float("nan"), 3e38])
def test_rows_that_do_not_count_have_no_gradient_whatever_the_factor(rows, out, factor, dtype):
    """A loss scaler that overflows: rows that do not count get zeros all the same, and so does dweight if no row counts."""
    x, W = randn(rows, 72, seed=1, dtype=dtype), randn(130, 72, seed=2, dtype=dtype)
    t = torch.arange(rows, device="cuda") % 130
    t[:out] = -100
    lse = ops.head_loss(x, W, t).lse
    dx, dW = ops.head_backward(x, W, t, lse, scale=4.0, upstream=torch.tensor(factor, device="cuda"))
    assert not bool(dx[:out].any())
    if out == rows:
        assert not bool(dW.any())
    else:
        assert not bool(torch.isfinite(dx[out:]).all())


# ---- norm --------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("cols", [9, 64, 700, 2048, 5000])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_8_bit_rows_near_nothing(cols, dtype):
    """Rows whose largest value is below what 1 / scale can bring to 448, zeros among them (dropout leaves such)."""
    x = randn(9, cols, seed=1, dtype=dtype)
    x[:, 1::3] = 0
    w = torch.tensor([1e-30, 1e-34, 1e-36, 1e-37, 1e-38, 1e-40, 1e-43, 1e-45, 0.0], device="cuda")
    for i in range(9):
        g = w[i].expand(cols).contiguous()
        n = ops.rms_norm(x[i:i + 1], g, eps=1e-5, out_dtype=E4M3)
        y = R.norm(n.h, g, 1e-5)[0]
        top = y.abs().amax().item()
        want = max(top / 448, 2.0 ** -126) if top > 2.0 ** -150 else 1.0
        scale = n.scale.double().item()
        # products of the row's values: 48 roundings, and steps of 2^-149 where they are below the type's normal numbers
        assert abs(scale - want) <= 48 * R.U * want + 2.0 ** -149, (i, scale, want)
        got = n.y.to(F32).double() * scale
        assert bool(torch.isfinite(got).all()) and not bool(got[0, 1::3].any())
        off = 2.0 ** -4 * y.abs() + 2.0 ** -10 * scale + 60 * R.U * (y.abs() + scale) + 2.0 ** -149
        if top > 2.0 ** -150:
            assert bool(((got - y).abs() <= off).all()), (i, float(((got - y).abs() - off).max()))
