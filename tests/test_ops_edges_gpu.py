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


def gradients(x, W, t, weight):
    """The gradients' errors against 64 bits over those of their rounding to bf16, which no result can be below."""
    r = ops.head_loss(x, W, t, row_weight=weight)
    want = R.head(x, W, t, row_weight=weight)
    worst = 0.0
    for name, got in zip(("dx", "dw"), ops.head_backward(x, W, t, r.lse, row_weight=weight)):
        worst = max(worst, float((got.double() - want[name]).norm() / (want[name].to(BF16).double() - want[name]).norm()))
    return worst


def some_rows_count(rows, live, weighted, vocab=1500, cols=160):
    g = torch.Generator("cuda").manual_seed(rows + live)
    W = (torch.randn(vocab, cols, device="cuda", generator=g) * (1.5 / cols ** 0.5)).to(BF16)
    t = torch.full((rows,), -100, device="cuda")
    at = torch.randperm(rows, device="cuda", generator=g)[:live]
    t[at] = torch.randint(0, vocab, (live,), device="cuda", generator=g)
    x = torch.randn(rows, cols, device="cuda", generator=g).to(BF16)
    return x, W, t, torch.randn(rows, device="cuda", generator=g) if weighted else None


@pytest.mark.parametrize("rows,live,weighted", [(4096, 16, False), (33, 32, False), (300, 1, False), (1025, 32, False), (2000, 50, True), (1300, 1024, True),
                                                (1025, 1000, True), (5000, 1, True), (1026, 0, True)])
def test_few_rows_that_count_keep_the_precision_of_the_type(rows, live, weighted):
    """How many rows count decides whether P is kept as two numbers, not how many there are: 2^-17 / 1.7e-3 = 0.5 % and the fp32 sums beside it."""
    x, W, t, weight = some_rows_count(rows, live, weighted)
    if live:
        assert gradients(x, W, t, weight) < 1.02
    # one gradient alone, and a replay with another number of rows that count
    r = ops.head_loss(x, W, t, row_weight=weight)
    dx, dW = ops.head_backward(x, W, t, r.lse, row_weight=weight)
    assert torch.equal(ops.head_backward(x, W, t, r.lse, row_weight=weight, need_dweight=False)[0], dx)
    assert torch.equal(ops.head_backward(x, W, t, r.lse, row_weight=weight, need_dx=False)[1], dW)
    assert not bool(dx[t < 0].any()) and (live or not bool(dW.any()))


@pytest.mark.parametrize("rows,live,weighted", [(33, 33, False), (2100, 40, False), (2100, 2100, False), (1025, 1025, True), (3000, 1500, True)])
def test_more_rows_that_count_lose_one_rounding_of_p(rows, live, weighted):
    """P as one bf16 number: independent of the gradients' own rounding and, where one element of P makes the gradient, as large: 2^0.5.  The
    mean square of the relative error of so many rows (weights: a third of them) is off by its own spread, 0.9 / n^0.5, five times that at most."""
    n = live / 3 if weighted else live
    assert gradients(*some_rows_count(rows, live, weighted)) < (2 + 5 * 0.9 / n ** 0.5) ** 0.5


def test_replays_while_few_and_many_rows_count():
    x, W, t, weight = some_rows_count(2000, 2000, True)
    keep = t.clone()
    ops.head_backward(x, W, t, ops.head_loss(x, W, t, row_weight=weight).lse, row_weight=weight)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = ops.head_loss(x, W, t, row_weight=weight)
        dx, dW = ops.head_backward(x, W, t, r.lse, row_weight=weight)
    for out in (1900, 0, 975, 976, 977, 2000, 1000):
        t.copy_(keep)
        t[:out] = -100
        graph.replay()
        torch.cuda.synchronize()
        want = ops.head_loss(x, W, t, row_weight=weight)
        for a, b in zip((*r, dx, dW), (*want, *ops.head_backward(x, W, t, want.lse, row_weight=weight))):
            assert torch.equal(a, b), out


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


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_norm_in_the_range_that_is_named(dtype):
    """Values of 1e17 in the widest row, and of 1e-16 without eps: squares and their sum stay fp32 numbers."""
    w = torch.ones(16384, device="cuda")
    for size, eps in ((1e17, 1e-5), (1e-16, 0.0)):
        x = (randn(2, 16384, seed=3).clamp(-1, 1) * size).to(dtype)
        n = ops.rms_norm(x, w, eps=eps)
        y, rstd = R.norm(x, w, eps)
        R.within("rstd", n.rstd, rstd, 42 * R.U * rstd)
        R.within("y", n.y, y, 46 * R.U * y.abs(), dtype)


# ---- over a table -------------------------------------------------------------------------------------------------------

def test_a_captured_end_of_a_model_draws_new_masks():
    """Replays of LMHead.step whose counter on the device moves on are the eager steps of those numbers."""
    from dataclasses import replace
    from paper_2510_09103_amd import workloads as WL
    from paper_2510_09103_amd.head import LMHead
    wl = WL.gpt2_350m()
    wl = replace(wl, blocks=tuple(replace(b, rows=600) if b.name == "wte" else b for b in wl.blocks if b.name in ("wte", "ln_f")))
    x, res, t = WL.head_batch(wl, 150, device="cuda")
    params = WL.initial_params(wl, device="cuda")
    grads = [torch.zeros_like(p) for p in params]
    end = LMHead(wl.blocks, p=0.2)
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    end.step(params, grads, x, res, t, 0, offset_dev=counter)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = end.step(params, grads, x, res, t, 0, offset_dev=counter)
    masks = []
    for step in (1, 2, 3):
        counter.fill_(step)
        graph.replay()
        torch.cuda.synchronize()
        got = [g.clone() for g in (*out, *grads)]
        want = end.step(params, grads, x, res, t, step)
        assert all(torch.equal(a, b) for a, b in zip(got, (*want, *grads))), step
        masks.append(got[2] == 0)
    dropped = torch.stack(masks).double().mean().item()
    assert abs(dropped - 0.2) < 5 * (0.16 / (3 * x.numel())) ** 0.5 + 1e-3            # exact zeros that were not dropped: few
    for a, b in ((0, 1), (1, 2), (0, 2)):
        both = (masks[a] & masks[b]).double().mean().item()
        assert abs(both - 0.04) < 5 * (0.04 * 0.96 / x.numel()) ** 0.5 + 1e-3


def test_parameters_are_taken_as_data():
    """Tensors that require gradients give the same bits as others, and nothing that is returned or written has a graph."""
    from dataclasses import replace
    from paper_2510_09103_amd import workloads as WL
    from paper_2510_09103_amd.head import LMHead
    wl = WL.llama_60m()
    wl = replace(wl, blocks=tuple(replace(b, rows=500) if b.name == "embed" else b for b in wl.blocks if b.name in ("embed", "norm_f")))
    x, res, t = WL.head_batch(wl, 90, device="cuda")
    params = WL.initial_params(wl, device="cuda")
    runs = []
    for wanted in (False, True):
        grads = [torch.zeros(b.rows, b.cols, dtype=BF16, device="cuda") for b in wl.blocks]
        leaves = [p.clone().requires_grad_(wanted) for p in params]
        out = LMHead(wl.blocks, p=0.1).step(leaves, grads, x.clone().requires_grad_(wanted), res.clone().requires_grad_(wanted), t, 1)
        assert not any(g.requires_grad for g in (*out, *grads)) and all(p.grad is None for p in leaves)
        runs.append([*out, *grads])
    assert all(torch.equal(a, b) for a, b in zip(*runs))
