"""The operators of a model's end on the GPU against their plain forms in 64 bits: sizes and masks where they can go wrong."""
import pytest
import torch

import ops_reference as R
from paper_2510_09103_amd import ops

pytestmark = pytest.mark.gpu
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn


def randn(*size, seed=0, dtype=F32, scale=1.0):
    g = torch.Generator("cuda").manual_seed(seed)
    return (torch.randn(*size, device="cuda", generator=g) * scale).to(dtype)


def pitched(t, extra):
    """The same values with `extra` elements between the rows, off 16-byte alignment by one element."""
    rows, cols = t.shape
    buf = torch.full((rows * (cols + extra) + 1,), float("nan"), dtype=t.dtype, device=t.device)
    view = buf[1:].view(rows, cols + extra)[:, :cols]
    view.copy_(t)
    return view


# ---- dropout ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("rows,cols,dtype,p,residual", [
    (1, 1, F32, 0.5, False), (1, 7, BF16, 0.1, True), (3, 8, BF16, 0.3, False), (17, 65, F32, 0.9, True), (33, 257, BF16, 0.1, True),
    (5, 1600, BF16, 0.1, False), (64, 100, F32, 0.0, True), (40, 24, F32, 0.99999, False), (9, 40, BF16, 1e-7, False),
])
def test_dropout(rows, cols, dtype, p, residual):
    x, r = randn(rows, cols, dtype=dtype, seed=1), randn(rows, cols, dtype=dtype, seed=2) if residual else None
    rng = ops.Rng(0x123456789ABCDEF0, (5 << 32) + 77)
    y = ops.dropout(x, p, rng, residual=r)
    f = (R.factors(rows, cols, p, *rng[:2]) if p else torch.ones(rows, cols, dtype=torch.float64)).cuda()
    want = x.double() * f + (r.double() if residual else 0.0)
    R.within("y", y, want, 3 * R.U * ((x.double() * f).abs() + want.abs()), dtype)
    # the gradient has the same mask; strided rows and work in place give the same bits
    g = ops.dropout(torch.ones_like(x), p, rng)
    assert torch.equal(g != 0, f.to(g.device) != 0)
    xs = pitched(x, 5)
    assert torch.equal(ops.dropout(xs, p, rng, residual=r, out=pitched(x, 3)), y)
    assert ops.dropout(xs, p, rng, residual=r, out=xs) is xs and torch.equal(xs, y)


def test_dropout_drops_whatever_stands_there_and_keeps_its_rate():
    x = torch.full((64, 4096), float("inf"), device="cuda")
    x[::2] = float("nan")
    y = ops.dropout(x, 0.25, ops.Rng(3))
    dropped = (y == 0).double().mean().item()
    assert abs(dropped - 0.25) < 5 * (0.25 * 0.75 / x.numel()) ** 0.5          # five standard deviations
    assert not bool(torch.isfinite(y[y != 0]).any())
    for other in (ops.Rng(4), ops.Rng(3, 1), ops.Rng(3 + (1 << 32)), ops.Rng(3, 1 << 32)):
        z = ops.dropout(x, 0.25, other) == 0
        both = (z & (y == 0)).double().mean().item()
        assert abs(both - 0.0625) < 5 * (0.0625 * 0.9375 / x.numel()) ** 0.5   # independent masks


def test_dropout_offset_on_the_device_is_added():
    x = randn(10, 100)
    at = torch.tensor([41], device="cuda")
    assert torch.equal(ops.dropout(x, 0.5, ops.Rng(1, 1, at)), ops.dropout(x, 0.5, ops.Rng(1, 42)))


def test_no_rows():
    x = torch.empty(0, 16, device="cuda", dtype=BF16)
    w = torch.ones(16, device="cuda")
    assert ops.dropout(x, 0.5, ops.Rng(1)).shape == x.shape
    n = ops.rms_norm(x, w, residual=x)
    assert n.y.shape == x.shape and n.rstd.shape == (0,)
    dw = ops.rms_norm_backward(x, n.h, w, n.rstd)[2]
    assert torch.equal(dw, torch.zeros_like(w))
    W, t = randn(20, 16, dtype=BF16), torch.empty(0, dtype=torch.int64, device="cuda")
    loss = ops.head_loss(x, W, t)
    assert loss.loss.item() == 0
    dx, dW = ops.head_backward(x, W, t, loss.lse)
    assert dx.shape == x.shape and not bool(dW.any())


# ---- norm --------------------------------------------------------------------------------------------------------------

NORMS = [(1, 1, F32, F32, 0.0, True), (1, 2048, BF16, BF16, 0.0, True), (2, 8, BF16, F32, 0.3, False), (7, 33, F32, BF16, 0.0, False),
         (5, 511, BF16, BF16, 0.1, True), (6, 513, F32, F32, 0.2, True), (3, 1025, BF16, F32, 0.0, True), (9, 1600, BF16, BF16, 0.1, True),
         (4, 2049, F32, F32, 0.0, True), (3, 5461, F32, F32, 0.0, False), (2, 8191, BF16, BF16, 0.1, True), (2, 16384, BF16, BF16, 0.0, True),
         (300, 72, BF16, F32, 0.1, True)]


@pytest.mark.parametrize("rows,cols,dtype,wtype,p,residual", NORMS)
def test_norm_forward(rows, cols, dtype, wtype, p, residual):
    x, w = randn(rows, cols, dtype=dtype, seed=1), (1 + randn(cols, seed=2) * 0.3).to(wtype)
    r = randn(rows, cols, dtype=dtype, seed=3, scale=3.0) if residual else None
    rng, eps = ops.Rng(99, 7), 1e-5
    n = ops.rms_norm(x, w, eps=eps, residual=r, p=p, rng=rng)
    if p or residual:
        f = (R.factors(rows, cols, p, *rng[:2]) if p else torch.ones(1, dtype=torch.float64)).cuda()
        want = x.double() * f + (r.double() if residual else 0.0)
        R.within("h", n.h, want, 3 * R.U * ((x.double() * f).abs() + want.abs()), dtype)
    else:
        assert n.h is x
    y, rstd = R.norm(n.h, w, eps)
    # a lane adds 64 squares in a row at most, then 8 sums: half of 72 roundings on rstd, then the root, the division and two products
    R.within("rstd", n.rstd, rstd, 42 * R.U * rstd)
    R.within("y", n.y, y, 46 * R.U * y.abs(), dtype)
    if dtype == BF16 or residual:
        q = ops.rms_norm(pitched(x, 3), w, eps=eps, residual=r, p=p, rng=rng, out_dtype=E4M3)
        assert torch.equal(q.h, n.h) and torch.equal(q.rstd, n.rstd)
        top = y.abs().amax(1)
        R.within("scale", q.scale, top / 448, 48 * R.U * top / 448)
        # below 2^-6 the steps of the type are 2^-9: half of one, times the scale
        got, s = q.y.to(F32).double() * q.scale.double()[:, None], q.scale.double()[:, None]
        R.within("e4m3", got, y, 2.0 ** -10 * s + 60 * R.U * (y.abs() + s), E4M3)


def test_norm_rows_of_zeros_and_values_that_are_not_finite():
    x = randn(6, 64, dtype=BF16)
    x[1] = 0
    x[2, 5] = float("nan")
    x[3, 6] = float("inf")
    n = ops.rms_norm(x, torch.ones(64, device="cuda"), eps=1e-5, out_dtype=E4M3)
    v = n.y.to(F32)
    assert not bool(v[1].any()) and n.scale[1] == 1
    assert bool(v[2].isnan().all()) and bool(v[3, 6].isnan()) and not bool(v[3, 7].any())
    assert bool(torch.isfinite(v[[0, 1, 4, 5]]).all())
    w = torch.ones(64, device="cuda")
    w[7] = float("nan")
    v = ops.rms_norm(x[4:], w, out_dtype=E4M3).y.to(F32)
    assert bool(v[:, 7].isnan().all()) and bool(torch.isfinite(v[:, :7]).all())


@pytest.mark.parametrize("rows,cols,dtype,wtype,p,residual", NORMS + [(2500, 40, F32, F32, 0.0, True), (1100, 3000, BF16, BF16, 0.0, False)])
def test_norm_backward(rows, cols, dtype, wtype, p, residual):
    h, w = randn(rows, cols, dtype=dtype, seed=1, scale=2.0), (1 + randn(cols, seed=2) * 0.3).to(wtype)
    dy = randn(rows, cols, dtype=dtype, seed=3)
    dh = randn(rows, cols, dtype=dtype, seed=4) if residual else None
    rstd = R.norm(h, w, 1e-5)[1].float()
    rng = ops.Rng(5, 6)
    dx, dres, dw = ops.rms_norm_backward(dy, h, w, rstd, dh=dh, p=p, rng=rng)
    want, size, want_w, size_w = R.norm_backward(dy, h, w, rstd, dh)
    off = 80 * R.U * size              # 64 + 8 sums of a row, and eight products and additions
    R.within("dresidual", dres, want, off, dtype)
    if p and rows <= 64:
        f = R.factors(rows, cols, p, *rng[:2]).cuda()
        R.within("dx", dx, want * f, (off + 2 * R.U * want.abs()) * f, dtype)
    elif not p:
        assert dx is dres
    # a thread adds the rows that it meets one after the other: rows / (1024 workgroups), then 4 wavefronts, then 64 sums and 16
    R.within("dweight", dw, want_w, (rows / 1024 + 90) * R.U * size_w, wtype)
    # the other type of dweight, strided rows, results in the place of the gradients
    other = BF16 if wtype == F32 else F32
    a, b = pitched(dy, 1), pitched(dh, 2) if residual else None
    dx2, dres2, dw2 = ops.rms_norm_backward(a, pitched(h, 4), w, rstd, dh=b, p=p, rng=rng, grad_dtype=other)
    assert torch.equal(dx2, dx) and torch.equal(dres2, dres) and dw2.dtype == other
    R.within("dweight", dw2, want_w, (rows / 1024 + 90) * R.U * size_w, other)


def test_norm_backward_is_the_derivative():
    """Central differences of sum(y c + h e) in 64 bits against the kernel in fp32."""
    rows, cols, eps, step = 3, 24, 1e-5, 1e-6
    x, r, c, e = (randn(rows, cols, seed=s).double() for s in range(4))
    w = 1 + 0.2 * randn(cols, seed=9).double()
    rng = ops.Rng(11, 12)
    f = R.factors(rows, cols, 0.4, *rng[:2]).cuda()

    def value(x, r, w):
        h = x * f + r
        return float((R.norm(h, w, eps)[0] * c + h * e).sum())

    n = ops.rms_norm(x.float(), w.float(), eps=eps, residual=r.float(), p=0.4, rng=rng)
    dx, dr, dw = ops.rms_norm_backward(c.float(), n.h, w.float(), n.rstd, dh=e.float(), p=0.4, rng=rng)
    for name, at, got in (("x", x, dx), ("r", r, dr), ("w", w, dw)):
        for i in range(0, at.numel(), 5):
            d = torch.zeros_like(at).view(-1)
            d[i] = step
            args = lambda s: [t + s * d.view(t.shape) if t is at else t for t in (x, r, w)]      # noqa: E731
            slope = (value(*args(1)) - value(*args(-1))) / (2 * step)
            # differences: third derivatives of order 10 times step^2, values of order 100 with 53 bits over the step; fp32: 1e-5
            assert abs(slope - got.view(-1)[i].item()) < 2e-5 * max(1.0, abs(slope)), (name, i)


# ---- loss over the vocabulary ----------------------------------------------------------------------------------------

def problem(rows, vocab, cols, dtype, masked=0.0, seed=0):
    g = torch.Generator("cuda").manual_seed(seed)
    W = (torch.randn(vocab, cols, device="cuda", generator=g) * (1.5 / cols ** 0.5)).to(dtype)
    t = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    x = (torch.randn(rows, cols, device="cuda", generator=g) + 2.0 * torch.rand(rows, 1, device="cuda", generator=g) * W[t].float()).to(dtype)
    out = torch.rand(rows, device="cuda", generator=g) < masked
    t[out] = torch.tensor([-100, -1, vocab, 1 << 40], device="cuda")[torch.randint(0, 4, (int(out.sum()),), device="cuda", generator=g)]
    return x, W, t


def check_head(x, W, t, **kw):
    up = kw.pop("upstream", None)
    r = ops.head_loss(x, W, t, **kw)
    dx, dW = ops.head_backward(x, W, t, r.lse, upstream=up, **kw)
    want = R.head(x, W, t, dtype=x.dtype, upstream=1.0 if up is None else up.item(), **kw)
    R.within("row_loss", r.row_loss, want["row"], want["row_off"])
    R.within("lse", r.lse, want["lse"], want["lse_off"])
    R.within("loss", r.loss, want["loss"], want["loss_off"])
    R.within("dx", dx, want["dx"], want["dx_off"], x.dtype)
    R.within("dweight", dW, want["dw"], want["dw_off"], x.dtype)
    for name, got in (("dx", dx), ("dw", dW)):
        norm = want[name].norm()
        if x.dtype == BF16 and want[name].numel() > 500 and norm > 0:
            # two roundings to bf16, each of root mean square 2^-8 / sqrt(3) at most
            assert float((got.double().reshape(want[name].shape) - want[name]).norm() / norm) < 2.0 ** -8, name
    return r, dx, dW


SIZES = [(1, 1, 1), (1, 2, 8), (1, 5000, 64), (2, 129, 7), (3, 100, 250), (16, 257, 72), (63, 1000, 128), (64, 64, 64), (65, 513, 96),
         (128, 300, 40), (129, 4099, 130), (257, 511, 256), (700, 1031, 200), (300, 2300, 512)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,vocab,cols", SIZES)
def test_head(rows, vocab, cols, dtype):
    check_head(*problem(rows, vocab, cols, dtype))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,vocab,cols,masked", [(1, 50, 16, 1.0), (6, 200, 64, 0.5), (20, 333, 72, 0.5), (32, 90, 40, 1.0), (40, 333, 24, 0.5), (400, 600, 64, 0.9), (1300, 700, 40, 0.4),
                                                    (2100, 130, 72, 1.0), (1500, 257, 33, 0.02), (33, 300, 64, 1.0), (200, 5000, 128, 0.3), (256, 129, 64, 0.5), (257, 600, 40, 0.5)])
def test_head_rows_without_a_target(rows, vocab, cols, masked, dtype):
    x, W, t = problem(rows, vocab, cols, dtype, masked, seed=3)
    out = (t < 0) | (t >= vocab)
    weight = randn(rows, seed=5)
    clean = check_head(x, W, t, row_weight=weight)
    # whatever stands in rows that do not count reaches nothing
    x[out] = float("nan")
    x[out & (torch.arange(rows, device="cuda") % 2 == 0)] = float("inf")
    weight[out] = float("nan")
    r = ops.head_loss(x, W, t, row_weight=weight)
    dx, dW = ops.head_backward(x, W, t, r.lse, row_weight=weight)
    for a, b in zip((*r, dx, dW), (*clean[0], *clean[1:])):
        assert torch.equal(a, b)
    assert not bool(dx[out].any()) and not bool(r.row_loss[out].any()) and not bool(r.lse[out].any())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_head_reduction_scale_upstream(dtype):
    x, W, t = problem(150, 400, 48, dtype, 0.2)
    check_head(x, W, t, reduction="sum", scale=0.125, upstream=torch.tensor([-3.0], device="cuda"))
    check_head(x, W, t, row_weight=randn(150, seed=1), scale=64.0, upstream=torch.tensor(0.5, device="cuda"))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", [(140, 64), (140, 50), (9, 64), (30, 50)])
def test_head_strided_operands_and_results(rows, cols, dtype):
    """Rows of x, W and the gradients with gaps and odd alignments: the same bits as packed ones, and nothing between the rows is written."""
    x, W, t = problem(rows, 300, cols, dtype, 0.1)
    r = ops.head_loss(x, W, t)
    dx, dW = ops.head_backward(x, W, t, r.lse)
    for ex, ew in ((8, 16), (3, 5)):
        xs, Ws, gx, gw = pitched(x, ex), pitched(W, ew), pitched(torch.zeros_like(x), ex), pitched(torch.zeros_like(W), ew)
        r2 = ops.head_loss(xs, Ws, t)
        ops.head_backward(xs, Ws, t, r2.lse, dx=gx, dweight=gw)
        assert torch.equal(r.row_loss, r2.row_loss) and torch.equal(gx, dx) and torch.equal(gw, dW)
        for g, e in ((gx, ex), (gw, ew)):
            gaps = g.as_strided((g.shape[0] - 1, e), (g.stride(0), 1), g.storage_offset() + g.shape[1])
            assert bool(gaps.isnan().all())
    part = ops.head_backward(x, W, t, r.lse, need_dx=False)
    assert part[0] is None and torch.equal(part[1], dW)
    part = ops.head_backward(x, W, t, r.lse, need_dweight=False)
    assert part[1] is None and torch.equal(part[0], dx)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,vocab,cols,out", [(1025, 300, 72, 0), (1500, 700, 200, 0), (2100, 513, 64, 1), (1100, 300, 50, 0)])
def test_head_many_rows_that_all_count(rows, vocab, cols, out, dtype):
    """Aligned rows that all count are read where they are, at any distance from one another, and dx may replace them."""
    x, W, t = problem(rows, vocab, cols, dtype, seed=11)
    t[-1:][:out] = -100
    r, dx, dW = check_head(x, W, t)
    wide = torch.full((rows, cols + 24), float("nan"), device="cuda", dtype=dtype)
    wide[:, 8:cols + 8] = x
    view = wide[:, 8:cols + 8]
    again = ops.head_loss(view, W, t)
    dx2, dW2 = ops.head_backward(view, W, t, again.lse)
    for a, b in zip((*again, dx2, dW2), (*r, dx, dW)):
        assert torch.equal(a, b)
    dx3, dW3 = ops.head_backward(view, W, t, again.lse, dx=view)
    assert torch.equal(view, dx) and torch.equal(dW3, dW) and wide[:, :8].isnan().all() and wide[:, cols + 8:].isnan().all()


def test_head_replays_while_the_rows_that_count_change():
    x, W, t = problem(1300, 400, 64, BF16, seed=12)
    keep = t.clone()
    ops.head_loss(x, W, t)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = ops.head_loss(x, W, t)
        dx, dW = ops.head_backward(x, W, t, r.lse)
    for out in (0, 400, 0, 1300, 1, 0):
        t.copy_(keep)
        t[:out] = -100
        graph.replay()
        torch.cuda.synchronize()
        want = ops.head_loss(x, W, t)
        dx2, dW2 = ops.head_backward(x, W, t, want.lse)
        for a, b in zip((*r, dx, dW), (*want, dx2, dW2)):
            assert torch.equal(a, b), out


@pytest.mark.parametrize("rows,vocab,cols,dtype", [(33000, 2500, 24, BF16), (16400, 2100, 40, F32)])
def test_head_in_several_pieces(rows, vocab, cols, dtype):
    check_head(*problem(rows, vocab, cols, dtype, 0.1))


@pytest.mark.parametrize("rows,weighted", [(1, False), (2, True), (17, False), (32, False), (33, True), (130, True), (400, True), (1024, True)])
def test_head_few_rows_keep_the_precision_of_the_type(rows, weighted):
    """Where a gradient comes from few elements of P, P is kept as two bf16 numbers (2^-17 of it is lost): the gradients' error is that of
    their own rounding, 1.7e-3 in root mean square, and 2^-17 / 1.7e-3 = 0.5 % and the fp32 sums beside it."""
    x, W, t = problem(rows, 1500, 160, BF16, 0.2 if rows > 2 else 0.0, seed=7)
    weight = randn(rows, seed=3) if weighted else None
    r = ops.head_loss(x, W, t, row_weight=weight)
    want = R.head(x, W, t, row_weight=weight)
    for name, got in zip(("dx", "dw"), ops.head_backward(x, W, t, r.lse, row_weight=weight)):
        off, least = (got.double() - want[name]).norm(), (want[name].to(BF16).double() - want[name]).norm()
        assert float(off / least) < 1.02, name


def test_head_in_several_pieces_one_gradient_at_a_time():
    """The scratch that is asked for without knowing which gradients are wanted serves either of them alone, with the same bits."""
    x, W, t = problem(16000, 20000, 16, BF16, 0.1)
    r = ops.head_loss(x, W, t)
    dx, dW = ops.head_backward(x, W, t, r.lse)
    assert torch.equal(ops.head_backward(x, W, t, r.lse, need_dweight=False)[0], dx)
    assert torch.equal(ops.head_backward(x, W, t, r.lse, need_dx=False)[1], dW)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_head_large_logits(dtype):
    """Logits of some hundreds: the maximum is taken out before the exponential, a sure row has loss 0 and no gradient."""
    x, W, t = problem(70, 200, 32, dtype)
    x = (x.float() * 40).to(dtype)
    sure = ops.head_loss(x, W, (x.float() @ W.float().t()).argmax(1))
    assert bool(torch.isfinite(sure.row_loss).all()) and sure.row_loss.min().item() >= -1e-4
    check_head(x, W, t)


def test_head_gradient_is_the_derivative():
    """Central differences in 64 bits of the plain loss against the kernels in fp32."""
    x, W, t = problem(5, 30, 12, F32)
    weight = randn(5, seed=8)
    r = ops.head_loss(x, W, t, row_weight=weight)
    dx, dW = ops.head_backward(x, W, t, r.lse, row_weight=weight)

    def value(x, W):
        s = x @ W.t()
        return float(((torch.logsumexp(s, 1) - s.gather(1, t[:, None])[:, 0]) * weight.double()).mean())

    x64, W64, step = x.double(), W.double(), 1e-6
    for at, got in ((x64, dx), (W64, dW)):
        for i in range(0, at.numel(), 7):
            d = torch.zeros_like(at).view(-1)
            d[i] = step
            args = lambda s: [z + s * d.view(z.shape) if z is at else z for z in (x64, W64)]      # noqa: E731
            slope = (value(*args(1)) - value(*args(-1))) / (2 * step)
            assert abs(slope - got.view(-1)[i].item()) < 1e-6


# ---- places past 32 bits -----------------------------------------------------------------------------------------------

def test_dropout_of_more_than_2_to_the_32_elements():
    rows, cols = 66000, 65600
    x = torch.ones(rows, cols, dtype=BF16, device="cuda")
    assert x.numel() > 1 << 32
    ops.dropout(x, 0.25, ops.Rng(8, 9), out=x)
    for first in (0, 65535, rows - 1):
        f = R.factors(1, cols, 0.25, 8, 9, first)[0].to(BF16)
        assert torch.equal(x[first].cpu(), f)


def test_norm_of_more_than_2_to_the_32_elements():
    rows, cols = 262500, 16384
    x = torch.empty(rows, cols, dtype=BF16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(1))
    w = torch.ones(cols, dtype=BF16, device="cuda")
    assert x.numel() > 1 << 32
    n = ops.rms_norm(x, w)
    for part in (slice(0, 3), slice(rows // 2, rows // 2 + 2), slice(rows - 3, rows)):
        assert torch.equal(n.y[part], ops.rms_norm(x[part].clone(), w).y)
    dx, _, dw = ops.rms_norm_backward(n.y, x, w, n.rstd, grad_dtype=F32)
    assert torch.equal(dx[-3:], ops.rms_norm_backward(n.y[-3:].clone(), x[-3:].clone(), w, n.rstd[-3:].clone())[0])
    # sum over the rows of y^2: rows times the mean square of a normed row, 1, within five standard deviations (2 / rows)^0.5
    assert abs(dw.double().mean().item() / rows - 1) < 5 * (2 / rows / cols) ** 0.5 + 1e-4


def test_head_of_more_than_2_to_the_32_bytes():
    rows, vocab, cols = 3, 1060000, 2048
    W = torch.empty(vocab, cols, dtype=BF16, device="cuda").normal_(std=0.05, generator=torch.Generator("cuda").manual_seed(2))
    assert W.numel() * 2 > 1 << 32
    x = randn(rows, cols, dtype=BF16, seed=3)
    t = torch.tensor([0, vocab - 1, vocab // 2], device="cuda")
    s = torch.cat([x.double() @ c.double().t() for c in W.split(100000)], 1)
    off = (cols + 2) * R.U * (x.double().abs() @ W[:1000].double().abs().t()).amax() * 4        # rows of W are alike: four times the largest of 1000
    r = ops.head_loss(x, W, t)
    lse = torch.logsumexp(s, 1)
    R.within("lse", r.lse, lse, off + 2.0 ** -19)
    R.within("row_loss", r.row_loss, lse - s.gather(1, t[:, None])[:, 0], 2 * off + 2.0 ** -18)
    _, dW = ops.head_backward(x, W, t, r.lse)
    at = torch.tensor([0, 1, vocab // 2, vocab - 2, vocab - 1], device="cuda")
    p = (s[:, at] - lse[:, None]).exp() - (t[:, None] == at[None]).double()
    want = p.t() @ x.double() / rows
    # P rounded to bf16, its exponentials off by twice a logit's bound; then dW rounded
    R.within("dweight", dW[at], want, ((2.0 ** -8 + 4 * off + 2.0 ** -18) * p.abs()).t() @ x.double().abs() / rows * (1 + 2.0 ** -7), BF16)


# ---- together ---------------------------------------------------------------------------------------------------------

def model_end(x, res, g, W, t, rng):
    n = ops.rms_norm(x, g, residual=res, p=0.1, rng=rng)
    r = ops.head_loss(n.y, W, t)
    dy, dW = ops.head_backward(n.y, W, t, r.lse)
    dx, dres, dg = ops.rms_norm_backward(dy, n.h, g, n.rstd, p=0.1, rng=rng)
    return [r.loss, r.row_loss, dW, dx, dres, dg]


def test_same_inputs_same_bits_on_any_stream_and_two_calls_at_once():
    x, W, t = problem(500, 1500, 128, BF16, 0.1)
    res, g = randn(500, 128, dtype=BF16, seed=2), torch.ones(128, dtype=BF16, device="cuda")
    first = model_end(x, res, g, W, t, ops.Rng(1))
    other = model_end(res, x, g, W, t, ops.Rng(1))
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(a):
            p = model_end(x, res, g, W, t, ops.Rng(1))
        with torch.cuda.stream(b):
            q = model_end(res, x, g, W, t, ops.Rng(1))
    torch.cuda.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(first, p)) and all(torch.equal(u, v) for u, v in zip(other, q))


def test_captured_into_a_graph():
    """Replays with new inputs, new targets (another number of rows that count) and new masks from a counter on the device."""
    rows, vocab, cols = 300, 900, 72
    x, W, t = problem(rows, vocab, cols, BF16)
    res, g = randn(rows, cols, dtype=BF16, seed=2), torch.ones(cols, dtype=BF16, device="cuda")
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        model_end(x, res, g, W, t, ops.Rng(5, 0, counter))
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = model_end(x, res, g, W, t, ops.Rng(5, 0, counter))
    losses = set()
    for i in range(4):
        nx, nW, nt = problem(rows, vocab, cols, BF16, 0.2 * i, seed=10 + i)
        x.copy_(nx); W.copy_(nW); t.copy_(nt); counter.fill_(i)
        graph.replay()
        torch.cuda.synchronize()
        eager = model_end(x, res, g, W, t, ops.Rng(5, i))
        assert all(torch.equal(u, v) for u, v in zip(out, eager)), i
        losses.add(out[0].item())
    assert len(losses) == 4


@pytest.mark.parametrize("name,vocab", [("llama_60m", None), ("gpt2_350m", 700), ("llama_1b", 1100)])
def test_end_of_a_table_and_its_optimizer_step(name, vocab):
    """LMHead writes the gradients of a table's norm and head blocks (tied, untied; fp32 masters, bf16) and AdaPM.step takes them."""
    from dataclasses import replace
    from paper_2510_09103_amd import workloads as WL
    from paper_2510_09103_amd.head import LMHead
    from paper_2510_09103_amd.optimizer import AdaPM, make_hparams
    wl = WL.CONFIGS[name]()
    keep = [b for b in wl.blocks if b.name in ("wte", "embed", "ln_f", "norm_f", "lm_head")]
    wl = replace(wl, blocks=tuple(replace(b, rows=vocab) if vocab and b.cols > 1 else b for b in keep))
    params = WL.initial_params(wl, device="cuda")
    grads = WL.GradientStream(wl, device="cuda").next()
    before = [g.clone() for g in grads]
    end = LMHead(wl.blocks, p=0.1)
    x, res, t = WL.head_batch(wl, 200, masked=0.1, device="cuda")
    out = end.step(params, grads, x, res, t, 3)
    W, gain = params[end.head].to(x.dtype), params[end.norm]
    f = R.factors(200, x.shape[1], 0.1, end.seed, 3).cuda()
    sum64 = x.double() * f + res.double()
    n = ops.rms_norm(x, gain, residual=res, p=0.1, rng=ops.Rng(end.seed, 3))
    # the product and the sum are rounded to fp32 before the rounding to bf16, which can then fall to the other side
    R.within("h", n.h, sum64, 3 * R.U * ((x.double() * f).abs() + sum64.abs()), x.dtype)
    h = n.h
    want = R.head(n.y, W, t, dtype=x.dtype)
    R.within("loss", out.loss, want["loss"], want["loss_off"])
    R.within("head", grads[end.head], want["dw"], want["dw_off"], x.dtype)
    dy = ops.head_backward(n.y, W, t, ops.head_loss(n.y, W, t).lse)[0]
    dres, size, dg, dg_size = R.norm_backward(dy, h, gain.view(-1), n.rstd)
    R.within("dresidual", out.dresidual, dres, 80 * R.U * size, x.dtype)
    R.within("norm", grads[end.norm].view(-1), dg, 91 * R.U * dg_size, grads[end.norm].dtype)
    for i, (a, b) in enumerate(zip(before, grads)):
        assert torch.equal(a, b) == (i not in (end.norm, end.head))
    # the step on these buffers is the step on copies of them
    copies = [p.clone() for p in params]
    for p, g in ((params, grads), (copies, [g.clone() for g in grads])):
        AdaPM(wl.blocks, make_hparams()).step(p, g, 1, 1e-3)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(params, copies))


def test_replays_beside_an_eager_optimizer_step():
    """The end of a model captured into a graph whose gradient buffers an eager AdaPM.step reads between the replays."""
    from dataclasses import replace
    from paper_2510_09103_amd import workloads as WL
    from paper_2510_09103_amd.head import LMHead
    from paper_2510_09103_amd.optimizer import AdaPM, make_hparams
    wl = WL.gpt2_350m()
    wl = replace(wl, blocks=tuple(replace(b, rows=600) if b.name == "wte" else b for b in wl.blocks if b.name in ("wte", "ln_f")))
    x, res, t = WL.head_batch(wl, 150, device="cuda")
    runs = []
    for captured in (False, True):
        params = WL.initial_params(wl, device="cuda")
        grads = [torch.zeros_like(p) for p in params]
        end, opt = LMHead(wl.blocks, p=0.2), AdaPM(wl.blocks, make_hparams())
        end.step(params, grads, x, res, t, 1)
        torch.cuda.synchronize()
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                out = end.step(params, grads, x, res, t, 1)
        for step in range(1, 4):
            if captured:
                graph.replay()
            else:
                out = end.step(params, grads, x, res, t, 1)
            opt.step(params, grads, step, 1e-2)
            torch.cuda.synchronize()
        runs.append([*params, *grads, out.loss])
    assert all(torch.equal(a, b) for a, b in zip(*runs))
