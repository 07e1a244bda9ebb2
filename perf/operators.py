"""The end of a language model as users of this package run it in a training step, one operator to a case:

  dropout        y = residual + dropout(x), the mask made from (seed, offset, row, column) and never stored
  norm           h = residual + dropout(x), y = h / sqrt(mean h^2 + eps) * weight, y in the type of h or in e4m3 with a scale per row
  norm_backward  the gradients of x, residual and weight
  head_loss      softmax cross entropy of x W^T against targets: the loss, each row's loss and its log-sum-exp
  head_step      the same and the gradients of x and W behind it

`own = False` computes the plain form in torch, `own = True` calls the package's operators.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_EPS = 1e-5


def listed():
    return [
        # dropout on the embeddings of a GPT-2-1.5B batch of 8 x 1024 tokens, p = 0.1 as in its published recipe
        _drop("dropout_gpt2_1p5b", 8192, 1600, "bf16", 0.1, residual=False),
        # a small fp32 experiment with a width that is no whole number of vectors, added to the residual
        _drop("dropout_residual_odd_f32", 1023, 257, "f32", 0.25, residual=True),
        # one token of a LLaMA-1B through the norm in front of an 8-bit projection: latency is everything
        _norm("norm_one_token_e4m3", 1, 2048, "bf16", out="e4m3"),
        # a training batch of the GPT-2-1.5B shape: residual dropout, addition and norm in one pass
        _norm("norm_dropout_gpt2_1p5b", 8192, 1600, "bf16", p=0.1),
        # a wide MLP-side norm in fp32 with the ragged width of the LLaMA-1B table (5461), without a residual
        _norm("norm_ragged_f32", 2047, 5461, "f32", residual=False, weight="f32"),
        # backward of the final norm of a LLaMA-1B micro-batch, with the gradient of the residual stream and dropout
        _norm("norm_backward_llama_1b", 16384, 2048, "bf16", p=0.1, backward=True),
        # the same on the fp32 parameters and bf16 activations of the LLaMA-60M table, a short odd batch
        _norm("norm_backward_llama_60m", 300, 512, "bf16", weight="f32", backward=True),
        # scoring of one token with the LLaMA-1B head: W is read once, everything else is latency
        _head("head_loss_one_token", 1, 32000, 2048, "bf16"),
        # evaluation of a GPT-2-1.5B batch of 4 x 1024 tokens over the unpadded vocabulary
        _head("head_loss_gpt2_1p5b", 4096, 50257, 1600, "bf16"),
        # supervised fine-tuning of a LLaMA-60M: a third of the tokens (prompts, padding) carry no target
        _head("head_step_llama_60m_masked", 8192, 32000, 512, "bf16", backward=True, masked=0.33),
        # pre-training micro-batch of a LLaMA-1B, the largest case
        _head("head_step_llama_1b", 8192, 32000, 2048, "bf16", backward=True),
        # a small fp32 model with rewards on the rows (policy gradients), sizes that are no multiple of anything
        _head("head_step_weighted_odd_f32", 997, 4099, 250, "f32", backward=True, masked=0.1, weighted=True),
    ]


def _drop(name, rows, cols, dtype, p, residual):
    return dict(name=name, op="dropout", rows=rows, cols=cols, dtype=dtype, p=p, residual=residual)


def _norm(name, rows, cols, dtype, *, residual=True, p=0.0, out="same", weight="bf16", backward=False):
    return dict(name=name, op="norm_backward" if backward else "norm", rows=rows, cols=cols, dtype=dtype, residual=residual, p=p, out=out,
                weight=weight)


def _head(name, rows, vocab, cols, dtype, *, backward=False, masked=0.0, weighted=False):
    return dict(name=name, op="head_step" if backward else "head_loss", rows=rows, vocab=vocab, cols=cols, dtype=dtype, masked=masked,
                weighted=weighted)


def _spread(rng, lo, hi):
    return round(lo * (hi / lo) ** rng.random())


def draw(rng):
    """One more case of the same ranges: one to 16384 tokens, widths of 32 to 8192 (whole vectors mostly, odd ones among them),
    vocabularies of 500 to 50304 entries, both types, with and without dropout, residual, masked rows and row weights."""
    op = rng.choice(["dropout", "norm", "norm_backward", "head_loss", "head_step", "head_step"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    p = rng.choice([0.0, 0.1, round(0.01 + 0.5 * rng.random(), 3)])

    def width(lo, hi):
        n = _spread(rng, lo, hi)
        kind = rng.random()
        return max(lo, 64 * round(n / 64)) if kind < 0.5 else max(8, 8 * round(n / 8)) if kind < 0.8 else n

    if op.startswith("head"):
        rows, cols, vocab = _spread(rng, 1, 8192), width(32, 2048), _spread(rng, 500, 50304)
        if dtype == "f32":      # small models; the arithmetic costs sixteen times as much
            rows, cols, vocab = _spread(rng, 1, 1024), width(32, 512), _spread(rng, 500, 32000)
        c = _head("", rows, vocab, cols, dtype, backward=op == "head_step", masked=rng.choice([0.0, 0.0, 0.1, 0.5]),
                  weighted=rng.random() < 0.3)
        while 3 * c["rows"] * c["vocab"] * c["cols"] > 3 * 8192 * 32000 * 2048:
            c["rows"] //= 2
    else:
        rows, cols = _spread(rng, 1, 16384), width(32, 8192)
        while rows * cols > 16384 * 2048:
            rows //= 2
        if op == "dropout":
            c = _drop("", rows, cols, dtype, p or 0.1, residual=rng.random() < 0.5)
        else:
            back = op == "norm_backward"
            c = _norm("", rows, cols, dtype, residual=rng.random() < 0.7, p=p, weight=rng.choice([dtype, "f32"]), backward=back,
                      out="same" if back else rng.choice(["same", "same", "e4m3"]))
    del c["name"]
    return c


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)

    def randn(*size):
        return torch.randn(*size, device="cuda", generator=g)

    dt, rows, cols = _DT[case["dtype"]], case["rows"], case["cols"]
    s = {"case": case, "seed": 0x5EED0000 + seed, "offset": 1000 + seed % 97}
    if case["op"].startswith("head"):
        vocab = case["vocab"]
        # the weight of a trained head, hidden states behind a norm, some of them turned towards their target's row
        s["weight"] = (randn(vocab, cols) * (0.6 / math.sqrt(cols))).to(dt)
        zipf = torch.rand(rows, device="cuda", generator=g, dtype=torch.float64)
        s["targets"] = (vocab ** zipf).long().clamp_(1, vocab) - 1
        sure = torch.rand(rows, 1, device="cuda", generator=g) * 10.0
        s["x"] = (randn(rows, cols) + sure * s["weight"][s["targets"]].float()).to(dt)
        if case["masked"]:
            s["targets"][torch.rand(rows, device="cuda", generator=g) < case["masked"]] = -100
        s["row_weight"] = randn(rows) if case["weighted"] else None
        return s
    s["x"] = (randn(rows, cols) * 0.7).to(dt)
    if case["op"] == "dropout":
        s["residual"] = randn(rows, cols).to(dt) if case["residual"] else None
        return s
    # a residual stream as deep models have it: a few columns are an order of magnitude larger
    big = 1.0 + 9.0 * (torch.rand(cols, device="cuda", generator=g) < 0.01)
    s["residual"] = (randn(rows, cols) * big).to(dt) if case["residual"] else None
    s["weight"] = (1.0 + 0.2 * randn(cols)).to(_DT[case["weight"]])
    if case["op"] == "norm_backward":
        # the saved tensors of the forward pass, and the gradients that arrive
        h = s["x"].float() + (s.pop("residual").float() if case["residual"] else 0.0)
        s["h"] = h.to(dt)
        s["rstd"] = torch.rsqrt(s["h"].double().square().mean(1) + _EPS).float()
        s["dy"] = (randn(rows, cols) * 1e-3).to(dt)
        s["dh"] = (randn(rows, cols) * 1e-3).to(dt) if case["residual"] else None
        del s["x"]
    return s


def run(state):
    return (_own if own else _plain)[state["case"]["op"]](state)


# ---- the package's operators --------------------------------------------------------------------------------------

def _rng(s):
    from paper_2510_09103_amd import ops
    return ops.Rng(s["seed"], s["offset"])


def _own_dropout(s):
    from paper_2510_09103_amd import ops
    return {"y": ops.dropout(s["x"], s["case"]["p"], _rng(s), residual=s["residual"])}


def _own_norm(s):
    from paper_2510_09103_amd import ops
    c = s["case"]
    n = ops.rms_norm(s["x"], s["weight"], eps=_EPS, residual=s["residual"], p=c["p"], rng=_rng(s),
                     out_dtype=torch.float8_e4m3fn if c["out"] == "e4m3" else None)
    out = {"y": n.y, "rstd": n.rstd}
    if n.h is not s["x"]:
        out["h"] = n.h
    if c["out"] == "e4m3":
        out.update(y=n.y.to(torch.bfloat16), scale=n.scale)     # the values of the 8-bit numbers, exact in bf16
    return out


def _own_norm_backward(s):
    from paper_2510_09103_amd import ops
    c = s["case"]
    dx, dres, dw = ops.rms_norm_backward(s["dy"], s["h"], s["weight"], s["rstd"], dh=s["dh"], p=c["p"], rng=_rng(s))
    return {"dx": dx, "dresidual": dres, "dweight": dw}


def _own_head_loss(s):
    from paper_2510_09103_amd import ops
    r = ops.head_loss(s["x"], s["weight"], s["targets"], row_weight=s["row_weight"])
    return {"loss": r.loss, "row_loss": r.row_loss, "lse": r.lse}


def _own_head_step(s):
    from paper_2510_09103_amd import ops
    r = ops.head_loss(s["x"], s["weight"], s["targets"], row_weight=s["row_weight"])
    dx, dw = ops.head_backward(s["x"], s["weight"], s["targets"], r.lse, row_weight=s["row_weight"])
    return {"loss": r.loss, "row_loss": r.row_loss, "lse": r.lse, "dx": dx, "dweight": dw}


_own = {"dropout": _own_dropout, "norm": _own_norm, "norm_backward": _own_norm_backward, "head_loss": _own_head_loss,
        "head_step": _own_head_step}


# ---- the plain forms ------------------------------------------------------------------------------------------------

def _factor(s, rows, cols, dtype):
    """0 or 1 / (1 - p) for every element.  Philox4x32 with ten rounds (Salmon et al., 2011): counter (column / 8, row, offset low,
    offset high), key = seed; an element takes the 16 bits of its place among the eight of a counter."""
    mask = 0xFFFFFFFF
    thr = min(65535, math.floor(65536 * s["case"]["p"] + 0.5))
    groups = (cols + 7) // 8
    c0 = torch.arange(groups, device="cuda").expand(rows, groups)
    c1 = torch.arange(rows, device="cuda")[:, None].expand(rows, groups)
    c2 = torch.full_like(c0, s["offset"] & mask)
    c3 = torch.full_like(c0, s["offset"] >> 32)
    k0, k1 = s["seed"] & mask, s["seed"] >> 32
    for _ in range(10):
        a, b = 0xD2511F53 * c0, 0xCD9E8D57 * c2
        c0, c1, c2, c3 = ((b >> 32) & mask) ^ c1 ^ k0, b & mask, ((a >> 32) & mask) ^ c3 ^ k1, a & mask
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    words = torch.stack([c0 & 0xFFFF, c0 >> 16, c1 & 0xFFFF, c1 >> 16, c2 & 0xFFFF, c2 >> 16, c3 & 0xFFFF, c3 >> 16], -1)
    keep = words.view(rows, groups * 8)[:, :cols] >= thr
    return keep.to(dtype) * (65536.0 / (65536 - thr))


def _plain_dropout(s):
    x = s["x"]
    y = x.float() * _factor(s, *x.shape, torch.float32)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(x.dtype)}


def _plain_norm(s):
    c, x = s["case"], s["x"]
    h = x
    if c["p"] or c["residual"]:
        h = x.float()
        if c["p"]:
            h = h * _factor(s, *x.shape, torch.float32)
        if c["residual"]:
            h = h + s["residual"].float()
        h = h.to(x.dtype)       # the residual stream is kept in its type, and the norm is of what is kept
    f = h.float()
    rstd = torch.rsqrt(f.square().mean(1) + _EPS)
    y = f * rstd[:, None] * s["weight"].float()
    out = {"y": y.to(x.dtype), "rstd": rstd}
    if h is not x:
        out["h"] = h
    if c["out"] == "e4m3":
        amax = y.abs().amax(1)
        scale = torch.where(amax > 0, amax / 448.0, torch.ones_like(amax))
        q = (y * (1.0 / scale)[:, None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
        out.update(y=q.to(torch.bfloat16), scale=scale)
    return out


def _plain_norm_backward(s):
    c, dt = s["case"], s["dy"].dtype
    n = s["h"].float() * s["rstd"][:, None]
    dy = s["dy"].float()
    dn = dy * s["weight"].float()
    dh = s["rstd"][:, None] * (dn - n * (dn * n).mean(1, keepdim=True))
    if s["dh"] is not None:
        dh = dh + s["dh"].float()
    dx = dh * _factor(s, *dy.shape, torch.float32) if c["p"] else dh
    return {"dx": dx.to(dt), "dresidual": dh.to(dt), "dweight": (dy * n).sum(0).to(s["weight"].dtype)}


def _plain_head(s):
    """Logits, the rows that count, and the outputs of the loss."""
    x, w, t = s["x"].float(), s["weight"].float(), s["targets"]
    valid = (t >= 0) & (t < w.shape[0])
    logits = x @ w.t()
    top = logits.amax(1)
    lse = top + (logits - top[:, None]).exp().sum(1).log()
    row = lse - logits.gather(1, t.clamp(0, w.shape[0] - 1)[:, None])[:, 0]
    zero = torch.zeros_like(lse)
    row, lse = torch.where(valid, row, zero), torch.where(valid, lse, zero)
    count = valid.sum().clamp(min=1).float()
    weight = valid.float() if s["row_weight"] is None else torch.where(valid, s["row_weight"], zero)
    loss = (weight.double() * row.double()).sum().float() / count
    return logits, weight, count, {"loss": loss, "row_loss": row, "lse": lse}


def _plain_head_loss(s):
    return _plain_head(s)[3]


def _plain_head_step(s):
    p, weight, count, out = _plain_head(s)
    p = p.sub_(out["lse"][:, None]).exp_()
    p.scatter_add_(1, s["targets"].clamp(0, p.shape[1] - 1)[:, None], torch.full_like(weight, -1.0)[:, None])
    p.mul_((weight / count)[:, None])
    dt = s["x"].dtype
    return dict(out, dx=(p @ s["weight"].float()).to(dt), dweight=(p.t() @ s["x"].float()).to(dt))


_plain = {"dropout": _plain_dropout, "norm": _plain_norm, "norm_backward": _plain_norm_backward, "head_loss": _plain_head_loss,
          "head_step": _plain_head_step}


# ---- what one pass cannot do without ---------------------------------------------------------------------------------

def work(case):
    size = {"f32": 4, "bf16": 2, "e4m3": 1}
    e, n = size[case["dtype"]], case["rows"] * case["cols"]
    if case["op"] == "dropout":
        # x, the residual and y; a multiplication and an addition for each element
        return {"bytes": n * e * (3 if case["residual"] else 2), "flops": 2 * n}
    if case["op"] == "norm":
        fused = bool(case["p"] or case["residual"])
        moved = e * (1 + bool(case["residual"]) + fused) + (e if case["out"] == "same" else 1)
        return {"bytes": n * moved + case["cols"] * size[case["weight"]] + 4 * case["rows"], "flops": 6 * n}
    if case["op"] == "norm_backward":
        moved = e * (3 + bool(case["residual"]) + bool(case["p"]))     # dy, h, dx; dh; dresidual where it is not dx
        return {"bytes": n * moved + 2 * case["cols"] * size[case["weight"]] + 4 * case["rows"], "flops": 10 * n}
    # the rows that count; x and W in, a product; their gradients out and two products more, beside the forward one
    live = max(1.0, case["rows"] * (1.0 - case["masked"]))
    step = case["op"] == "head_step"
    return {"bytes": (live + case["vocab"]) * case["cols"] * e * (2 if step else 1) + 16 * case["rows"],
            "flops": live * case["vocab"] * case["cols"] * (6 if step else 2)}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------

def _mulhilo(a, m):
    """High and low 32 bits of m * a (int64 tensors of 32-bit values) from 16-bit halves."""
    lo, hi = m * (a & 0xFFFF), m * (a >> 16)
    mid = hi + (lo >> 16)
    return mid >> 16, ((mid & 0xFFFF) << 16) | (lo & 0xFFFF)


def _kept(case, seed, offset):
    """The mask from the generator's definition, element by element."""
    rows, cols = case["rows"], case["cols"]
    col = torch.arange(cols, device="cuda").expand(rows, cols)
    ctr = [col >> 3, torch.arange(rows, device="cuda")[:, None].expand(rows, cols), torch.full_like(col, offset % 2**32),
           torch.full_like(col, offset // 2**32)]
    key = [seed % 2**32, seed // 2**32]
    for r in range(10):
        h0, l0 = _mulhilo(ctr[0], 0xD2511F53)
        h1, l1 = _mulhilo(ctr[2], 0xCD9E8D57)
        ctr = [h1 ^ ctr[1] ^ ((key[0] + r * 0x9E3779B9) % 2**32), l1, h0 ^ ctr[3] ^ ((key[1] + r * 0xBB67AE85) % 2**32), l0]
    word = torch.where(col % 8 < 4, torch.where(col % 8 < 2, ctr[0], ctr[1]), torch.where(col % 8 < 6, ctr[2], ctr[3]))
    bits = torch.where(col % 2 == 0, word % 65536, word // 65536)
    drop = min(65535, int(case["p"] * 65536 + 0.5))
    return (bits >= drop).double() * 65536 / (65536 - drop)


def exact(case, seed):
    s = prepare(case, seed)
    x64 = {k: v.double() for k, v in s.items() if torch.is_tensor(v) and v.is_floating_point()}
    if case["op"] == "dropout":
        y = x64["x"] * _kept(case, s["seed"], s["offset"])
        return {"y": y + x64["residual"] if case["residual"] else y}
    if case["op"] == "norm":
        h = x64["x"] * _kept(case, s["seed"], s["offset"]) if case["p"] else x64["x"]
        h = h + x64["residual"] if case["residual"] else h
        kept = h.to(_DT[case["dtype"]]).double()         # the definition: the norm of the residual stream as it is kept
        rstd = (kept.pow(2).sum(1) / case["cols"] + _EPS) ** -0.5
        y = kept * rstd[:, None] * x64["weight"]
        out = {"y": y, "rstd": rstd}
        if case["p"] or case["residual"]:
            out["h"] = h
        if case["out"] == "e4m3":
            amax = y.abs().max(1).values
            out["scale"] = torch.where(amax > 0, amax / 448, torch.ones_like(amax))
            q = y / out["scale"][:, None]
            step = 2.0 ** (torch.frexp(q).exponent.clamp(min=-5) - 4).double()      # four significant bits, from 2^-6 on
            out["y"] = (q / step).round() * step
        return out
    if case["op"] == "norm_backward":
        n = x64["h"] * x64["rstd"][:, None]
        dn = x64["dy"] * x64["weight"]
        d = x64["rstd"][:, None] * (dn - n * ((dn * n).sum(1) / case["cols"])[:, None])
        d = d + x64["dh"] if case["residual"] else d
        return {"dx": d * _kept(case, s["seed"], s["offset"]) if case["p"] else d, "dresidual": d,
                "dweight": (x64["dy"] * n).sum(0)}
    x, w, t = x64["x"], x64["weight"], s["targets"]
    live = torch.nonzero((t >= 0) & (t < case["vocab"]))[:, 0]
    row, lse = torch.zeros_like(x[:, 0]), torch.zeros_like(x[:, 0])
    dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    scale = (x64["row_weight"] if case["weighted"] else torch.ones_like(row)) / max(1, len(live))
    for at in live.split(2048):
        z = x[at] @ w.t()
        lse[at] = torch.logsumexp(z, 1)
        row[at] = lse[at] - z[torch.arange(len(at)), t[at]]
        if case["op"] == "head_step":
            p = torch.softmax(z, 1)
            p[torch.arange(len(at)), t[at]] -= 1.0
            p *= scale[at][:, None]
            dx[at] = p @ w
            dw += p.t() @ x[at]
    out = {"loss": (row * scale).sum(), "row_loss": row, "lse": lse}
    return dict(out, dx=dx, dweight=dw) if case["op"] == "head_step" else out
