"""Refusals and layouts of the operators of a model's end, through the C ABI and on tensors.  No GPU: every call here is turned down
before anything is launched."""
import ctypes as C

import pytest
import torch

import ops_reference as R
from paper_2510_09103_amd import binding as B
from paper_2510_09103_amd import ops

A = 1 << 20                                     # an address that is never used
OKR = B.rows(A, 64)


def refused(call, *words):
    with pytest.raises(B.AdapmError) as e:
        call()
    assert e.value.status == B.ADAPM_EINVAL
    for w in words:
        assert w in str(e.value), str(e.value)


def test_struct_sizes():
    assert [C.sizeof(t) for t in (B.adapm_rows_t, B.adapm_dropout_t, B.adapm_norm_t, B.adapm_head_t)] == [16, 32, 40, 40]


def test_generator_known_answers():
    """The published vectors of Philox4x32-10."""
    assert R.philox((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert R.philox((R.LOW,) * 4, (R.LOW,) * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


@pytest.mark.parametrize("kw,word", [
    (dict(y=B.rows()), "y is null"), (dict(x=B.rows(A + 1, 64)), "x is not aligned"), (dict(x=B.rows(A, 63)), "x: row stride"),
    (dict(residual=B.rows(A, 3)), "residual"), (dict(n=-1), "rows"), (dict(cols=0), "cols"), (dict(n=1 << 33), "rows"),
    (dict(n=1 << 32, cols=1 << 20), "out of range"),
    (dict(dtype=2), "dtype"), (dict(dtype=-1), "dtype"), (dict(drop=None), "drop is null"), (dict(p=1.0), "probability"), (dict(p=-0.1), "probability"),
    (dict(p=float("nan")), "probability"), (dict(at=A + 4), "offset_dev"),
])
def test_dropout_refusals(kw, word):
    d = dict(y=OKR, x=OKR, residual=B.rows(), n=4, cols=64, dtype=B.ADAPM_BF16, p=0.1, at=None)
    d.update(kw)
    drop = d.get("drop", B.adapm_dropout_t(1, 2, d["at"], d["p"], 0))
    refused(lambda: B.adapm_dropout(d["y"], d["x"], d["residual"], d["n"], d["cols"], d["dtype"], drop), word)


def norm(**kw):
    d = dict(rows=4, cols=64, dtype=1, weight_dtype=0, y_dtype=1, grad_dtype=0, eps=1e-5)
    d.update(kw)
    return B.adapm_norm_t(d["rows"], d["cols"], d["dtype"], d["weight_dtype"], d["y_dtype"], d["grad_dtype"], d["eps"], 0)


@pytest.mark.parametrize("n,kw,word", [
    (None, {}, "norm is null"), (norm(rows=-1), {}, "rows"), (norm(cols=0), {}, "cols"), (norm(cols=16385), {}, "cols"), (norm(dtype=2), {}, "dtype"),
    (norm(weight_dtype=2), {}, "dtype"), (norm(y_dtype=0), {}, "y_dtype"), (norm(y_dtype=3), {}, "y_dtype"), (norm(eps=-1.0), {}, "eps"),
    (norm(eps=float("inf")), {}, "eps"), (norm(), dict(x=B.rows()), "x is null"), (norm(), dict(y=B.rows(A, 8)), "y: row stride"),
    (norm(), dict(residual=OKR, h=B.rows()), "h is null"), (norm(), dict(h=B.rows(), drop=B.adapm_dropout_t(0, 0, None, 0.5, 0)), "h is null"),
    (norm(), dict(h=B.rows(A + 1, 64)), "h is not aligned"), (norm(), dict(weight=0), "weight is null"), (norm(), dict(weight=A + 2), "weight"),
    (norm(), dict(rstd=0), "rstd"), (norm(y_dtype=2), dict(scale=0), "y_scale"), (norm(), dict(drop=B.adapm_dropout_t(0, 0, None, 2.0, 0)), "probability"),
    (norm(), dict(h=OKR, y=OKR), "y is h"),
])
def test_norm_forward_refusals(n, kw, word):
    d = dict(x=OKR, residual=B.rows(), h=B.rows(2 * A, 64), weight=A, y=OKR, scale=A, rstd=A, drop=None)
    d.update(kw)
    refused(lambda: B.adapm_norm_forward(n, d["x"], d["residual"], d["h"], d["weight"], d["y"], d["scale"], d["rstd"], d["drop"]), word)


@pytest.mark.parametrize("n,kw,word", [
    (norm(cols=0), {}, "cols"), (norm(grad_dtype=2), {}, "grad_dtype"), (norm(), dict(dy=B.rows()), "dy is null"),
    (norm(), dict(h=B.rows()), "h is null"), (norm(), dict(dx=B.rows()), "dx is null"), (norm(), dict(dh=B.rows(A, 1)), "dh: row stride"),
    (norm(), dict(dres=B.rows(A + 1, 64)), "dresidual"), (norm(), dict(dw=0), "dweight"), (norm(), dict(dw=A + 2), "dweight"),
    (norm(), dict(weight=0), "weight"), (norm(), dict(rstd=0), "rstd"), (norm(), dict(ws=0), "workspace"), (norm(), dict(ws=A + 64), "workspace"),
    (norm(), dict(drop=B.adapm_dropout_t(0, 0, None, 0.5, 0)), "dx and dresidual differ"),
])
def test_norm_backward_refusals(n, kw, word):
    d = dict(dy=OKR, dh=B.rows(), h=OKR, weight=A, rstd=A, dx=OKR, dres=OKR, dw=A, ws=A, drop=None)
    d.update(kw)
    refused(lambda: B.adapm_norm_backward(n, d["dy"], d["dh"], d["h"], d["weight"], d["rstd"], d["dx"], d["dres"], d["dw"], d["drop"], d["ws"]), word)


def head(**kw):
    d = dict(rows=4, vocab=100, cols=64, dtype=1, reduction=1, scale=1.0)
    d.update(kw)
    return B.adapm_head_t(d["rows"], d["vocab"], d["cols"], d["dtype"], d["reduction"], d["scale"], 0)


BAD_HEADS = [(head(rows=-1), "rows"), (head(rows=(1 << 22) + 1), "rows"), (head(vocab=0), "vocab"), (head(vocab=(1 << 21) + 1), "vocab"),
             (head(cols=0), "cols"), (head(cols=(1 << 16) + 1), "cols"), (head(dtype=2), "dtype"), (head(reduction=2), "reduction"),
             (head(scale=float("nan")), "scale"), (None, "head is null")]


@pytest.mark.parametrize("h,kw,word", [(h, {}, w) for h, w in BAD_HEADS] + [
    (head(), dict(x=B.rows()), "x is null"), (head(), dict(x=B.rows(A + 1, 64)), "x is not aligned"), (head(), dict(w=B.rows(A, 63)), "weight"),
    (head(), dict(w=B.rows(A, 1 << 22)), "weight: row stride"), (head(), dict(t=0), "targets"), (head(), dict(t=A + 4), "targets"),
    (head(), dict(rw=A + 2), "row_weight"), (head(), dict(ws=0), "workspace"), (head(), dict(ws=A + 128), "workspace"),
    (head(), dict(size=256), "are needed"), (head(), dict(loss=0), "loss"), (head(), dict(row=0), "row_loss"), (head(), dict(lse=0), "lse"),
])
def test_head_loss_refusals(h, kw, word):
    d = dict(x=OKR, w=OKR, t=A, rw=0, loss=A, row=A, lse=A, ws=A, size=1 << 30)
    d.update(kw)
    refused(lambda: B.adapm_head_loss(h, d["x"], d["w"], d["t"], d["rw"], d["loss"], d["row"], d["lse"], d["ws"], d["size"]), word)


@pytest.mark.parametrize("h,kw,word", [(h, {}, w) for h, w in BAD_HEADS] + [
    (head(), dict(dx=B.rows(), dw=B.rows()), "both null"), (head(), dict(lse=0), "lse"), (head(), dict(up=A + 2), "upstream"),
    (head(), dict(dx=B.rows(A, 1)), "dx: row stride"), (head(), dict(dw=B.rows(A + 1, 64)), "dweight"), (head(), dict(size=0), "are needed"),
    (head(), dict(t=0), "targets"), (head(), dict(dw=OKR), "dweight is an input"), (head(), dict(dx=B.rows(5 * A, 64), dw=B.rows(5 * A, 64)), "dx is"),
    (head(), dict(w=B.rows(3 * A, 64), dw=B.rows(3 * A, 64)), "dweight is an input"), (head(), dict(w=B.rows(3 * A, 64), dx=B.rows(3 * A, 64)), "dx is"),
])
def test_head_backward_refusals(h, kw, word):
    d = dict(x=OKR, w=OKR, t=A, rw=0, lse=A, up=0, dx=B.rows(2 * A, 64), dw=B.rows(4 * A, 64), ws=A, size=1 << 30)
    d.update(kw)
    refused(lambda: B.adapm_head_backward(h, d["x"], d["w"], d["t"], d["rw"], d["lse"], d["up"], d["dx"], d["dw"], d["ws"], d["size"]), word)


def test_workspace_sizes():
    assert B.adapm_norm_workspace_bytes(norm(cols=0)) == 0 and B.adapm_head_workspace_bytes(head(vocab=0), OKR, True) == 0
    assert B.adapm_norm_workspace_bytes(norm(rows=0)) >= 4 * 64          # dweight of no rows is written too
    # the logits of a batch are never all there: 8192 x 50304 of them are 824 MB in bf16
    big = head(rows=8192, vocab=50304, cols=1024)
    w = B.rows(A, 1024)
    fwd, bwd = (B.adapm_head_workspace_bytes(big, w, b) for b in (False, True))
    x = 8192 * 1024 * 2
    assert x < fwd < x + 8 * 8192 * 800 and bwd < 2 * x + (256 << 20) + 4 * 8192 * 1024 * 8
    # rows of W that are no whole vectors are copied
    odd = B.adapm_head_workspace_bytes(big, B.rows(A, 1025), True)
    assert odd >= bwd + 50304 * 1024 * 2
    assert B.adapm_head_workspace_bytes(big, B.rows(A + 2, 1024), True) == odd


@pytest.mark.parametrize("dtype", [B.ADAPM_BF16, B.ADAPM_F32])
def test_more_tiles_than_a_launch_holds(dtype):
    for cols in (64, 1000, 16384):
        for rows in (1 << 15, 300000, 1 << 22):         # 2^36 logits
            h, w = head(rows=rows, vocab=(1 << 36) // rows, cols=cols, dtype=dtype), B.rows(A, cols)
            assert all(B.adapm_head_workspace_bytes(h, w, b) > 0 for b in (False, True))
        big, x = head(rows=1 << 22, vocab=1 << 21, cols=cols, dtype=dtype), B.rows(A, cols)
        assert B.adapm_head_workspace_bytes(big, w, False) == 0
        refused(lambda: B.adapm_head_loss(big, x, w, A, 0, A, A, A, A, 1 << 62), "too many for one call")


def test_tensors_are_checked():
    x, w = torch.zeros(4, 8), torch.ones(8)
    t = torch.zeros(4, dtype=torch.int64)
    for call in (lambda: ops.dropout(x, 0.1, ops.Rng(1)), lambda: ops.rms_norm(x, w), lambda: ops.rms_norm_backward(x, x, w, torch.ones(4)),
                 lambda: ops.head_loss(x, torch.zeros(5, 8), t), lambda: ops.head_backward(x, torch.zeros(5, 8), t, torch.zeros(4))):
        with pytest.raises(ValueError, match="a GPU tensor is wanted"):
            call()
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        ops.dropout(x.half(), 0.1, ops.Rng(1))


def test_end_of_a_table_finds_its_blocks():
    from paper_2510_09103_amd import workloads as WL
    from paper_2510_09103_amd.head import LMHead
    for name, norm, last, tied in (("llama_60m", "norm_f", "embed", True), ("gpt2_350m", "ln_f", "wte", True), ("llama_1b", "norm_f", "lm_head", False),
                                   ("gpt2_1p5b", "ln_f", "lm_head", False), ("llama_350m_paper", "ln_f", "wte", True)):
        wl = WL.CONFIGS[name]()
        end = LMHead(wl.blocks)
        assert (wl.blocks[end.norm].name, wl.blocks[end.head].name, end.tied) == (norm, last, tied)
    with pytest.raises(ValueError, match="final norm"):
        LMHead(WL.tiny_block().blocks)
    with pytest.raises(ValueError, match="columns"):
        LMHead([b for b in WL.gpt2_350m().blocks if b.name == "ln_f"] + [b for b in WL.llama_1b().blocks if b.name == "lm_head"])


def test_head_batch_is_seeded():
    from paper_2510_09103_amd import workloads as WL
    wl = WL.llama_60m()
    x, res, t = WL.head_batch(wl, 300, masked=0.3, seed=4)
    again = WL.head_batch(wl, 300, masked=0.3, seed=4)
    assert all(torch.equal(a, b) for a, b in zip((x, res, t), again)) and not torch.equal(x, WL.head_batch(wl, 300, seed=5)[0])
    assert x.dtype == torch.bfloat16 and x.shape == res.shape == (300, 512)
    # a binomial share of rows without a target: five standard deviations
    assert abs((t == -100).float().mean().item() - 0.3) < 5 * (0.21 / 300) ** 0.5 and t.max() < 32000 and t[t != -100].min() >= 0
