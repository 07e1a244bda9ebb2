"""The end of a model over a block table: residual dropout and addition, final norm, output head and loss, and their gradients written
into the gradient tensors of the table's blocks, where AdaPM.step reads them.

    h = residual + dropout(x);  y = h / sqrt(mean(h^2) + eps) * params[norm];  loss = cross entropy of y params[head]^T

The norm is the root-mean-square norm, whatever the table calls its vector.  A model whose final norm is a LayerNorm (GPT-2, blocks named
ln_f: the mean is taken out first, and there is a bias) has other gradients than those made here; its tables stand for shapes.
"""
from __future__ import annotations

from typing import List, NamedTuple, Optional, Sequence

import torch

from . import ops
from .workloads import HEAD_NAMES, NORM_NAMES, BlockSpec, find_block


class HeadStep(NamedTuple):
    loss: torch.Tensor           # fp32, no dimensions
    row_loss: torch.Tensor       # fp32, one a token
    dx: torch.Tensor             # gradient of x
    dresidual: torch.Tensor      # gradient of the residual (dx itself without dropout)


class LMHead:
    """blocks: the table, whose norm block is taken for an RMS norm.  p, seed: dropout on x before it is added (GPT-2 runs); every step draws from the counter (seed, t), or
    (seed, t + offset_dev) where a captured step reads its counter on the device."""

    def __init__(self, blocks: Sequence[BlockSpec], eps: float = 1e-5, p: float = 0.0, seed: int = 0x5EED):
        self.norm = find_block(blocks, NORM_NAMES, "final norm")
        self.head = find_block(blocks, HEAD_NAMES, "output head")
        n, h = blocks[self.norm], blocks[self.head]
        if n.numel != h.cols:
            raise ValueError(f"block {n.name} has {n.numel} elements, {h.name} {h.cols} columns")
        self.blocks, self.eps, self.p, self.seed = list(blocks), eps, p, seed
        self.tied = h.name != "lm_head"

    def step(self, params: List[torch.Tensor], grads: List[torch.Tensor], x: torch.Tensor, residual: Optional[torch.Tensor],
             targets: torch.Tensor, t: int, row_weight: Optional[torch.Tensor] = None, scale: float = 1.0,
             offset_dev: Optional[torch.Tensor] = None) -> HeadStep:
        """Forward and backward pass of step t (1-based) on a batch of hidden states (any leading dimensions, the type of the table's
        gradients).  Overwrites grads[norm] and grads[head] (micro-batches are added up by the caller, in buffers of their own) and leaves
        no autograd graph; where the head is the embedding, what the embedding's look-up adds to
        that gradient is the caller's to add afterwards.  Parameters of another type (fp32 masters of a bf16 model) are cast first.
        A captured step holds t for ever: with p > 0 give it offset_dev, an int64 tensor of one element that is added to t on the device,
        and set that before every replay; without it all replays have one mask."""
        rng = ops.Rng(self.seed, t, offset_dev)
        weight, gain = params[self.head].detach(), params[self.norm].detach()
        if weight.dtype != x.dtype:
            weight = weight.to(x.dtype)
        n = ops.rms_norm(x, gain, eps=self.eps, residual=residual, p=self.p, rng=rng)
        out = ops.head_loss(n.y, weight, targets, row_weight=row_weight, scale=scale)
        dy, _ = ops.head_backward(n.y, weight, targets, out.lse, row_weight=row_weight, scale=scale, dweight=grads[self.head])
        dx, dres, _ = ops.rms_norm_backward(dy, n.h, gain, n.rstd, p=self.p, rng=rng, dweight=grads[self.norm])
        return HeadStep(out.loss, out.row_loss, dx, dres)
