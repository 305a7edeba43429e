"""Training a drafter on the target's Top-K records through torch's autograd.

The records are what binding.compress makes of the target's rows.  One call forward (picospec_distill) and one backward
(picospec_distill_grad), which reads the logits again: nothing of the size of the logits is kept between them.  A program that knows its
rows' weights beforehand takes binding.distill(..., weight=..., grad=True), which reads long rows once for both.
"""
from __future__ import annotations

import torch

from . import binding as _ps


class _DistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, idx, prob, count, mass, lse, k, V, temperature, tail):
        rec = _ps.Compressed(idx, prob, count, mass, lse, k)
        d = _ps.distill(logits, V, temperature, rec, tail)
        ctx.save_for_backward(logits, idx, prob, count, d.stats)
        ctx.rest = k, V, temperature, tail
        ctx.mark_non_differentiable(d.accept)
        ctx.set_materialize_grads(False)
        return d.loss, d.accept

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g_loss, _g_accept):
        if g_loss is None:
            return (None,) * 10
        logits, idx, prob, count, stats = ctx.saved_tensors
        k, V, temperature, tail = ctx.rest
        grad = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        if logits.shape[1] > V:                  # (columns behind the vocabulary are not read)
            grad[:, V:].zero_()
        # (the gradient of a sum or mean over the rows arrives as one value seen from every row)
        _ps.distill_grad(logits, V, temperature, _ps.Compressed(idx, prob, count, None, None, k), stats, tail, g_loss.contiguous(), out=grad)
        return grad, None, None, None, None, None, None, None, None, None


def distill_loss(logits: torch.Tensor, rec: "_ps.Compressed", V: int, temperature: float, tail: int = 0):
    """(loss, accept), float32 [rows] each: the divergence of softmax(logits / temperature) from the target's records, differentiable in
    the logits ([rows, >= V], fp32 or bf16), and the expected acceptance, which is not."""
    return _DistillLoss.apply(logits, rec.idx, rec.prob, rec.count, rec.mass, rec.lse, rec.k, V, temperature, tail)
