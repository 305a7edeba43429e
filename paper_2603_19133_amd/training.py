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
    def forward(ctx, logits, rec, V, temperature, tail):
        d = _ps.distill(logits, V, temperature, rec, tail)
        ctx.save_for_backward(logits, rec.idx, rec.prob, rec.count, d.stats)
        ctx.rest = rec.k, V, temperature, tail
        ctx.mark_non_differentiable(d.accept)
        ctx.set_materialize_grads(False)
        return d.loss, d.accept

    @staticmethod
    def backward(ctx, g_loss, _g_accept):
        if g_loss is None:
            return None, None, None, None, None
        if torch.is_grad_enabled():              # (create_graph: what the library's kernel does is not on the tape)
            raise RuntimeError("distill_loss is differentiable once")
        logits, idx, prob, count, stats = ctx.saved_tensors
        k, V, temperature, tail = ctx.rest
        grad = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        if logits.shape[1] > V:                  # (columns behind the vocabulary are not read)
            grad[:, V:].zero_()
        if not g_loss.is_contiguous():           # (the gradient of a sum or mean over the rows arrives as one value seen from every row)
            g_loss = g_loss.contiguous()
        # (what the forward call has checked is not checked again: the engine's thread is what small batches wait for)
        dt, ld, rows = _ps._nat.rows2d(logits)
        _ps._check(_ps._nat.distill_grad(logits, dt, ld, rows, V, temperature, idx, prob, count, k, tail, g_loss, stats, grad, logits.shape[1], _ps._stream()))
        return grad, None, None, None, None


def distill_loss(logits: torch.Tensor, rec: "_ps.Compressed", V: int, temperature: float, tail: int = 0):
    """(loss, accept), float32 [rows] each: the divergence of softmax(logits / temperature) from the target's records, differentiable in
    the logits ([rows, >= V], fp32 or bf16), once, and the expected acceptance, which is not."""
    return _DistillLoss.apply(logits, rec, V, temperature, tail)
