"""Training a drafter on the target's Top-K records through torch's autograd.

The records are what binding.compress makes of the target's rows.  One call forward (picospec_distill) and one backward
(picospec_distill_grad), which reads the logits again: nothing of the size of the logits is kept between them.  A program that knows its
rows' weights beforehand takes binding.distill(..., weight=..., grad=True), which reads long rows once for both.
"""
from __future__ import annotations

import torch

from . import binding as _ps


def distill_loss(logits: torch.Tensor, rec: "_ps.Compressed", V: int, temperature: float, tail: int = 0):
    """(loss, accept), float32 [rows] each: the divergence of softmax(logits / temperature) from the target's records, differentiable in
    the logits ([rows, >= V], fp32 or bf16), once, and the expected acceptance, which is not."""
    r = _ps._nat.distill_loss(logits, rec.idx, rec.prob, rec.count, rec.k, V, temperature, tail)
    if r.__class__ is int:
        raise _ps.PicoSpecError(r)
    return r
