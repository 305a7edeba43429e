"""Training a drafter on the target's Top-K records through torch's autograd: its embeddings, adjusted logits, the loss, and the clipping of its gradients.

The records are what binding.compress makes of the target's rows.  One call forward (picospec_distill) and one backward
(picospec_distill_grad), which reads the logits again: nothing of the size of the logits is kept between them.  A program that knows its
rows' weights beforehand takes binding.distill(..., weight=..., grad=True), which reads long rows once for both.
embed, adjust and distill_loss are differentiable once, in the table and in the logits; what they are given besides (tokens, histories, masks) must stay as it is until
the backward call, which reads it again.
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


def embed(table: torch.Tensor, tok: torch.Tensor, scale: float = 1.0) -> torch.Tensor:
    """scale * table[tok], [*tok.shape, d], for int32 tokens; zeros for ids outside the table, which have no gradient.  The table's gradient is dense and the same bits every time."""
    r = _ps._nat.embed_on_tape(table, tok, scale)
    if r.__class__ is int:
        raise _ps.PicoSpecError(r)
    return r


def adjust(logits: torch.Tensor, V: int, hist: "_ps.History | None" = None, repetition=1.0, presence=0.0, frequency=0.0, bias: "_ps.Bias | None" = None,
           mask: torch.Tensor | None = None, mask_row: torch.Tensor | None = None, seq_off: torch.Tensor | None = None,
           draft_tok: torch.Tensor | None = None) -> torch.Tensor:
    """binding.adjust, differentiable in the logits (settings and biases may not require a gradient); rows that no sequence has are zeros and have a gradient of 0."""
    h = (hist.tok, hist.length, hist.prompt) if hist is not None else (None, None, None)
    b = (bias.off, bias.id, bias.value) if bias is not None else (None, None, None)
    r = _ps._nat.adjust_on_tape(logits, V, *h, repetition, presence, frequency, *b, mask, mask_row, seq_off, draft_tok)
    if r.__class__ is int:
        raise _ps.PicoSpecError(r)
    return r


def clip_grad_norm(parameters, max_norm: float) -> torch.Tensor:
    """Scales the parameters' gradients in place to a norm of at most max_norm over all of them; returns the norm they had, float32 [1], without waiting for it.  Parameters
    without a gradient are passed over."""
    if isinstance(parameters, torch.Tensor):
        parameters = [parameters]
    return _ps.clip_grad([p.grad for p in parameters if p.grad is not None], max_norm)
