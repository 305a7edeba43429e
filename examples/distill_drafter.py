"""Trains a small drafter on a target's Top-K records and measures what the speculative round gains.

The calls as a program uses them, in turn:

  binding.sample       rolls out tokens from the target (temperature, top-p) and drafts from the drafter
  binding.compress     Top-K records of the target's rows: all that a trainer keeps of the target
  training.distill_loss  the drafter's divergence from the records and the expected acceptance, through torch's autograd
  binding.round        compress, verification and draw of a speculative round, before and after the training

Both models are a table of bigram logits of low rank (no downloads): the target's is fixed, the drafter starts at random.

    python examples/distill_drafter.py [--steps 150]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2603_19133_amd import binding as ps  # noqa: E402
from paper_2603_19133_amd.training import distill_loss  # noqa: E402

V, T, K, GAMMA = 4096, 0.8, 64, 4


class Bigram(torch.nn.Module):
    def __init__(self, rank: int, scale: float, generator: torch.Generator):
        super().__init__()
        self.emb = torch.nn.Parameter(torch.randn(V, rank, generator=generator, device="cuda"))
        self.out = torch.nn.Parameter(torch.randn(rank, V, generator=generator, device="cuda") * scale / rank ** 0.5)

    def forward(self, tok: torch.Tensor) -> torch.Tensor:
        return self.emb[tok.long()] @ self.out


@torch.no_grad()
def accepted(target: Bigram, drafter: Bigram, start: torch.Tensor, g: torch.Generator) -> float:
    """Mean number of accepted tokens, of GAMMA drafted, over the sequences that `start` begins."""
    B = start.numel()
    inputs, drafted = [start], []
    for _ in range(GAMMA):                       # the drafter draws from its records, which the round compresses again from the same rows
        q = ps.compress(drafter(inputs[-1]).contiguous(), V, T, V)
        tok, _ = ps.sample_draft(q, torch.rand(B, generator=g, device="cuda"))
        drafted.append(tok)
        inputs.append(tok)
    seen = torch.stack(inputs, 1)                # [B, GAMMA + 1]: what each position has in front of it
    seq_off = torch.arange(B + 1, dtype=torch.int32, device="cuda") * GAMMA
    uniforms = torch.rand(B * (GAMMA + 1), generator=g, device="cuda")
    _, ver, _ = ps.round(drafter(seen[:, :GAMMA].reshape(-1)).contiguous(), target(seen.reshape(-1)).contiguous(), V, T, seq_off, B * GAMMA,
                         torch.stack(drafted, 1).reshape(-1).contiguous(), V, uniforms)
    return ver.n_accept.float().mean().item()


def main(steps: int = 150, batch: int = 512, seed: int = 0, verbose: bool = True) -> dict:
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    target, drafter = Bigram(24, 2.5, g), Bigram(24, 0.1, g)
    target.requires_grad_(False)
    opt = torch.optim.Adam(drafter.parameters(), lr=0.03)
    start = torch.randint(0, V, (256,), generator=g, device="cuda", dtype=torch.int32)
    before = accepted(target, drafter, start, g)
    tok = torch.randint(0, V, (batch,), generator=g, device="cuda", dtype=torch.int32)
    first = last = None
    for step in range(steps):
        logits = target(tok)
        rec = ps.compress(logits, V, T, K)                                       # (what the target sends: 8 bytes an entry)
        loss, accept = distill_loss(drafter(tok), rec, V, T, tail=1)
        opt.zero_grad(set_to_none=True)
        loss.mean().backward()
        opt.step()
        last = loss.mean().item(), accept.mean().item()
        first = first or last
        if verbose and (step % 25 == 0 or step == steps - 1):
            print(f"step {step:4d}  loss {last[0]:.4f}  expected acceptance {last[1]:.4f}", flush=True)
        # the next tokens of the roll-out, a nucleus draw from the target
        tok = ps.sample(logits, V, torch.rand(batch, generator=g, device="cuda"), temperature=T, top_p=0.95).tok
    after = accepted(target, drafter, start, g)
    if verbose:
        print(f"accepted of {GAMMA} drafted tokens: {before:.2f} before, {after:.2f} after")
    return {"loss": (first[0], last[0]), "expected": (first[1], last[1]), "accepted": (before, after)}


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=150)
    main(ap.parse_args().steps)
