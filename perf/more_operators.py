"""The operators in front of and behind a model's rows: adjusted logits, token embeddings with their gradient, clipped gradients.

  adjust       picospec_adjust: penalties for repeated tokens, biases and grammar masks on rows of logits, decoding rows (one a
               sequence) or the rows of a speculative round, where each row sees the drafted tokens in front of it
  adjust_grad  picospec_adjust_grad: the gradient of the same, for a drafter that is trained on adjusted rows
  embed        picospec_embed: rows of an embedding table by token, scaled
  embed_grad   picospec_embed_grad: the table's gradient, a sum over the positions of every token
  clip         picospec_clip_grad: the norm over all gradients of a model, and the gradients scaled to at most that norm

Every case is one pass through the public calls on inputs that are on the GPU.  With `own` false the same outputs come from
elementary torch operations.

Adjusted logits, for a row z of sequence b: a token is seen where it is in the sequence's history or among the drafted tokens in front of the
row, and n is how often it is there behind the prompt.  In turn:
  z <- z / repetition where z > 0, z * repetition elsewhere       (seen tokens)
  z <- z - frequency * n - presence                               (tokens with n > 0)
  z <- z + bias                                                   (the sequence's own list of tokens)
  z <- -inf                                                       (tokens that the row's mask does not allow)
Its gradient: g / repetition or g * repetition for seen tokens, 0 for masked ones, g for the others.

Embedding: out[i] = scale * table[tok[i]], 0 where tok[i] is no token (padding); grad[v] = scale * sum of g[i] over tok[i] = v.

Clipping: norm = sqrt(sum of g^2 over all tensors), g <- g * min(1, max_norm / (norm + 1e-6)).
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}


def _adjust(name, kind, seqs, gamma, V, dtype, hist, bias=0, masks=0, mixed=False, pad=0):
    c = dict(kind=kind, seqs=seqs, gamma=gamma, V=V, dtype=dtype, hist=hist, bias=bias, masks=masks, mixed=mixed, pad=pad)
    return dict(c, name=name) if name else c


def _embed(name, kind, n, V, d, dtype, scale=1.0, padding=0.0):
    c = dict(kind=kind, n=n, V=V, d=d, dtype=dtype, scale=scale, padding=padding)
    return dict(c, name=name) if name else c


def _clip(name, V, d, layers, dtype, quiet=False, odd=False):
    c = dict(kind="clip", V=V, d=d, layers=layers, dtype=dtype, quiet=quiet, odd=odd)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user's next token, a chat of some hundred tokens: bound by launches and latency
        _adjust("adjust_b1", "adjust", 1, 0, 32000, "f32", 512),
        # the target's rows of a ragged round, up to eight drafted tokens: settings per request, biases, grammars for half of the rows, an
        # odd vocabulary in rows off the 16-byte boundary
        _adjust("adjust_b64_odd", "adjust", 64, 8, 50001, "bf16", 4096, bias=300, masks=32, mixed=True, pad=2),
        # the largest: the target's rows of 256 sequences with long histories, up to sixteen drafted tokens each
        _adjust("adjust_b256_long", "adjust", 256, 16, 151936, "bf16", 16384, masks=64, mixed=True),
        # a training batch of a drafter whose rows are adjusted: every position of 32 sequences
        _adjust("adjust_grad_b32", "adjust_grad", 32, 16, 32000, "f32", 2048, masks=16),
        # the same on long rows and histories, without masks
        _adjust("adjust_grad_b128", "adjust_grad", 128, 8, 128256, "bf16", 8192, mixed=True),
        # the drafter's next tokens of a few sequences
        _embed("embed_n8", "embed", 8, 32000, 1024, "bf16"),
        # a training batch or a prefill
        _embed("embed_n16384", "embed", 16384, 128256, 4096, "bf16", scale=64.0, padding=0.1),
        # a small batch, an odd vocabulary and rows that end inside a vector
        _embed("embed_grad_n777_odd", "embed_grad", 777, 50001, 501, "f32", scale=22.4),
        # the largest table, ragged sequences padded to their longest
        _embed("embed_grad_n32768", "embed_grad", 32768, 151936, 4096, "bf16", padding=0.2),
        # the two tables of examples/distill_drafter.py
        _clip("clip_pair", 4096, 24, 0, "f32"),
        # some dozen tensors of odd sizes in one buffer, a norm below the limit: what most steps of a training meet
        _clip("clip_quiet_odd", 50001, 333, 6, "f32", quiet=True, odd=True),
        # the largest: a model of 0.7 billion parameters
        _clip("clip_large", 128256, 2048, 7, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_MOST = 256 * 9 * 151936 * 2          # bytes of the largest rows above


def draw(rng: random.Random):
    kind = rng.choice(["adjust", "adjust", "adjust_grad", "embed", "embed_grad", "embed_grad", "clip", "clip"])
    dtype = rng.choice(["f32", "bf16"])
    V = _log_int(rng, 32000, 152064)
    if rng.random() < 0.5:
        V &= ~7                                             # (most vocabularies are padded to a multiple of 8 or more)
    if kind in ("adjust", "adjust_grad"):
        gamma = rng.choice([0, 4, 8, 16])
        most = _MOST // (V * _BYTES[dtype] * (gamma + 1))
        seqs = min(_log_int(rng, 1, 512), max(1, most))
        return _adjust(None, kind, seqs, gamma, V, dtype, _log_int(rng, 64, 32768), rng.choice([0, 0, _log_int(rng, 1, 300)]),
                       rng.choice([0, 0, rng.randint(1, 64)]), rng.random() < 0.6, 0 if rng.random() < 0.7 else rng.randint(1, 8))
    if kind in ("embed", "embed_grad"):
        d = _log_int(rng, 64, 4096 if dtype == "bf16" else 2048)
        if rng.random() < 0.6:
            d = (d + 63) & ~63
        return _embed(None, kind, _log_int(rng, 1, 32768), V, d, dtype, rng.choice([1.0, round(d ** 0.5, 3)]), rng.choice([0.0, round(rng.uniform(0.0, 0.5), 2)]))
    d = _log_int(rng, 24, 960)
    return _clip(None, V, d, rng.randint(0, 4 if d > 512 else 8), dtype, rng.random() < 0.4, rng.random() < 0.4)


# ---------------------------------------------------------------- inputs

def _gen(seed, what, device):
    g = torch.Generator(device=device)
    g.manual_seed((int(seed) * 16 + what) & 0x7FFFFFFFFFFF)
    return g


def _tokens(shape, V, g):
    """Tokens by a Zipf law, frequent ones at low ids as in most vocabularies."""
    u = torch.rand(shape, device=g.device, generator=g)
    return (torch.exp(u * math.log(V + 1)) - 1).to(torch.int32).clamp_(0, V - 1)


class _State:
    pass


def _gammas(c):
    """Drafted tokens of each sequence: every number up to gamma, the same ones in every batch of the case."""
    return [c["gamma"] - i % c["gamma"] if c["gamma"] else 0 for i in range(c["seqs"])]


def _sizes(c):
    """The tensors of a model with tied tables: the table, four square and three wide matrices, two vectors a layer, a vector behind them."""
    d, wide = c["d"], (8 * c["d"] // 3 + 15) // 16 * 16
    if c["odd"]:
        wide += 7
    layer = [(d, d)] * 4 + [(wide, d)] * 3 + [(d,)] * 2
    return [(c["V"], d)] + layer * c["layers"] + ([(d,)] if c["layers"] else [(d, c["V"])])


def prepare(case, seed):
    c, s, dev = case, _State(), torch.device("cuda")
    s.c, dt = c, _DTYPES[c["dtype"]]
    g = _gen(seed, 3, dev)
    r = random.Random(int(seed) * 7 + 5)
    if c["kind"] in ("adjust", "adjust_grad"):
        B, V = c["seqs"], c["V"]
        gamma = _gammas(c)
        r.shuffle(gamma)
        s.N, s.rows = sum(gamma), sum(gamma) + B
        s.seq_off = torch.tensor([0] + list(np.cumsum(gamma)), dtype=torch.int32, device=dev)
        s.draft_tok = _tokens((s.N,), V, g)
        s.hist_tok = _tokens((B, c["hist"]), V, g)
        length = [r.randint(0, c["hist"]) for _ in range(B)]
        length[0] = c["hist"]
        if B > 2:
            length[1] = 0                                   # (a request that has no token yet)
        s.length = torch.tensor(length, dtype=torch.int32, device=dev)
        s.prompt = torch.tensor([r.randint(0, n) for n in length], dtype=torch.int32, device=dev)
        s.logits = torch.zeros((s.rows, V + c["pad"]), dtype=dt, device=dev)[:, :V]
        s.logits.copy_(torch.randn((s.rows, V), device=dev, generator=g) * 4.0)
        f32 = lambda v: torch.tensor(v, dtype=torch.float32, device=dev)                                       # noqa: E731
        if c["mixed"]:
            s.repetition = f32([r.choice([1.0, r.uniform(1.0, 1.5)]) for _ in range(B)])
            s.presence = f32([r.choice([0.0, r.uniform(-0.5, 1.5)]) for _ in range(B)])
            s.frequency = f32([r.choice([0.0, r.uniform(0.0, 0.5)]) for _ in range(B)])
        else:
            s.repetition, s.presence, s.frequency = float(np.float32(1.2)), 0.5, 0.25
        s.bias = None
        if c["bias"]:
            n = [r.choice([0, r.randint(1, c["bias"])]) for _ in range(B)]
            off = torch.tensor([0] + list(np.cumsum(n)), dtype=torch.int32, device=dev)
            ids = torch.argsort(torch.rand((B, 4 * c["bias"]), device=dev, generator=g), 1).to(torch.int32) * (V // (4 * c["bias"]))
            keep = torch.arange(4 * c["bias"], device=dev).unsqueeze(0) < torch.tensor(n, device=dev).unsqueeze(1)
            ids = ids[keep].contiguous()
            s.bias = (off, ids, torch.randn(ids.shape, device=dev, generator=g) * 5.0)
        s.mask = s.mask_row = None
        if c["masks"]:
            words = (V + 31) // 32
            share = torch.rand((c["masks"], 1), device=dev, generator=g)
            bits = torch.rand((c["masks"], words * 32), device=dev, generator=g) < share * share
            bits[0] = False                                 # (a grammar that allows nothing)
            packed = (bits.view(c["masks"], words, 32).to(torch.int64) << torch.arange(32, device=dev)).sum(2)
            s.mask = torch.where(packed >= 2 ** 31, packed - 2 ** 32, packed).to(torch.int32)
            s.mask_row = torch.tensor([r.choice([-1, r.randrange(c["masks"])]) for _ in range(s.rows)], dtype=torch.int32, device=dev)
        if c["kind"] == "adjust_grad":
            s.grad = (torch.randn((s.rows, V), device=dev, generator=g) * 1e-3).to(dt)
    elif c["kind"] in ("embed", "embed_grad"):
        s.scale = float(np.float32(c["scale"]))
        s.tok = _tokens((c["n"],), c["V"], g)
        s.tok[torch.rand(c["n"], device=dev, generator=g) < c["padding"]] = -1
        if c["kind"] == "embed":
            s.table = torch.randn((c["V"], c["d"]), device=dev, generator=g).to(dt)
        else:
            s.grad = (torch.randn((c["n"], c["d"]), device=dev, generator=g) * 1e-2).to(dt)
    else:
        shapes = _sizes(c)
        numel = [math.prod(x) for x in shapes]
        # tensors of one buffer behind each other, as those of a bucket are
        s.flat = torch.empty(sum(numel), dtype=dt, device=dev)
        s.out_flat = s.flat if c["quiet"] else torch.empty_like(s.flat)
        s.grads = [t.view(x) for t, x in zip(s.flat.split(numel), shapes)]
        s.outs = [t.view(x) for t, x in zip(s.out_flat.split(numel), shapes)]
        for i, t in enumerate(s.grads):
            t.copy_(torch.randn(t.shape, device=dev, generator=g) * 10.0 ** r.uniform(-4.0, -2.0))
        s.max_norm = 1e4 if c["quiet"] else 1.0
        s.grads[0].view(-1)[0] = 2.0                        # (a norm above 1, whatever the sizes)
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    if own:
        return _run_own(s)
    return {"adjust": _plain_adjust, "adjust_grad": _plain_adjust, "embed": _plain_embed, "embed_grad": _plain_embed_grad, "clip": _plain_clip}[s.c["kind"]](s)


def _run_own(s):
    from paper_2603_19133_amd import binding as ps
    c = s.c
    if c["kind"] in ("adjust", "adjust_grad"):
        hist = ps.History(s.hist_tok, s.length, s.prompt)
        drafts = dict(seq_off=s.seq_off, draft_tok=s.draft_tok) if c["gamma"] else {}
        if c["kind"] == "adjust":
            bias = ps.Bias(*s.bias) if s.bias else None
            return {"logits": ps.adjust(s.logits, c["V"], hist, repetition=s.repetition, presence=s.presence, frequency=s.frequency, bias=bias,
                                        mask=s.mask, mask_row=s.mask_row, **drafts)}
        return {"grad": ps.adjust_grad(s.grad, s.logits, c["V"], hist, repetition=s.repetition, mask=s.mask, mask_row=s.mask_row, **drafts)}
    if c["kind"] == "embed":
        return {"rows": ps.embed(s.table, s.tok, scale=s.scale)}
    if c["kind"] == "embed_grad":
        return {"grad": ps.embed_grad(s.grad, s.tok, c["V"], scale=s.scale)}
    norm = ps.clip_grad(s.grads, s.max_norm, out=None if c["quiet"] else s.outs)
    return {"norm": norm, "grads": s.out_flat}


def _plain_adjust(s):
    c, dev = s.c, s.logits.device
    B, V, rows = c["seqs"], c["V"], s.rows
    # every token of the histories counted, per sequence (a column behind the vocabulary takes what does not count), then the drafted ones per row
    at = torch.arange(s.hist_tok.shape[1], device=dev).unsqueeze(0)
    inside, made = at < s.length.unsqueeze(1), at >= s.prompt.unsqueeze(1)
    ones = torch.ones_like(s.hist_tok)
    seen = torch.zeros((B, V + 1), dtype=torch.int32, device=dev).scatter_add_(1, torch.where(inside, s.hist_tok, V).long(), ones)
    made = torch.zeros((B, V + 1), dtype=torch.int32, device=dev).scatter_add_(1, torch.where(inside & made, s.hist_tok, V).long(), ones)
    first = s.seq_off[:-1].long() + torch.arange(B, device=dev)
    row = torch.arange(rows, device=dev)
    seq = torch.searchsorted(first, row, right=True) - 1
    seen, made = seen[seq], made[seq]
    if c["gamma"]:
        j = torch.arange(c["gamma"], device=dev).unsqueeze(0)
        there = j < (row - first[seq]).unsqueeze(1)
        tok = torch.where(there, s.draft_tok[torch.where(there, s.seq_off[seq].long().unsqueeze(1) + j, 0)], V).long()
        seen.scatter_add_(1, tok, torch.ones_like(tok, dtype=torch.int32))
        made.scatter_add_(1, tok, torch.ones_like(tok, dtype=torch.int32))
    seen, made = seen[:, :V], made[:, :V]
    per_row = lambda v: v[seq].unsqueeze(1) if isinstance(v, torch.Tensor) else v                               # noqa: E731
    z, rep = s.logits.float(), per_row(s.repetition)
    if s.mask is not None:
        bits = (s.mask.unsqueeze(2) >> torch.arange(32, dtype=torch.int32, device=dev)) & 1
        allowed = bits.view(s.mask.shape[0], -1)[:, :V] == 1
        allowed = allowed[s.mask_row.clamp(min=0).long()] | (s.mask_row < 0).unsqueeze(1)
    if c["kind"] == "adjust_grad":
        d = s.grad.float()
        d = torch.where(seen > 0, torch.where(z > 0, d / rep, d * rep), d)
        return {"grad": (d if s.mask is None else torch.where(allowed, d, 0.0)).to(s.grad.dtype)}
    z = torch.where(seen > 0, torch.where(z > 0, z / rep, z * rep), z)
    z = z - per_row(s.frequency) * made - torch.where(made > 0, per_row(s.presence), 0.0)
    if s.bias is not None:
        off, ids, value = s.bias
        of = torch.searchsorted(off[1:].contiguous(), torch.arange(ids.shape[0], dtype=torch.int32, device=dev), right=True)
        dense = torch.zeros((B, V), device=dev)
        dense[of, ids.long()] = value
        z = z + dense[seq]
    if s.mask is not None:
        z = torch.where(allowed, z, -math.inf)
    return {"logits": z.to(s.logits.dtype)}


def _plain_embed(s):
    there = (s.tok >= 0).unsqueeze(1)
    rows = s.table[s.tok.clamp(min=0).long()].float() * s.scale
    return {"rows": torch.where(there, rows, 0.0).to(s.table.dtype)}


def _plain_embed_grad(s):
    c = s.c
    total = torch.zeros((c["V"] + 1, c["d"]), device=s.grad.device)          # (a row behind the table takes the padding's)
    total.index_add_(0, torch.where(s.tok >= 0, s.tok, c["V"]).long(), s.grad.float())
    return {"grad": (total[:c["V"]] * s.scale).to(s.grad.dtype)}


def _plain_clip(s):
    norm = torch.stack([g.float().square().sum() for g in s.grads]).sum().sqrt().reshape(1)
    factor = torch.clamp(s.max_norm / (norm + 1e-6), max=1.0)
    [o.copy_(g.float() * factor) for g, o in zip(s.grads, s.outs)]
    return {"norm": norm, "grads": s.out_flat}


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"adjust": _exact_adjust, "adjust_grad": _exact_adjust, "embed": _exact_embed, "embed_grad": _exact_embed_grad, "clip": _exact_clip}[case["kind"]](s)


def _exact_adjust(s):
    c, V, dev = s.c, s.c["V"], s.logits.device
    off, length, prompt = s.seq_off.tolist(), s.length.tolist(), s.prompt.tolist()
    of = lambda v, b: float(v[b]) if isinstance(v, torch.Tensor) else float(np.float32(v))                       # noqa: E731
    rep, pres, freq = ([of(v, b) for b in range(c["seqs"])] for v in (s.repetition, s.presence, s.frequency))
    which = s.mask_row.tolist() if s.mask is not None else [-1] * s.rows
    lists = [x.tolist() for x in s.bias] if s.bias is not None else None
    words = s.mask.cpu().numpy().view(np.uint32) if s.mask is not None else None
    out = torch.empty((s.rows, V), dtype=torch.float64, device=dev)
    for b in range(c["seqs"]):
        for t in range(off[b + 1] - off[b] + 1):
            row = off[b] + b + t
            drafted = s.draft_tok[off[b]:off[b] + t]
            met = torch.zeros(V, dtype=torch.bool, device=dev)
            met[s.hist_tok[b, :length[b]].long()] = True
            met[drafted.long()] = True
            n = torch.bincount(torch.cat([s.hist_tok[b, prompt[b]:length[b]], drafted]), minlength=V).double()
            z = s.logits[row].double()
            if c["kind"] == "adjust_grad":
                out[row] = s.grad[row].double() * torch.where(met, torch.where(z > 0, 1.0 / rep[b], rep[b]), 1.0)
            else:
                z = torch.where(met, torch.where(z > 0, z / rep[b], z * rep[b]), z) - freq[b] * n - pres[b] * (n > 0)
                if lists is not None and lists[0][b + 1] > lists[0][b]:
                    e = slice(lists[0][b], lists[0][b + 1])
                    z[torch.tensor(lists[1][e], device=dev)] += torch.tensor(lists[2][e], dtype=torch.float64, device=dev)
                out[row] = z
            if which[row] >= 0:
                allowed = torch.from_numpy(np.unpackbits(words[which[row]].view(np.uint8), bitorder="little")[:V].astype(bool)).to(dev)
                out[row][~allowed] = 0.0 if c["kind"] == "adjust_grad" else -math.inf
    return {"grad" if c["kind"] == "adjust_grad" else "logits": out}


def _exact_embed(s):
    out = torch.zeros((s.c["n"], s.c["d"]), dtype=torch.float64, device=s.table.device)
    there = torch.nonzero(s.tok >= 0)[:, 0]
    out[there] = s.table.index_select(0, s.tok[there]).double() * s.scale
    return {"rows": out}


def _exact_embed_grad(s):
    # positions in the order of their tokens; a token's sum is what the running sum gains over them
    c, dev = s.c, s.grad.device
    out = torch.zeros((c["V"], c["d"]), dtype=torch.float64, device=dev)
    order = torch.argsort(s.tok, stable=True)
    order = order[s.tok[order] >= 0]
    if order.numel():
        ids, n = torch.unique_consecutive(s.tok[order], return_counts=True)
        end = torch.cumsum(n, 0) - 1
        running = torch.cumsum(s.grad[order].double(), 0)[end]
        out[ids.long()] = torch.diff(running, dim=0, prepend=torch.zeros_like(running[:1])) * s.scale
    return {"grad": out}


def _exact_clip(s):
    norm = math.sqrt(math.fsum(float((g.double() ** 2).sum()) for g in s.grads))
    return {"norm": torch.tensor([norm], dtype=torch.float64), "grads": s.flat.double() * min(1.0, s.max_norm / (norm + 1e-6))}


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    c = case
    esz = _BYTES[c["dtype"]]
    if c["kind"] in ("adjust", "adjust_grad"):
        # the rows in and out, half of the histories' capacity, the masks; a product per element
        rows = c["seqs"] + sum(_gammas(c))
        return {"bytes": 2 * rows * c["V"] * esz + 2 * c["seqs"] * c["hist"] + c["masks"] * (c["V"] + 7) // 8, "flops": rows * c["V"]}
    if c["kind"] == "embed":
        used = c["n"] * (1 - c["padding"])
        return {"bytes": (used + c["n"]) * c["d"] * esz + 4 * c["n"], "flops": used * c["d"]}
    if c["kind"] == "embed_grad":
        used = c["n"] * (1 - c["padding"])
        return {"bytes": (used + c["V"]) * c["d"] * esz + 4 * c["n"], "flops": used * c["d"]}
    n = sum(math.prod(x) for x in _sizes(c))
    return {"bytes": n * esz * (1 if c["quiet"] else 2), "flops": n * (2 if c["quiet"] else 3)}
