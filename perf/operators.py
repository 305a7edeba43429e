"""The drafter's operators beside the round: drawing tokens with the usual filters, and training on the target's records.

  sample    picospec_sample: one token per row with temperature, top-k, top-p and min-p from given uniforms (the seed token of a
            request, decoding without a draft, a drafter that keeps no record)
  loss      picospec_distill: Kullback-Leibler divergence of a drafter's distribution from the target's Top-K record, forward
            only (evaluation), with the expected acceptance
  step      picospec_distill with its gradient in the same call: a training step that knows its rows' weights beforehand
  autograd  the same loss through torch's autograd: picospec_distill forward, picospec_distill_grad backward

Every case is one pass through the public calls on inputs that are on the GPU.  With `own` false the same outputs come from
elementary torch operations.

The sampler, for one row of logits z, temperature T (0: the largest logit, lowest id first), top_k, top_p, min_p and a uniform u
(NaN counts as -inf, +inf as the largest finite number): w = exp((z - max z) / T); the row is ordered by logit descending, id
ascending; the first top_k are kept; of these the shortest prefix whose weight reaches top_p of theirs; of these the ones with w >=
min_p; the token is the first id, ascending, at which the kept weight up to and with it exceeds u times all of it.

The loss, for one row of student logits z and a record (id_j, p_j), j < count, q = softmax(z / T):
  tail = 0   sum_j ph_j (ln ph_j - ln q_j), ph = p / sum p
  tail = 1   sum_j p_j (ln p_j - ln q_j) + pt (ln pt - ln qt), pt = max(0, 1 - sum p) and qt = the student's mass off the record
and accept = sum_j min(p_j, q_j).  Rows with count = 0 have loss, accept and gradient 0.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_CHUNK = 1 << 26          # elements handled at a time


def _sample(name, rows, V, dtype, recipe, T=1.0, top_k=0, top_p=0.0, min_p=0.0, pad=0, mixed=False, masked=False):
    c = dict(kind="sample", rows=rows, V=V, dtype=dtype, recipe=recipe, T=T, top_k=top_k, top_p=top_p, min_p=min_p, pad=pad, mixed=mixed, masked=masked)
    return dict(c, name=name) if name else c


def _distill(name, kind, rows, V, dtype, recipe, k, tail, T=1.0, pad=0, ragged=False):
    c = dict(kind=kind, rows=rows, V=V, dtype=dtype, recipe=recipe, k=k, tail=tail, T=T, pad=pad, ragged=ragged)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user's token with the filters most programs set: bound by launches and latency
        _sample("sample_b1", 1, 32000, "f32", "normal3", T=0.8, top_k=50, top_p=0.95),
        # a serving batch in which every request brings its own settings, greedy ones among them
        _sample("sample_b64_mixed", 64, 128256, "bf16", "zipf1.1", mixed=True),
        # a batch of roll-outs: plain draws from the whole distribution
        _sample("sample_b256_plain", 256, 151936, "f32", "normal3"),
        # the largest batch, nucleus draws from flat rows (kept sets of some ten thousand tokens)
        _sample("sample_b512_topp", 512, 152064, "bf16", "zipf1.2", top_p=0.95),
        # an odd vocabulary in rows off the 16-byte boundary, masked ids, a row that is masked whole
        _sample("sample_b300_odd", 300, 50001, "bf16", "mix4", T=0.9, min_p=0.05, pad=2, masked=True),
        # a held-out handful of positions
        _distill("loss_b8", "loss", 8, 32000, "bf16", "mix4", 64, 0),
        # evaluation of a drafter on long records, with the tail
        _distill("loss_b1088_tail", "loss", 1088, 152064, "bf16", "zipf1.2", 2048, 1),
        # a small training batch through autograd
        _distill("autograd_b512", "autograd", 512, 32000, "bf16", "mix4", 256, 0),
        # ragged records (positions that are not trained on have none), odd vocabulary, fp32
        _distill("autograd_b333_odd", "autograd", 333, 50001, "f32", "normal3", 777, 1, T=0.9, pad=3, ragged=True),
        # fp32 logits and the tail in one call
        _distill("step_b2048_tail", "step", 2048, 128256, "f32", "zipf1.1", 1024, 1, T=0.7),
        # the largest: a training batch of 4096 positions
        _distill("step_b4096", "step", 4096, 151936, "bf16", "mix4", 64, 0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_MOST_SAMPLE = 512 * 152064 * 2
_MOST_DISTILL = 4096 * 151936 * 2


def draw(rng: random.Random):
    kind = rng.choice(["sample", "sample", "sample", "loss", "step", "autograd"])
    dtype = rng.choice(["f32", "bf16"])
    esz = 4 if dtype == "f32" else 2
    V = _log_int(rng, 32000, 152064)
    if rng.random() < 0.5:
        V &= ~7                                             # (most vocabularies are padded to a multiple of 8 or more)
    pad = 0 if rng.random() < 0.7 else rng.randint(1, 8)
    recipe = rng.choice(["normal3", "mix4", "resample5", "zipf1.1", "zipf1.2"])
    T = round(rng.uniform(0.6, 1.2), 2)
    if kind == "sample":
        rows = min(_log_int(rng, 1, 512), _MOST_SAMPLE // ((V + pad) * esz))
        if rng.random() < 0.3:
            return _sample(None, rows, V, dtype, recipe, pad=pad, mixed=True, masked=rng.random() < 0.3)
        top_k = rng.choice([0, 0, _log_int(rng, 1, 1024)])
        top_p = rng.choice([0.0, 0.9, round(rng.uniform(0.5, 0.99), 3)])
        min_p = rng.choice([0.0, 0.0, round(rng.uniform(0.01, 0.2), 3)])
        return _sample(None, rows, V, dtype, recipe, T, top_k, top_p, min_p, pad, masked=rng.random() < 0.2)
    rows = min(_log_int(rng, 8, 4096), _MOST_DISTILL // ((V + pad) * esz))
    k = _log_int(rng, 10, 4096)
    return _distill(None, kind, rows, V, dtype, recipe, k, rng.choice([0, 1]), T, pad, ragged=rng.random() < 0.3)


# ---------------------------------------------------------------- inputs

def _gen(seed, what, device):
    g = torch.Generator(device=device)
    g.manual_seed((int(seed) * 16 + what) & 0x7FFFFFFFFFFF)
    return g


def _logits(recipe, n, V, g):
    """[n, V] fp32 logits: independent normal ones, or those of a Zipf law over a shuffled vocabulary with jitter."""
    z = torch.randn((n, V), device=g.device, generator=g)
    if recipe.startswith("zipf"):
        rank = torch.floor(torch.rand((n, V), device=g.device, generator=g) * V) + 1.0
        return z * 0.5 - float(recipe[4:]) * torch.log(rank)
    return z * {"normal3": 3.0, "mix4": 4.0, "resample5": 5.0}[recipe]


class _State:
    pass


def prepare(case, seed):
    c, s, dev = case, _State(), torch.device("cuda")
    s.c, rows, V, dt = c, c["rows"], c["V"], _DTYPES[c["dtype"]]
    g = _gen(seed, 1, dev)
    s.logits = torch.zeros((rows, V + c["pad"]), dtype=dt, device=dev)[:, :V]
    step = max(1, _CHUNK // V)
    if c["kind"] == "sample":
        for r0 in range(0, rows, step):
            n = min(step, rows - r0)
            z = _logits(c["recipe"], n, V, g)
            if c["masked"]:                                 # (a grammar that allows one id in eight; the type's lowest value and -inf in turn)
                low = torch.where((torch.arange(r0, r0 + n, device=dev) % 2 == 0).unsqueeze(1), -math.inf, torch.finfo(dt).min)
                z = torch.where(torch.rand(z.shape, device=dev, generator=g) < 0.875, low, z)
            s.logits[r0:r0 + n] = z.to(dt)
        if c["masked"] and rows > 5:
            s.logits[5] = -math.inf                         # (a request whose grammar allows nothing)
        s.u = torch.rand(rows, device=dev, generator=g)
        if c["mixed"]:
            r = random.Random(int(seed) * 7 + 3)
            pick = lambda *of: [r.choice(of)() for _ in range(rows)]                                     # noqa: E731
            f = lambda lo, hi: (lambda: r.uniform(lo, hi))                                               # noqa: E731
            zero = lambda: 0                                                                             # noqa: E731
            t = lambda v, d: torch.tensor(v, dtype=d, device=dev)                                        # noqa: E731
            s.T = t(pick(f(0.6, 1.2), f(0.6, 1.2), f(0.6, 1.2), zero), torch.float32)
            s.top_k = t(pick(zero, lambda: r.randint(1, 100), lambda: 50, lambda: r.randint(100, 1000)), torch.int32)
            s.top_p = t(pick(zero, f(0.8, 0.98), lambda: 0.9), torch.float32)
            s.min_p = t(pick(zero, zero, f(0.02, 0.1)), torch.float32)
        else:
            s.T, s.top_k, s.top_p, s.min_p = c["T"], c["top_k"], c["top_p"], c["min_p"]
        return s
    s.T = float(np.float32(c["T"]))                         # (the type in which it reaches the library)
    k = min(c["k"], V)
    s.idx = torch.empty((rows, k), dtype=torch.int32, device=dev)
    s.prob = torch.empty((rows, k), dtype=torch.float32, device=dev)
    for r0 in range(0, rows, step):
        n = min(step, rows - r0)
        t = _logits(c["recipe"], n, V, g)
        s.logits[r0:r0 + n] = (0.9 * t + 1.2 * torch.randn(t.shape, device=dev, generator=g)).to(dt)
        v, i = torch.sort(t, dim=1, descending=True, stable=True)
        lse = torch.logsumexp(t.double() / s.T, 1, keepdim=True)
        s.idx[r0:r0 + n] = i[:, :k].to(torch.int32)
        s.prob[r0:r0 + n] = torch.exp(v[:, :k].double() / s.T - lse).float()
    s.count = torch.full((rows,), k, dtype=torch.int32, device=dev)
    if c["ragged"]:
        s.count = torch.randint(0, k + 1, (rows,), device=dev, generator=g).to(torch.int32)
        s.count[torch.rand(rows, device=dev, generator=g) < 0.2] = 0
        unused = torch.arange(k, device=dev).unsqueeze(0) >= s.count.unsqueeze(1)
        s.idx[unused] = -1
        s.prob[unused] = 0.0
    s.mass = s.prob.double().sum(1).float()
    s.weight = torch.rand(rows, device=dev, generator=g) + 0.5
    if own:
        from paper_2603_19133_amd import binding as ps
        s.rec = ps.Compressed(s.idx, s.prob, s.count, s.mass, torch.zeros_like(s.mass), k)
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    if own:
        return _run_own(s)
    c = s.c
    if c["kind"] == "sample":
        return _plain_sample(s)
    return _plain_distill(s)


def _run_own(s):
    from paper_2603_19133_amd import binding as ps
    c = s.c
    if c["kind"] == "sample":
        r = ps.sample(s.logits, c["V"], s.u, temperature=s.T, top_k=s.top_k, top_p=s.top_p, min_p=s.min_p)
        return {"tok": r.tok, "prob": r.prob, "count": r.count, "lse": r.lse}
    if c["kind"] == "loss":
        d = ps.distill(s.logits, c["V"], s.T, s.rec, tail=c["tail"])
        return {"loss": d.loss, "accept": d.accept}
    if c["kind"] == "step":
        d = ps.distill(s.logits, c["V"], s.T, s.rec, tail=c["tail"], weight=s.weight, grad=True)
        return {"loss": d.loss, "accept": d.accept, "grad": d.grad}
    from paper_2603_19133_amd.training import distill_loss
    z = s.logits.detach().requires_grad_()
    loss, accept = distill_loss(z, s.rec, c["V"], s.T, tail=c["tail"])
    loss.backward(s.weight)
    return {"loss": loss.detach(), "accept": accept, "grad": z.grad}


def _per_row(v, rows, dtype, dev):
    """A setting as a column in 64 bits; one for all rows goes through the type in which it reaches the library."""
    if not isinstance(v, torch.Tensor):
        v = torch.full((rows,), v, dtype=dtype, device=dev)
    return v.to(torch.float64 if dtype == torch.float32 else torch.int64).unsqueeze(1)


def _plain_sample(s):
    rows, V = s.logits.shape
    dev = s.logits.device
    T, k = _per_row(s.T, rows, torch.float32, dev), _per_row(s.top_k, rows, torch.int32, dev)
    top_p, min_p = _per_row(s.top_p, rows, torch.float32, dev), _per_row(s.min_p, rows, torch.float32, dev)
    greedy = T == 0
    k = torch.where(greedy, 1, k)
    T = torch.where(greedy, 1.0, T)
    out = {n: torch.empty(rows, dtype=d, device=dev) for n, d in (("tok", torch.int32), ("prob", torch.float32), ("count", torch.int32), ("lse", torch.float32))}
    at = torch.arange(V, device=dev).unsqueeze(0)
    step = max(1, _CHUNK // V)
    for r0 in range(0, rows, step):
        r = slice(r0, min(rows, r0 + step))
        # (64 bits: the ends of the kept prefix and of the draw are comparisons of sums over the whole vocabulary)
        z = torch.nan_to_num(s.logits[r].double(), nan=-math.inf, posinf=torch.finfo(torch.float32).max, neginf=-math.inf)
        v, i = torch.sort(z, dim=1, descending=True, stable=True)
        some = v[:, :1] > -math.inf
        top = torch.where(some, v[:, :1], 0.0)
        w = torch.exp((v - top) / T[r])
        keep = (v > -math.inf) & ((k[r] <= 0) | (at < k[r]))
        wk = torch.where(keep, w, 0.0)
        before = torch.cumsum(wk, 1)
        total = before[:, -1:].clone()
        before = torch.cat([torch.zeros_like(total), before[:, :-1]], 1)
        keep &= (top_p[r] <= 0) | (top_p[r] >= 1) | (before < top_p[r] * total)
        keep &= (min_p[r] <= 0) | (w >= min_p[r])
        byid = torch.zeros_like(w).scatter_(1, i, torch.where(keep, w, 0.0))
        upto = torch.cumsum(byid, 1)
        total = upto[:, -1:]
        tok = (upto <= s.u[r].double().unsqueeze(1) * total).sum(1).clamp(max=V - 1)
        some = some[:, 0]
        out["tok"][r] = torch.where(some, tok, -1).to(torch.int32)
        out["prob"][r] = torch.where(some, byid.gather(1, tok.unsqueeze(1))[:, 0] / total[:, 0], 0.0).float()
        out["count"][r] = keep.sum(1).to(torch.int32)
        out["lse"][r] = torch.where(some, top[:, 0] / T[r][:, 0] + torch.log(total[:, 0]), -math.inf).float()
    return out


def _plain_distill(s):
    c, rows, V = s.c, *s.logits.shape
    dev, T, kk = s.logits.device, s.T, s.idx.shape[1]
    out = {"loss": torch.empty(rows, device=dev), "accept": torch.empty(rows, device=dev)}
    if c["kind"] != "loss":
        out["grad"] = torch.empty((rows, V), dtype=s.logits.dtype, device=dev)
    step = max(1, _CHUNK // V)
    for r0 in range(0, rows, step):
        r = slice(r0, min(rows, r0 + step))
        used = torch.arange(kk, device=dev).unsqueeze(0) < s.count[r].unsqueeze(1)
        idx = torch.where(used, s.idx[r], 0).long()
        p = torch.where(used, s.prob[r], 0.0)
        y = s.logits[r].float() / T
        top = y.max(1, keepdim=True).values
        e = torch.exp(y - top)
        total = e.sum(1, keepdim=True)
        lnq = y.gather(1, idx) - top - torch.log(total)
        q = torch.exp(lnq)
        mass = p.double().sum(1, keepdim=True)              # (64 bits: what is left of 1)
        some = (s.count[r] > 0).unsqueeze(1)
        row = torch.arange(e.shape[0], device=dev).unsqueeze(1).expand_as(idx)
        if c["tail"]:
            pt = (1.0 - mass).clamp(min=0.0).float()
            off = e.clone()
            off[row[used], idx[used]] = 0.0
            qt = off.sum(1, keepdim=True) / total
            ph, whole = p, mass.float() + pt
            extra = torch.where(pt > 0, pt * (torch.log(pt) - torch.log(qt)), 0.0)
            b = whole - torch.where(pt > 0, pt / qt, 0.0)
        else:
            ph = p / torch.where(mass > 0, mass, 1.0).float()
            extra, whole = torch.zeros_like(total), torch.ones_like(total)
            b = whole
        terms = torch.where(ph > 0, ph * (torch.log(ph) - lnq), 0.0)
        out["loss"][r] = torch.where(some, terms.sum(1, keepdim=True) + extra, 0.0)[:, 0]
        out["accept"][r] = torch.where(used, torch.minimum(p, q), 0.0).sum(1)
        if c["kind"] != "loss":
            scale = torch.where(some, s.weight[r].unsqueeze(1) / T, 0.0)
            grad = e.mul_(scale * b / total)
            grad[row[used], idx[used]] = (scale * (whole * q - ph))[used]
            out["grad"][r] = grad.to(s.logits.dtype)
    return out


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return _exact_sample(s) if case["kind"] == "sample" else _exact_distill(s)


def _exact_sample(s):
    rows, V = s.logits.shape
    col = lambda v, d: np.asarray(v.cpu().numpy() if isinstance(v, torch.Tensor) else np.full(rows, v), dtype=d)          # noqa: E731
    T, top_k = col(s.T, np.float32), col(s.top_k, np.int64)
    top_p, min_p, u = col(s.top_p, np.float32), col(s.min_p, np.float32), s.u.cpu().numpy()
    tok, count = np.full(rows, -1, np.int32), np.zeros(rows, np.int32)
    prob, lse = np.zeros(rows), np.full(rows, -np.inf)
    for r in range(rows):
        z = s.logits[r].double().cpu().numpy()
        z[np.isnan(z)] = -np.inf
        z = np.minimum(z, float(np.finfo(np.float32).max))
        best = z.max()
        if best == -np.inf:
            continue
        if T[r] == 0:
            ids = np.array([int(z.argmax())])
            temp = 1.0
        else:
            ids, temp = np.flatnonzero(z > -np.inf), float(T[r])
        if top_k[r] > 0 and top_k[r] < ids.size:            # (the k-th value; of those equal to it the lowest ids)
            edge = np.partition(z[ids], ids.size - top_k[r])[ids.size - top_k[r]]
            above, equal = ids[z[ids] > edge], ids[z[ids] == edge]
            ids = np.sort(np.concatenate([above, equal[:top_k[r] - above.size]]))
        if 0 < top_p[r] < 1:
            order = ids[np.lexsort((ids, -z[ids]))]
            mass = np.cumsum(np.exp((z[order] - best) / temp))
            ids = np.sort(order[:1 + int(np.searchsorted(mass, float(top_p[r]) * mass[-1], side="left"))])
        w = np.exp((z[ids] - best) / temp)
        if min_p[r] > 0:
            ids, w = ids[w >= float(min_p[r])], w[w >= float(min_p[r])]
        mass = np.cumsum(w)
        at = min(int(np.searchsorted(mass, float(u[r]) * mass[-1], side="right")), ids.size - 1)
        tok[r], count[r] = ids[at], ids.size
        prob[r], lse[r] = w[at] / mass[-1], best / temp + math.log(mass[-1])
    return {"tok": tok, "prob": prob, "count": count, "lse": lse}


def _exact_distill(s):
    c, rows, V = s.c, *s.logits.shape
    dev, T = s.logits.device, s.T
    want = c["kind"] != "loss"
    loss, accept = torch.zeros(rows, dtype=torch.float64, device=dev), torch.zeros(rows, dtype=torch.float64, device=dev)
    grad = torch.zeros((rows, V), dtype=torch.float64, device=dev) if want else None
    kk = s.idx.shape[1]
    step = max(1, (_CHUNK // 4) // V)
    for r0 in range(0, rows, step):
        r = slice(r0, min(rows, r0 + step))
        n = r.stop - r.start
        lnq = torch.log_softmax(s.logits[r].double() / T, 1)
        # the target as a dense row: the record's entries in their places (slots without an entry go behind the row)
        inside = torch.arange(kk, device=dev).expand(n, kk) < s.count[r].unsqueeze(1)
        where = torch.where(inside, s.idx[r].long(), V)
        p = torch.zeros((n, V + 1), dtype=torch.float64, device=dev).scatter_(1, where, torch.where(inside, s.prob[r].double(), 0.0))[:, :V]
        on = torch.zeros((n, V + 1), dtype=torch.bool, device=dev).scatter_(1, where, True)[:, :V]
        q = torch.exp(lnq)
        accept[r] = torch.where(on, torch.minimum(p, q), 0.0).sum(1)
        rest = (1.0 - p.sum(1)).clamp(min=0.0)
        share = torch.where(on, 0.0, q).sum(1)
        if c["tail"]:
            total = p.sum(1) + rest
            tail = torch.where(rest > 0, rest * (torch.log(rest) - torch.log(share)), 0.0)
            slope = torch.where(rest > 0, rest / share, 0.0)
        else:
            p = p / torch.where(p.sum(1) > 0, p.sum(1), 1.0).unsqueeze(1)
            total, tail, slope = torch.ones_like(rest), torch.zeros_like(rest), torch.zeros_like(rest)
        some = s.count[r] > 0
        kl = torch.where(p > 0, p * (torch.log(p) - lnq), 0.0).sum(1) + tail
        loss[r] = torch.where(some, kl, 0.0)
        if want:
            d = q * total.unsqueeze(1) - p - torch.where(on, 0.0, q * slope.unsqueeze(1))
            grad[r] = d * torch.where(some, s.weight[r].double() / T, 0.0).unsqueeze(1)
    out = {"loss": loss, "accept": accept}
    return dict(out, grad=grad) if want else out


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    c = case
    rows, V, esz = c["rows"], c["V"], 4 if c["dtype"] == "f32" else 2
    once = rows * V * esz
    if c["kind"] == "sample":
        # the logits in, four words a row out (and the uniform and the settings in); a subtraction, an exponential and a sum per element
        return {"bytes": once + rows * (4 + 16) + (16 * rows if c["mixed"] else 0), "flops": 3 * rows * V}
    record = rows * (min(c["k"], V) * 8 + 4)
    if c["kind"] == "loss":
        return {"bytes": once + record + 8 * rows, "flops": 3 * rows * V}
    # the gradient out as well: one more exponential and product per element
    return {"bytes": 2 * once + record + 12 * rows, "flops": 6 * rows * V}
