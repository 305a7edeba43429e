"""Seeded random cases of picospec_adjust, picospec_embed, picospec_clip_grad and their gradients against 64 bits, with the sizes around the kernels' internal boundaries (chunks, vectors,
shares of a row, pieces, the border between one launch and two).  PICOSPEC_SWEEP_CASES and PICOSPEC_SWEEP_SEED lengthen and move the hunt."""
import math
import os
import random

import pytest
import torch

from test_gpu_adjust import ODD, Case, hold, same_bits
from test_gpu_clip import OFF
from test_gpu_embed import HALF, _expect

pytestmark = pytest.mark.gpu

CASES = int(os.environ.get("PICOSPEC_SWEEP_CASES", 40))
SEED = int(os.environ.get("PICOSPEC_SWEEP_SEED", 0))
TYPES = (torch.float32, torch.bfloat16)


@pytest.fixture(scope="module")
def ps():
    from paper_2603_19133_amd import binding
    return binding


def _near(r, of):
    return max(1, r.choice(of) + r.randint(-3, 3))


@pytest.mark.parametrize("i", range(CASES))
def test_adjust(gpu, ps, i):
    r = random.Random(SEED * 100003 + i)
    V = r.choice([_near(r, [1, 32, 1024, 2048, 4096, 8192, 16384]), r.randint(1, 30000)])
    B = r.choice([1, 2, 5, 40, 300]) if V < 5000 else r.choice([1, 2, 9])
    most = r.choice([0, 0, 1, 6, 20])
    target = r.random() < 0.7
    gammas = [r.randint(0, most) for _ in range(B)]
    cap = r.choice([0, 1, 3, 4, 5, 100, 2000, 9000])
    kw = dict(seed=SEED + i, V=V, dtype=r.choice(TYPES), gammas=gammas, target=target, cap=cap, masks=r.choice([0, 1, 5]), mixed=r.random() < 0.7, bias=r.choice([0, 0, 7, 300]),
              pad=r.choice([0, 0, 1, 5]), values=r.choice([None, None, ODD]), token_range=r.choice([None, None, min(V, 20)]))
    print(f"[case] {kw}", flush=True)
    c = Case(**kw)
    _, z = c.device_rows(gpu, c.z, kw["pad"])
    hist, args = c.arguments(ps, gpu)
    out = ps.adjust(z, c.V, hist, **args)
    hold(out, *c.expect(), c.z)
    ps.adjust(z, c.V, hist, out=z, **args)
    assert same_bits(z, out)
    _, z = c.device_rows(gpu, c.z, kw["pad"])
    hist, args = c.arguments(ps, gpu, grad=True)
    g = ps.adjust_grad(c.grad.to(gpu), z, c.V, hist, **args)
    hold(g, *c.expect_grad(), c.grad)
    into = c.grad.to(gpu)
    ps.adjust_grad(into, z, c.V, hist, out=into, **args)
    assert same_bits(into, g)


@pytest.mark.parametrize("i", range(CASES))
def test_embed(gpu, ps, i):
    r = random.Random(SEED * 100003 + 50000 + i)
    n = r.choice([_near(r, [1, 8, 64, 1024, 2048]), r.randint(1, 6000), 30000])
    V = r.choice([_near(r, [1, 8, 256, 2048]), r.randint(1, 40000)])
    d = r.choice([_near(r, [1, 4, 8, 32, 256, 1024, 2048, 4096]), r.randint(1, 300)]) if n * V < 3e7 else r.randint(1, 40)
    dtype, out_dtype, scale = r.choice(TYPES), r.choice(TYPES), r.choice([1.0, 2.5, -0.3])
    print(f"[case] {n} {V} {d} {dtype} {out_dtype} {scale}", flush=True)
    g = torch.Generator(device=gpu).manual_seed(SEED + i)
    power = r.choice([1.0, 4.0, 20.0])                        # (tokens by how often the first ones occur)
    tok = (torch.rand(n, device=gpu, generator=g) ** power * (V + r.choice([0, 1]))).to(torch.int32) - r.choice([0, 0, 1])
    there = ((tok >= 0) & (tok < V)).unsqueeze(1)
    table = torch.randn((V, d), device=gpu, generator=g).to(dtype)
    s32 = float(torch.tensor(scale, dtype=torch.float32))
    want = torch.where(there, table[tok.clamp(0, V - 1).long()].double() * s32, 0.0)
    assert bool(((ps.embed(table, tok, scale).double() - want).abs() <= (HALF[dtype] + 2.0 ** -24) * (1 + 2.0 ** -20) * want.abs()).all())
    rows = torch.randn((n, d + 2), device=gpu, generator=g).to(dtype)[:, :d]
    add = r.random() < 0.4
    old = torch.randn((V, d), device=gpu, generator=g).to(out_dtype)
    s, bound, k = _expect(rows, tok, V, scale, old if add else None)
    out = ps.embed_grad(rows, tok, V, scale, out=old.clone(), accumulate=add)
    assert bool(((out.double() - s).abs() <= bound + HALF[out_dtype] * (s.abs() + bound)).all())
    assert torch.equal(out[(k == 0)[:, 0]], old[(k == 0)[:, 0]] if add else torch.zeros_like(old)[(k == 0)[:, 0]])
    assert torch.equal(out, ps.embed_grad(rows, tok, V, scale, out=old.clone(), accumulate=add))


@pytest.mark.parametrize("i", range(CASES))
def test_clip(gpu, ps, i):
    r = random.Random(SEED * 100003 + 90000 + i)
    count = r.choice([1, 2, 15, 16, 17, 127, 128, 129, 260])
    sizes = [r.choice([r.randint(0, 50), _near(r, [1024, 4096, 16384]), r.randint(1, 100000)]) for _ in range(count)]
    print(f"[case] {count} {sum(sizes)}", flush=True)
    g = torch.Generator(device=gpu).manual_seed(SEED + i)
    flats = {t: torch.randn(sum(sizes) + 8, device=gpu, generator=g).to(t) for t in TYPES}
    at, grads = r.randint(0, 7), []
    for n in sizes:                                           # (views at any element)
        grads.append(flats[r.choice(TYPES)][at:at + n])
        at += n
    before = [x.clone() for x in grads]
    want = math.sqrt(math.fsum(float((x.double() ** 2).sum()) for x in before))
    limit = r.choice([0.0, 0.5, 10.0, 1e6, math.inf])
    factor = 1.0 if math.isinf(limit) else min(1.0, limit / (want + 1e-6))
    outs = [torch.full_like(x, 3.0) for x in grads] if r.random() < 0.5 else None
    around = {t: f.clone() for t, f in flats.items()}
    norm = ps.clip_grad(grads, limit, outs)
    assert abs(norm.item() - want) <= want * 2.0 ** -24 * (1 + 2.0 ** -10)
    for x, b, o in zip(grads, before, outs or grads):
        assert torch.equal(o, b) if factor == 1.0 else bool(((o.double() - b.double() * factor).abs() <= OFF[b.dtype] * b.double().abs() * factor + 2.0 ** -133).all())
    for x, b in zip(grads, before):                           # (and nothing beside the tensors)
        x.copy_(b)
    assert all(torch.equal(flats[t], around[t]) for t in TYPES)
