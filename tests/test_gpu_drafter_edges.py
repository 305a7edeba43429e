"""The sampler and the distillation loss at the edges of what they take."""
import math

import numpy as np
import pytest
import torch

import test_gpu_distill as td
import test_gpu_sample as ts

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ps():
    from paper_2603_19133_amd import binding
    return binding


def test_a_vocabulary_wider_than_the_view_is_refused(gpu, ps):
    """... by the forward call (the backward call, whose gradient has the view's columns, would be the first to notice)."""
    from paper_2603_19133_amd.training import distill_loss
    z = torch.zeros(4, 108, device="cuda")[:, :100]
    rec = ps.Compressed(torch.zeros(4, 5, dtype=torch.int32, device="cuda"), torch.ones(4, 5, device="cuda"), torch.ones(4, dtype=torch.int32, device="cuda"),
                        torch.ones(4, device="cuda"), torch.zeros(4, device="cuda"), 5)
    for call in (lambda v: distill_loss(z, rec, v, 1.0), lambda v: ps.distill(z, v, 1.0, rec), lambda v: ps.sample(z, v, torch.zeros(4, device="cuda"))):
        with pytest.raises(ps.PicoSpecError):
            call(101)
        call(100)
    torch.cuda.synchronize()


# ---------------------------------------------------------------- the sampler: uniforms at the ends over masked ids

def _masked(rows, V, dtype, seed, T=1.0):
    """Rows whose first and last ids are masked, whole segments of them: with -inf, with the type's lowest value, with both in turn, or all but 20 ids."""
    z, _ = ts.rows_of(rows, V, dtype, "normal", seed, 3, 1)
    low, a, b = torch.finfo(dtype).min, V // 5, V - V // 7
    for r in range(rows):
        fill = torch.full((V,), -math.inf if r % 2 == 0 else low, dtype=dtype, device="cuda")
        if r % 6 >= 4:                                             # (both in turn)
            fill[::2] = -math.inf if r % 2 else low
        if r % 3 == 2:                                             # (a grammar that allows 20 ids)
            keep = torch.zeros(V, dtype=torch.bool, device="cuda")
            keep[torch.from_numpy(np.random.default_rng(r).choice(np.arange(a, b), min(20, b - a), replace=False)).cuda()] = True
        else:
            keep = torch.zeros(V, dtype=torch.bool, device="cuda")
            keep[a:b] = True
        z[r] = torch.where(keep, z[r], fill)
    return z


@pytest.mark.parametrize("setting", [dict(), dict(top_k=50), dict(top_k=50, top_p=0.9), dict(top_k=700), dict(top_k=900, min_p=1e-30), dict(top_k=9000), dict(top_p=0.9), dict(top_p=0.999), dict(min_p=0.02)],
                         ids=str)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(6, 37), (6, 5003), (6, 40009), (138, 20011)])
def test_uniforms_at_the_ends_over_masked_ids(gpu, ps, rows, V, dtype, setting):
    """u = 0 draws the first id with any weight in 64 bits, the largest u below 1 the last but for 2^-24 of the mass: masked ids in front of and behind them
    are not drawn, whether they hold -inf or the type's lowest value, and also where top-k keeps more ids than are allowed.  (Of many rows u = 0 alone: the other
    two lie near steps of some 10^-8 of the mass.)"""
    print(f"[case] sample ends {rows} x {V} {dtype} {setting}", flush=True)
    z = _masked(rows, V, dtype, rows + V)
    s = dict(dict(top_k=0, top_p=0.0, min_p=0.0), **setting)
    for v in (0.0, 2.0 ** -24, 1.0 - 2.0 ** -24) if rows < 10 else (0.0,):
        u = torch.full((rows,), v, device="cuda")
        ts.compare(ps.sample(z, V, u, temperature=0.8, **s), z, 0.8, s["top_k"], s["top_p"], s["min_p"], u)
    got = ps.sample(z, V, torch.ones(rows, device="cuda"), temperature=0.8, **s)              # (outside the range: the last)
    torch.cuda.synchronize()
    tok = got.tok.long()
    assert (z[torch.arange(rows, device="cuda"), tok] > -1e30).all() and (tok >= 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(5, 30011), (138, 9001)])
def test_a_uniform_on_the_border_of_a_masked_segment(gpu, ps, rows, V, dtype):
    """Equal logits on either side of a masked block, u at the border exactly: the first id behind the block."""
    z = torch.full((rows, V), torch.finfo(dtype).min, dtype=dtype, device="cuda")
    z[::2] = -math.inf
    z[:, 16:528], z[:, 8200:8712] = 0.0, 0.0
    u = torch.full((rows,), 0.5, device="cuda")
    for s in (dict(), dict(top_k=2000), dict(top_k=400), dict(top_p=0.75), dict(min_p=0.5)):
        s = dict(dict(top_k=0, top_p=0.0, min_p=0.0), **s)
        ts.compare(ps.sample(z, V, u, **s), z, 1.0, s["top_k"], s["top_p"], s["min_p"], u)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("setting", [dict(top_k=300), dict(top_k=1500), dict(top_k=4000, top_p=0.999), dict(min_p=1e-25), dict()], ids=str)
@pytest.mark.parametrize("rows,V", [(3, 5003), (4, 40009), (138, 20011)])
def test_the_first_kept_id_of_hardly_any_weight(gpu, ps, rows, V, dtype, setting):
    """u = 0 where the kept ids' weights lie up to e^-300 apart: the first kept id, however little it weighs."""
    z, _ = ts.rows_of(rows, V, dtype, "normal", 5 * V)
    s = dict(dict(top_k=0, top_p=0.0, min_p=0.0), **setting)
    u = torch.zeros(rows, device="cuda")
    ts.compare(ps.sample(z, V, u, temperature=0.08, **s), z, 0.08, s["top_k"], s["top_p"], s["min_p"], u)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_a_temperature_per_row_that_the_host_would_refuse_is_greedy(gpu, ps, dtype):
    z, u = ts.rows_of(8, 9001, dtype, "normal", 15)
    T = torch.tensor([math.inf, 1.0, math.nan, -1.0, -math.inf, 0.0, 3.0e38, 0.5], device="cuda")
    as_said = torch.where(torch.isfinite(T) & (T > 0), T, torch.zeros_like(T))
    ts.compare(ps.sample(z, 9001, u, temperature=T), z, as_said, 0, 0.0, 0.0, u)


# ---------------------------------------------------------------- the loss: masks of finite values in blocks

@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("low,T", [(-1e4, 1.0), (-1e9, 1.0), (-1e10, 1.0), (-1e20, 1.0), (-1e30, 0.7), (None, 1.0), (None, 2.0), (None, 0.5), (-5e7, 1.0), (-2e7, 1.0)], ids=str)
@pytest.mark.parametrize("rows,V,k", [(3, 700, 8), (5, 9001, 40), (5, 9001, 700), (3, 70001, 12), (4, 40003, 2000)])
def test_blocks_of_ids_masked_with_finite_values(gpu, ps, rows, V, k, low, T, dtype, tail):
    """A vocabulary's first ids, its last ones or whole stretches in between, masked with a finite value: what a wave sees first is masked, all that it sees or what it
    sees last, and so is a whole part of a row that several workgroups share."""
    print(f"[case] distill blocks {rows} x {V} k={k} low={low} T={T} {dtype} tail={tail}", flush=True)
    z, idx, prob, count = td.inputs(rows, V, k, dtype, T, V + k, 1, 1)
    low = torch.finfo(dtype).min if low is None else low
    on = torch.zeros(rows, V, dtype=torch.bool, device="cuda")
    on.scatter_(1, torch.from_numpy(idx.astype(np.int64)).cuda(), True)
    off = torch.zeros(rows, V, dtype=torch.bool, device="cuda")
    off[0, : V // 2] = True
    off[1, V // 2:] = True
    off[2, V // 3: 2 * V // 3] = True
    if rows > 3:
        off[3, : 9 * V // 10] = True
        off[3, ::2] = True
    if rows > 4:
        off[4] = True
        off[4, V // 2: V // 2 + 64] = False
    z[off & ~on] = low
    td.run_all(ps, z, V, T, idx, prob, count, tail, np.random.default_rng(k).uniform(0.5, 1.5, rows).astype(np.float32))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("low,T", [(-1e10, 1.0), (-1e30, 2.0), (None, 2.0)], ids=str)
def test_a_masked_block_with_record_ids_in_it(gpu, ps, low, T, dtype):
    """The same with record ids masked as well: they have probability 0 there."""
    rows, V, k = 4, 9001, 40
    z, idx, prob, count = td.inputs(rows, V, k, dtype, T, 5, 1, 1)
    low = torch.finfo(dtype).min if low is None else low
    z[:, : V // 2] = low
    prob[idx < V // 2] = 0.0
    for tail in (0, 1):
        td.run_all(ps, z, V, T, idx, prob, count, tail, np.ones(rows, np.float32))


# ---------------------------------------------------------------- the loss: what is off the record far below what is on it

def _gapped(rows, V, k, dtype, T, gap, seed):
    """Logits whose record ids lie `gap` nats above all others, and records with 0.99 of the mass."""
    rng = np.random.default_rng(seed)
    s = rng.normal(size=(rows, V)) - gap
    idx = np.stack([rng.choice(V, k, replace=False) for _ in range(rows)]).astype(np.int32)
    np.put_along_axis(s, idx, np.clip(rng.normal(size=(rows, k)), -3.0, 3.0), 1)
    p = rng.random((rows, k)) + 0.1
    z = torch.zeros(rows, V + 3, dtype=dtype, device="cuda")[:, :V]
    z.copy_(torch.from_numpy(s * T).to(dtype))
    return z, idx, (p / p.sum(1, keepdims=True) * 0.99).astype(np.float32), np.full(rows, k, np.int32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("gap,T", [(20.0, 1.0), (80.0, 1.0), (95.0, 1.0), (110.0, 1.0), (110.0, 0.1), (300.0, 1.0), (300.0, 4.0), (700.0, 1.0), (700.0, 0.01)], ids=str)
@pytest.mark.parametrize("rows,V,k", [(3, 1000, 12), (4, 9001, 300), (4, 9001, 1500), (600, 2049, 600), (3, 70001, 20), (66, 61001, 900)], ids=str)
def test_the_tail_far_below_the_record(gpu, ps, rows, V, k, gap, T, dtype):
    """The gradient off the record has a sum of -pt q_v / qt = -pt however small qt is, as long as 64 bits hold it."""
    print(f"[case] distill gap {gap} T={T} {rows} x {V} k={k} {dtype}", flush=True)
    z, idx, prob, count = _gapped(rows, V, k, dtype, T, gap, k)
    d = td.run_all(ps, z, V, T, idx, prob, count, 1, np.ones(rows, np.float32))
    on = torch.from_numpy(idx.astype(np.int64)).cuda()
    off = d.grad.double().scatter(1, on, 0.0)
    assert ((off.sum(1) * T + 0.01).abs() <= 0.01 * 2.0 ** -7).all()             # (all of one sign: bf16's roundings, 2^-8 relative each)


def test_the_tail_far_below_a_record_far_from_zero(gpu, ps):
    """The same where the exponents are beyond the fused form: offsets that all logits share, of which fp32 holds steps of 2 nats."""
    rows, V, k = 4, 9001, 300
    for k in (12, 300):
        rng = np.random.default_rng(8)
        s = 3.0e7 - 300.0 + 2.0 * rng.integers(0, 6, (rows, V))
        idx = np.stack([rng.choice(V, k, replace=False) for _ in range(rows)]).astype(np.int32)
        np.put_along_axis(s, idx, 3.0e7 + 2.0 * rng.integers(0, 4, (rows, k)), 1)
        p = rng.random((rows, k)) + 0.1
        z = torch.from_numpy(s).float().cuda()
        assert (z.double().cpu().numpy() == s).all()
        td.run_all(ps, z, V, 1.0, idx, (p / p.sum(1, keepdims=True) * 0.99).astype(np.float32), np.full(rows, k, np.int32), 1, np.ones(rows, np.float32))


# ---------------------------------------------------------------- the loss: records that hold all of the row's support

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,V,k,low", [(4, 300, 300, 0.0), (4, 4096, 4096, 0.0), (5, 9001, 20, -math.inf), (5, 9001, 1500, None), (600, 2049, 600, None), (3, 70001, 20, -1e30)], ids=str)
def test_a_record_of_all_of_the_support(gpu, ps, rows, V, k, low, dtype):
    """All that top-k can keep is in the record, and nothing has any mass off it: what the entries' roundings leave of 1 is no tail.  Where a record leaves more than
    that, the loss is infinite."""
    rng = np.random.default_rng(k)
    idx = np.stack([rng.choice(V, k, replace=False) for _ in range(rows)]).astype(np.int32)
    z = torch.full((rows, V), torch.finfo(dtype).min if low is None else low, dtype=dtype, device="cuda")
    z.scatter_(1, torch.from_numpy(idx.astype(np.int64)).cuda(), torch.from_numpy(rng.normal(size=(rows, k))).to(dtype).cuda())
    p = rng.random((rows, k)) + 0.1
    p /= p.sum(1, keepdims=True)
    left = np.array([2.0 ** -24, 2.0 ** -22, -2.0 ** -23, 2.0 ** -21, 1e-3])[np.arange(rows) % 5]
    prob = (p * (1.0 - left[:, None])).astype(np.float32)
    count = np.full(rows, k, np.int32)
    short = left == 1e-3
    z64, p64 = z.double().cpu().numpy(), prob.astype(np.float64)
    assert (1.0 - p64.sum(1))[left > 0].min() > 0.0
    lnq = np.take_along_axis(z64 - np.log(np.exp(z64).sum(1, keepdims=True)), idx, 1)
    loss = (p64 * (np.log(p64) - lnq)).sum(1)
    loss[short] = np.inf
    whole = np.where(short, 1.0, p64.sum(1))
    grad, tol = np.zeros((rows, V)), np.zeros((rows, V))
    np.put_along_axis(grad, idx, whole[:, None] * np.exp(lnq) - p64, 1)
    np.put_along_axis(tol, idx, td.E * np.exp(lnq) + 2.0 ** -40, 1)
    from paper_2603_19133_amd.training import distill_loss
    rec = td.record(ps, idx, prob, count)
    d = ps.distill(z, V, 1.0, rec, tail=1, grad=True)
    f = ps.distill(z, V, 1.0, rec, tail=1)
    leaf = z.detach().requires_grad_()
    lo, _ = distill_loss(leaf, rec, V, 1.0, tail=1)
    lo.sum().backward()
    for t in (d.loss, f.loss, lo):
        assert torch.equal(torch.isinf(t.detach().cpu()), torch.from_numpy(short))
        td.check(t, loss, td.E)
    for t in (d.grad, ps.distill_grad(z, V, 1.0, rec, f.stats, tail=1), leaf.grad):
        td.check(t, grad, tol, dtype)


def test_records_of_compress_of_all_of_the_support(gpu, ps):
    """What the framework's own records of a whole vocabulary, and of rows of which a grammar allows fewer ids than the record has places, leave of 1 by rounding."""
    for V, k in ((4096, 4096), (5003, 64)):
        z, _ = ts.rows_of(64, V, torch.float32, "normal", V)
        if k < V:
            z[:, : V - 50] = -math.inf
        rec = ps.compress(z, V, 0.9, k)
        left = 1.0 - rec.prob.double().sum(1) if k == V else 1.0 - torch.where(torch.arange(k, device="cuda") < rec.count[:, None], rec.prob, 0.0).double().sum(1)
        assert (left > 0).any() and left.max() < 2.0 ** -20
        s = torch.where(z > -1e30, z * 0.9, z)
        d = ps.distill(s, V, 0.9, rec, tail=1, grad=True)
        assert torch.isfinite(d.loss).all() and torch.isfinite(d.grad).all()


# ---------------------------------------------------------------- the loss: NaN and +inf

@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V,k", [(3001, 16), (9001, 300), (9001, 2000), (90001, 16)])
def test_nan_and_inf_make_a_row_nan(gpu, ps, V, k, dtype, tail):
    """Loss, acceptance and every element of the gradient: NaN throughout the row, among nothing but masked ids, in all of one workgroup's share of it, on the record
    (with probability 0 as well), off it; +inf on and off it.  The other rows keep their bits."""
    from paper_2603_19133_amd.training import distill_loss
    z, idx, prob, count = td.inputs(12, V, k, dtype, 1.0, 3)
    prob[6, 4] = 0.0
    rec = td.record(ps, idx, prob, count)

    def outputs():
        d = ps.distill(z, V, 1.0, rec, tail=tail, grad=True)
        f = ps.distill(z, V, 1.0, rec, tail=tail)
        g = ps.distill_grad(z, V, 1.0, rec, f.stats, tail=tail)
        leaf = z.detach().requires_grad_()
        lo, ac = distill_loss(leaf, rec, V, 1.0, tail=tail)
        lo.sum().backward()
        torch.cuda.synchronize()
        return [d.loss, f.loss, lo.detach(), d.accept, f.accept, ac], [d.grad, g, leaf.grad]
    want = outputs()
    off = [next(x for x in range(V // 2, V) if x not in set(idx[r].tolist())) for r in range(12)]
    z[1] = math.nan
    z[2] = -math.inf
    z[2, off[2]] = math.nan
    z[3, : V // 3] = math.nan
    z[4, int(idx[4, 4])] = math.nan
    z[5, off[5]] = math.nan
    z[6, int(idx[6, 4])] = math.nan
    z[7, int(idx[7, 4])] = math.inf
    z[8, off[8]] = math.inf
    z[9] = math.inf
    z[10, ::2], z[10, 1::2] = math.inf, math.nan
    got = outputs()
    for t in got[0]:
        assert torch.isnan(t[1:11]).all(), t
    for t in got[1]:
        assert torch.isnan(t[1:11].float()).all(), (~torch.isnan(t.float())).sum(1)
    for a, b in zip(got[0] + got[1], want[0] + want[1]):
        assert torch.equal(a[0], b[0]) and torch.equal(a[11], b[11])
