"""picospec_distill, picospec_distill_grad and training.distill_loss against the definition in 64 bits.

Tolerances.  A weight 2^x, x = (z - M) log2(e) / T in fp32, has a relative error of at most ln 2 |x| 2^-22 (the subtraction, the
factor's two roundings, the product) + 2^-23 (the exponential).  What a sum over the row is made of lies within 2^-24 of it: |x| <= 24 +
log2 V <= 42 covers all but 2^-18 of its rounding, so sums, and with them ln S, are off by at most E = 42 ln 2 2^-22 + 2^-20 = 8e-6
(everything behind the sums is 64-bit).  Loss: E + half a step of fp32; acceptance likewise (values up to 1).  A gradient off the record is
(weight / T) b q_v, q_v off by ln 2 |x_v| 2^-22 + E + 2^-22 relatively and b = W - pt / qt by E pt / qt; on the record W q - p is formed in 64 bits from a
64-bit weight: off by E W q.  Rounded once: half a step of the type."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

E = 42 * math.log(2) * 2.0 ** -22 + 2.0 ** -20


@pytest.fixture(scope="module")
def ps():
    from paper_2603_19133_amd import binding
    return binding


def reference(z, V, T, idx, prob, count, tail, weight=None):
    """Definition, row by row, in float64: loss, accept, grad [rows, V] and the gradient's tolerance without the type's rounding."""
    z = z[:, :V].astype(np.float64)
    n, T = z.shape[0], float(np.float32(T))
    loss, acc, grad, tol = np.zeros(n), np.zeros(n), np.zeros((n, V)), np.zeros((n, V))
    for r in range(n):
        c = min(max(int(count[r]), 0), idx.shape[1])
        if c == 0 or z[r].max() == -np.inf:
            continue
        ids, p = idx[r, :c], prob[r, :c].astype(np.float64)
        ok = (ids >= 0) & (ids < V)
        ids, p = ids[ok], p[ok]
        y = (z[r] - z[r].max()) / T
        w = np.exp(y)
        q, lnq = w / w.sum(), y - np.log(w.sum())
        mass = p.sum()
        off = np.ones(V, bool)
        off[ids] = False
        scale = (1.0 if weight is None else float(weight[r])) / T
        if tail:
            pt, qt = max(0.0, 1.0 - mass), q[off].sum()
            whole, slope = mass + pt, (pt / qt if pt > 0 and qt > 0 else 0.0)
            b = whole - slope if not (pt > 0 and qt == 0) else 0.0
        else:
            p = p / mass if mass > 0 else p
            pt, qt, whole, slope = 0.0, 1.0, float(mass > 0), 0.0
            b = whole
        with np.errstate(divide="ignore", invalid="ignore"):
            loss[r] = np.where(p > 0, p * (np.log(np.where(p > 0, p, 1.0)) - lnq[ids]), 0.0).sum()
            if pt > 0:
                loss[r] += pt * (np.log(pt) - np.log(qt))
        acc[r] = np.minimum(prob[r, :c].astype(np.float64)[ok], q[ids]).sum()
        grad[r] = scale * b * q
        grad[r, ids] = scale * (whole * q[ids] - p)
        x = np.minimum(np.abs(y) / math.log(2), 200.0)
        tol[r] = abs(scale) * q * (abs(b) * (math.log(2) * x * 2.0 ** -22 + E + 2.0 ** -22) + slope * E)
        tol[r, ids] = abs(scale) * (E * whole * q[ids] + 2.0 ** -40 * p)
    return loss, acc, grad, tol


def inputs(rows, V, k, dtype, T, seed, pad=0, shift=0, ragged=False, spread=3.0):
    """Student logits as a view [rows, V] off any boundary, and a record of a correlated target (host arrays and device tensors)."""
    rng = np.random.default_rng(seed)
    t = rng.normal(size=(rows, V)) * spread
    s = 0.9 * t + 1.2 * rng.normal(size=(rows, V))
    flat = torch.zeros(rows * (V + pad) + shift, dtype=dtype, device="cuda")
    z = flat[shift:].view(rows, V + pad)[:, :V]
    z.copy_(torch.from_numpy(s).to(dtype))
    order = np.argsort(-t, axis=1, kind="stable")[:, :k].astype(np.int32)
    p = np.exp((t - t.max(1, keepdims=True)) / T)
    p = np.take_along_axis(p / p.sum(1, keepdims=True), order, 1).astype(np.float32)
    count = np.full(rows, k, np.int32)
    if ragged:
        count = rng.integers(0, k + 1, rows).astype(np.int32)
        count[::3] = 0
        unused = np.arange(k)[None] >= count[:, None]
        order[unused], p[unused] = -1, 0.0
    return z, order, p, count


def record(ps, idx, prob, count):
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return ps.Compressed(d(idx), d(prob), d(count), torch.zeros(len(count), device="cuda"), torch.zeros(len(count), device="cuda"), idx.shape[1])


def check(got, want, tol, dtype=torch.float32):
    got = got.detach().double().cpu().numpy()
    tol = tol + np.abs(want) * (torch.finfo(dtype).eps / 2) * (1 + 2.0 ** -10) + float(torch.finfo(dtype).smallest_normal)
    same_inf = np.isinf(want) & (got == want)
    bad = ~(np.abs(got - np.where(np.isinf(want), 0.0, want)) <= tol) & ~same_inf
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5].tolist(), got[bad][:5], want[bad][:5], np.broadcast_to(tol, bad.shape)[bad][:5])


def run_all(ps, z, V, T, idx, prob, count, tail, weight):
    """Step, forward + backward through autograd, and the calls apart: all against the definition."""
    from paper_2603_19133_amd.training import distill_loss
    rec = record(ps, idx, prob, count)
    w = torch.from_numpy(weight).cuda()
    loss, acc, grad, tol = reference(z.float().cpu().numpy(), V, T, idx, prob, count, tail, weight)
    d = ps.distill(z, V, T, rec, tail=tail, weight=w, grad=True)
    f = ps.distill(z, V, T, rec, tail=tail)
    g = ps.distill_grad(z, V, T, rec, f.stats, tail=tail, weight=w)
    leaf = z.detach().requires_grad_()
    lo, ac = distill_loss(leaf, rec, V, T, tail=tail)
    lo.backward(w)
    torch.cuda.synchronize()
    for o in (d, f):
        check(o.loss, loss, E)
        check(o.accept, acc, E)
    check(lo, loss, E)
    check(ac, acc, E)
    assert f.grad is None and not ac.requires_grad
    for o in (d.grad, g, leaf.grad):
        assert o.dtype == z.dtype and o.shape == (z.shape[0], V)
        check(o, grad, tol, z.dtype)
    return d


@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,V,k,T,pad,shift,ragged", [
    (3, 1, 1, 1.0, 0, 0, False),                  # a vocabulary of one: the record holds everything
    (2, 2, 2, 0.5, 3, 1, False),
    (5, 7, 3, 1.0, 0, 3, False),
    (4, 65, 10, 0.7, 5, 1, False),
    (3, 1000, 1, 1.0, 0, 0, False),
    (3, 1000, 1000, 1.3, 1, 7, False),            # a record of the whole row: nothing is left off it
    (9, 4099, 64, 0.9, 2, 3, True),
    (4, 8192, 1025, 1.0, 0, 0, True),             # more entries than threads
    (3, 32000, 256, 0.6, 0, 0, False),
    (2, 50001, 4096, 1.0, 3, 1, False),           # the longest record
    (2, 163841, 777, 0.8, 0, 5, False),           # longer than what is held between sum and gradient
    (2, 40001, 300, 1.0, 1, 1, True),
    (2, 30003, 1600, 1.0, 0, 3, True),
    (600, 2049, 600, 1.0, 1, 0, True),            # slots, bf16, gradient in the call
    (1100, 515, 7, 1.0, 0, 1, True),              # many rows
    (1, 420001, 1000, 1.0, 0, 1, False),          # marks that do not fit beside the slots
    (1, 1048576, 300, 1.0, 0, 1, False),          # the longest row
], ids=str)
def test_against_the_definition(gpu, ps, rows, V, k, T, pad, shift, ragged, dtype, tail):
    print(f"[case] distill rows={rows} V={V} k={k} T={T} pad={pad} shift={shift} {dtype} tail={tail}", flush=True)
    z, idx, prob, count = inputs(rows, V, k, dtype, T, rows * 1000 + V, pad, shift, ragged)
    weight = np.random.default_rng(V).uniform(-1.0, 2.0, rows).astype(np.float32)
    run_all(ps, z, V, T, idx, prob, count, tail, weight)


@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,V,k,shift", [(5, 90001, 30, 1), (20, 70003, 700, 3), (3, 200000, 4096, 0), (100, 130001, 12, 1), (60, 65001, 12, 1)])
def test_split_rows(gpu, ps, rows, V, k, shift, dtype, tail):
    """Few long rows: with scratch, without it and with too little of it, against the definition; masked parts, a row that is masked whole, one without entries."""
    print(f"[case] distill split {rows} x {V} k={k} {dtype} tail={tail}", flush=True)
    z, idx, prob, count = inputs(rows, V, k, dtype, 1.0, V, 2, shift)
    z[1, : V // 2] = -math.inf
    z[2] = -math.inf
    count[0] = 0
    weight = np.random.default_rng(V).uniform(0.5, 1.5, rows).astype(np.float32)
    d = run_all(ps, z, V, 1.0, idx, prob, count, tail, weight)
    loss, acc, grad, tol = reference(z.float().cpu().numpy(), V, 1.0, idx, prob, count, tail, weight)
    dt, rec, w = 0 if dtype == torch.float32 else 1, record(ps, idx, prob, count), torch.from_numpy(weight).cuda()
    need = ps.scratch_bytes(ps.CALL_DISTILL, dt, rows, 0, V, 0)
    assert need == ps.workspace_bytes(ps.CALL_DISTILL, dt, rows, V, 0) and need > 0
    for size in (0, max(need - 1, 0)):
        ws = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
        lo, ac, g = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda"), torch.zeros(rows, V, dtype=dtype, device="cuda")
        assert ps.lib.picospec_distill(z.data_ptr(), dt, z.stride(0), rows, V, 1.0, rec.idx.data_ptr(), rec.prob.data_ptr(), rec.count.data_ptr(), k, tail, w.data_ptr(), lo.data_ptr(),
                                       ac.data_ptr(), None, g.data_ptr(), V, ws.data_ptr() if size else None, size, None) == ps.OK
        torch.cuda.synchronize()
        check(lo, loss, E)
        check(ac, acc, E)
        check(g, grad, tol, dtype)


@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shift,T", [(1000.0, 1.0), (-3e7, 1e4), (2e9, 1.0), (0.0, 1e-3)])
def test_logits_far_from_zero(gpu, ps, shift, T, dtype, tail):
    """Rows whose exponents are large: an offset that all logits share, beyond what the fused form of the exponents takes, a small temperature."""
    print(f"[case] distill far {shift} T={T} {dtype} tail={tail}", flush=True)
    z, idx, prob, count = inputs(4, 3001, 300, torch.float32, 1.0, 17)
    z = (z.double() * (1.0 if T >= 1.0 else 1e-2) * T + shift).to(dtype)
    run_all(ps, z, 3001, T, idx, prob, count, tail, np.ones(4, np.float32))


@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("k", [40, 1700])
def test_masks(gpu, ps, k, dtype, tail):
    """Masked ids (-inf and the type's lowest value), a row that is masked whole, record ids on masked logits, probabilities of 0, a mass
    of 0 and one above 1, entries outside the vocabulary, counts outside 0..k."""
    print(f"[case] distill masks k={k} {dtype} tail={tail}", flush=True)
    rows, V = 12, 5003
    z, idx, prob, count = inputs(rows, V, k, dtype, 1.0, 77, 1, 1)
    rng = np.random.default_rng(5)
    keep = torch.from_numpy(rng.random((rows, V)) < 0.125).cuda()
    for r in range(rows):
        keep[r, torch.from_numpy(idx[r].astype(np.int64)).cuda()] = True
    z[0:4] = torch.where(keep[0:4], z[0:4], torch.full_like(z[0:4], -math.inf))
    z[4:6] = torch.where(keep[4:6], z[4:6], torch.full_like(z[4:6], torch.finfo(dtype).min))
    z[1] = -math.inf                                          # no distribution
    z[2, int(idx[2, 3])] = -math.inf                          # p > 0 where q = 0: loss +inf, the gradient finite
    z[3, int(idx[3, 3])] = -math.inf
    prob[3, 3] = 0.0                                          # ... and p = 0 there: nothing
    off = torch.ones(V, dtype=torch.bool, device="cuda")
    off[torch.from_numpy(idx[6].astype(np.int64)).cuda()] = False
    z[6, off] = -math.inf                                     # nothing left off the record: tail 1 has loss +inf
    prob[7] = 0.0                                             # a record without mass
    prob[8] = prob[8] / prob[8].sum() * np.float32(1.25)      # ... with more than all of it: no tail
    idx[9, 5], idx[9, 6] = -1, V                              # passed over
    count[10], count[11] = -3, k + 9                          # clamped
    weight = np.ones(rows, np.float32)
    d = run_all(ps, z, V, 1.0, idx, prob, count, tail, weight)
    assert torch.isinf(d.loss[2]) and d.loss[1] == 0 and d.loss[10] == 0
    assert bool(torch.isinf(d.loss[6])) == bool(tail)
    assert torch.isfinite(d.grad.float()).all() and not d.grad[1].any() and not d.grad[10].any()


def test_nan_and_inf_stay_in_their_rows(gpu, ps):
    print("[case] distill nan", flush=True)
    z, idx, prob, count = inputs(4, 3001, 16, torch.float32, 1.0, 3)
    want = ps.distill(z, 3001, 1.0, record(ps, idx, prob, count), tail=1, grad=True)
    z[1, 17], z[2, 18] = math.nan, math.inf
    d = ps.distill(z, 3001, 1.0, record(ps, idx, prob, count), tail=1, grad=True)
    torch.cuda.synchronize()
    assert torch.isnan(d.loss[1:3]).all()
    for r in (0, 3):
        assert torch.equal(d.loss[r], want.loss[r]) and torch.equal(d.grad[r], want.grad[r])


@pytest.mark.parametrize("tail", [0, 1])
def test_gradient_against_differences(gpu, ps, tail):
    """Central differences of the definition in 64 bits: truncation h^2 / 6 |L'''| <= h^2, cancellation 2^-50 / h (losses below 8)."""
    print(f"[case] distill differences tail={tail}", flush=True)
    rows, V, k, T, h = 3, 50, 7, 0.8, 1e-4
    z, idx, prob, count = inputs(rows, V, k, torch.float32, T, 11, spread=1.5)
    d = ps.distill(z, V, T, record(ps, idx, prob, count), tail=tail, grad=True)
    z64 = z.double().cpu().numpy()
    num = np.zeros((rows, V))
    for v in range(V):
        up, dn = z64.copy(), z64.copy()
        up[:, v] += h
        dn[:, v] -= h
        num[:, v] = (reference(up, V, T, idx, prob, count, tail)[0] - reference(dn, V, T, idx, prob, count, tail)[0]) / (2 * h)
    tol = reference(z64, V, T, idx, prob, count, tail)[3]
    check(d.grad, num, tol + h * h / T ** 3 + 2.0 ** -50 / h)


def test_one_gradient_for_all_rows_and_a_wider_tensor(gpu, ps):
    """loss.mean().backward() hands one value for all rows; columns behind the vocabulary get a gradient of 0; a loss without a use none."""
    print("[case] distill mean", flush=True)
    from paper_2603_19133_amd.training import distill_loss
    z, idx, prob, count = inputs(6, 1003, 20, torch.float32, 1.0, 9)
    wide = torch.randn(6, 1010, device="cuda")
    wide[:, :1003] = z
    wide.requires_grad_()
    rec = record(ps, idx, prob, count)
    loss, acc = distill_loss(wide, rec, 1003, 1.0)
    loss.mean().backward()
    w = torch.full((6,), 1.0 / 6.0, device="cuda")
    want = ps.distill(wide.detach(), 1003, 1.0, rec, weight=w, grad=True).grad        # (the same rows: sums in the same order)
    torch.cuda.synchronize()
    assert torch.equal(wide.grad[:, :1003], want) and not wide.grad[:, 1003:].any()
    with pytest.raises(RuntimeError):
        acc.sum().backward()
    loss, _ = distill_loss(wide, rec, 1003, 1.0)
    with pytest.raises(RuntimeError, match="once"):
        torch.autograd.grad(loss.sum(), wide, create_graph=True)
    loss, _ = distill_loss(wide, rec, 1003, 1.0)
    rec.prob.mul_(0.5)                                         # (what the backward call reads may not change in between)
    with pytest.raises(RuntimeError, match="modified"):
        loss.sum().backward()


def test_streams_and_graph(gpu, ps):
    """The call works on the current stream; a captured one gives the eager result on every replay, with eager work between."""
    print("[case] distill stream and graph", flush=True)
    z, idx, prob, count = inputs(5, 9001, 33, torch.bfloat16, 1.0, 21)
    rec = record(ps, idx, prob, count)
    want = ps.distill(z, 9001, 1.0, rec, tail=1, grad=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ps.distill(z, 9001, 1.0, rec, tail=1, grad=True)
    side.synchronize()
    assert torch.equal(got.loss, want.loss) and torch.equal(got.grad, want.grad)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cap = ps.distill(z, 9001, 1.0, rec, tail=1, grad=True)
        gr = ps.distill_grad(z, 9001, 1.0, rec, cap.stats, tail=1)
    for i in range(3):
        z.copy_(torch.randn_like(z) * (1 + i))
        graph.replay()
        torch.cuda.synchronize()
        now = ps.distill(z, 9001, 1.0, rec, tail=1, grad=True)
        torch.cuda.synchronize()
        assert torch.equal(cap.loss, now.loss) and torch.equal(cap.grad, now.grad) and torch.equal(cap.accept, now.accept)
        assert (gr.float() - now.grad.float()).abs().max() <= 2.0 ** -8


def test_refusals_of_the_binding(gpu, ps):
    from paper_2603_19133_amd.training import distill_loss
    z, idx, prob, count = inputs(4, 100, 5, torch.float32, 1.0, 2)
    rec = record(ps, idx, prob, count)
    short = ps.Compressed(rec.idx[:3], rec.prob[:3], rec.count[:3], rec.mass, rec.lse, 5)
    f = ps.distill(z, 100, 1.0, rec)
    for call in (lambda: ps.distill(z, 100, 1.0, short), lambda: ps.distill(z[:, ::2], 50, 1.0, rec), lambda: ps.distill(z.cpu(), 100, 1.0, rec),
                 lambda: ps.distill(z, 100, 1.0, rec, weight=torch.ones(3, device="cuda")), lambda: ps.distill(z.half(), 100, 1.0, rec),
                 lambda: ps.distill(z, 100, 0.0, rec), lambda: ps.distill(z, 101, 1.0, rec),
                 lambda: ps.distill_grad(z, 100, 1.0, rec, f.stats, out=torch.empty(4, 100, dtype=torch.bfloat16, device="cuda")),
                 lambda: ps.distill_grad(z, 100, 1.0, rec, f.stats, out=torch.empty(4, 99, device="cuda")),
                 lambda: ps.distill_grad(z, 100, 1.0, rec, f.stats[:2]),
                 lambda: distill_loss(z, short, 100, 1.0), lambda: distill_loss(z[:, ::2], rec, 50, 1.0), lambda: distill_loss(z.half(), rec, 100, 1.0),
                 lambda: distill_loss(z, rec, 101, 1.0), lambda: distill_loss(z, rec, 100, 0.0), lambda: distill_loss(z, rec, 100, 1.0, tail=2)):
        with pytest.raises(ps.PicoSpecError):
            call()
    torch.cuda.synchronize()


def test_records_that_are_not_the_rows_are_refused(gpu, ps):
    """Arrays with gaps, of another length, type or place: each is an error of both entry points, before anything runs."""
    from paper_2603_19133_amd.training import distill_loss
    z, idx, prob, count = inputs(6, 100, 8, torch.float32, 1.0, 2)
    rec = record(ps, idx, prob, count)
    of = lambda **kw: ps.Compressed(**{**dict(idx=rec.idx, prob=rec.prob, count=rec.count, mass=rec.mass, lse=rec.lse, k=8), **kw})       # noqa: E731
    bad = [of(idx=rec.idx[:, :5], prob=rec.prob[:, :5], k=5), of(k=5), of(k=9), of(prob=rec.prob[:, :5]), of(prob=rec.prob[:3]), of(count=rec.count[:3]),
           of(idx=rec.idx.long()), of(prob=rec.prob.double()), of(count=rec.count.long()), of(idx=rec.idx.cpu()), of(count=rec.count.cpu()),
           of(prob=torch.rand(8, 6, device="cuda").t())]
    for r in bad:
        with pytest.raises(ps.PicoSpecError):
            ps.distill(z, 100, 1.0, r)
        with pytest.raises(ps.PicoSpecError):
            distill_loss(z, r, 100, 1.0)
    stats = ps.distill(z, 100, 1.0, rec).stats
    for kw in (dict(weight=torch.ones(6)), dict(weight=torch.ones(12, device="cuda")[::2])):
        with pytest.raises(ps.PicoSpecError):
            ps.distill_grad(z, 100, 1.0, rec, stats, **kw)
    for s in (stats.cpu(), torch.zeros(6, 8, dtype=torch.float64, device="cuda")[:, ::2]):
        with pytest.raises(ps.PicoSpecError):
            ps.distill_grad(z, 100, 1.0, rec, s)
    torch.cuda.synchronize()
