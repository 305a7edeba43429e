"""picospec_sample against the definition in 64 bits: tokens and counts equal, probabilities and log masses within their rounding.

A weight is off by at most 1.1e-12 (the polynomial) + 60 * 2^-52 (the exponent's rounding), so masses, and what is compared with them, by 2e-12:
a token or an end of a prefix differs from the definition only where a border lies within that of a step of the sum, one draw in a
million.  prob: 4e-12 and half a step of fp32; lse: the same of its value and 4e-12."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

FAR = 4e-12


@pytest.fixture(scope="module")
def ps():
    from paper_2603_19133_amd import binding
    return binding


def reference(z, T, top_k, top_p, min_p, u):
    """One row: (tok, prob, count, lse)."""
    z = z.astype(np.float64).copy()
    z[np.isnan(z)] = -np.inf
    z = np.minimum(z, float(np.finfo(np.float32).max))
    if z.max() == -np.inf:
        return -1, 0.0, 0, -np.inf
    T, top_p, min_p = (float(np.float32(v)) for v in (T, top_p, min_p))
    if T == 0:
        T, top_k = 1.0, 1
    order = np.argsort(-z, kind="stable")
    order = order[z[order] > -np.inf]
    if top_k > 0:
        order = order[:top_k]
    w = np.exp((z[order] - z.max()) / T)
    if 0 < top_p < 1:
        mass = np.cumsum(w)
        n = 1 + int(np.searchsorted(mass, top_p * mass[-1], side="left"))
        order, w = order[:n], w[:n]
    if min_p > 0:
        order, w = order[w >= min_p], w[w >= min_p]
    byid = np.argsort(order)
    mass = np.cumsum(w[byid])
    at = min(int(np.searchsorted(mass, float(np.float32(u)) * mass[-1], side="right")), len(order) - 1)
    return int(order[byid][at]), w[byid][at] / mass[-1], len(order), z.max() / T + math.log(mass[-1])


def compare(got, z, T, top_k, top_p, min_p, u):
    torch.cuda.synchronize()
    tok, prob, count, lse = (t.cpu().numpy() for t in (got.tok, got.prob, got.count, got.lse))
    z, u = z.float().cpu().numpy(), u.cpu().numpy()
    rows = len(tok)
    col = lambda v: v.cpu().numpy() if isinstance(v, torch.Tensor) else np.full(rows, v)
    T, top_k, top_p, min_p = col(T), col(top_k), col(top_p), col(min_p)
    for r in range(rows):
        want = reference(z[r], T[r], int(top_k[r]), top_p[r], min_p[r], u[r])
        where = (r, float(T[r]), int(top_k[r]), float(top_p[r]), float(min_p[r]), float(u[r]))
        assert (int(tok[r]), int(count[r])) == (want[0], want[2]), (where, int(tok[r]), int(count[r]), want)
        half = float(np.finfo(np.float32).eps) / 2
        assert abs(float(prob[r]) - want[1]) <= want[1] * (half + FAR) + 1e-44, (where, float(prob[r]), want)
        with np.errstate(over="ignore"):                          # (a log mass beyond fp32's range rounds to infinity)
            rounded = np.float32(want[3])
        assert lse[r] == rounded or abs(float(lse[r]) - want[3]) <= abs(want[3]) * half * (1 + 2.0 ** -20) + FAR, (where, float(lse[r]), want)


def rows_of(n, V, dtype, kind, seed, pad=0, shift=0):
    """[n, V] device logits, a view off any boundary."""
    rng = np.random.default_rng(seed)
    if kind == "normal":
        z = rng.normal(size=(n, V)) * 3
    elif kind == "flat":
        z = rng.normal(size=(n, V)) * 0.5 - 1.2 * np.log(np.floor(rng.random((n, V)) * V) + 1.0)
    elif kind == "trend":                                          # (frequent tokens at low ids)
        z = rng.normal(size=(n, V)) - 1.1 * np.log(np.arange(V) + 1.0)
    elif kind == "grid":                                           # (few values: many ties)
        z = np.round(rng.normal(size=(n, V)) * 2) / 2
    elif kind == "const":
        z = np.full((n, V), -2.5)
    flat = torch.zeros(n * (V + pad) + shift, dtype=dtype, device="cuda")
    out = flat[shift:].view(n, V + pad)[:, :V]
    out.copy_(torch.from_numpy(z).to(dtype))
    return out, torch.from_numpy(rng.random(n).astype(np.float32)).cuda()


SETTINGS = [dict(), dict(T=0.0), dict(T=0.7, top_k=1), dict(T=0.8, top_k=50, top_p=0.95), dict(top_p=0.9), dict(T=0.6, top_p=0.5, min_p=0.01),
            dict(T=1.2, min_p=0.1), dict(top_k=700), dict(top_k=700, min_p=0.02), dict(T=1.5, top_k=300, top_p=0.8, min_p=0.05), dict(top_p=1.0, min_p=1.0),
            dict(top_k=5000, top_p=0.99), dict(T=100.0, top_p=0.3), dict(T=0.01), dict(top_p=1e-6)]


@pytest.mark.parametrize("setting", SETTINGS, ids=lambda s: ",".join(f"{k}={v}" for k, v in s.items()) or "plain")
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,V,kind,pad,shift", [
    (3, 1, "normal", 0, 0), (4, 2, "grid", 1, 1), (5, 9, "normal", 0, 3), (6, 1023, "grid", 2, 1), (4, 4096, "normal", 0, 0), (5, 5003, "flat", 1, 5),
    (3, 32000, "normal", 0, 0), (4, 50001, "flat", 2, 1), (2, 50001, "grid", 0, 0), (2, 40000, "trend", 0, 0), (2, 33333, "const", 3, 0),
    (2, 152064, "flat", 0, 0), (2, 151936, "normal", 5, 0),
], ids=str)
def test_against_the_definition(gpu, ps, rows, V, kind, pad, shift, dtype, setting):
    print(f"[case] sample rows={rows} V={V} {kind} pad={pad} shift={shift} {dtype} {setting}", flush=True)
    z, u = rows_of(rows, V, dtype, kind, rows * 100003 + V, pad, shift)
    s = dict(dict(T=1.0, top_k=0, top_p=0.0, min_p=0.0), **setting)
    got = ps.sample(z, V, u, temperature=s["T"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
    compare(got, z, s["T"], s["top_k"], s["top_p"], s["min_p"], u)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(24, 20001), (96, 33000), (300, 8200)])
def test_settings_per_row(gpu, ps, rows, V, dtype):
    """Every row with its own settings, greedy ones among them, and the ones that count as something else."""
    print(f"[case] sample per row {rows} x {V} {dtype}", flush=True)
    rng = np.random.default_rng(rows)
    z, u = rows_of(rows, V, dtype, "flat", rows)
    d = lambda a, t: torch.from_numpy(np.asarray(a).astype(t)).cuda()
    T = d(rng.choice([0.0, 0.6, 0.9, 1.3], rows), np.float32)
    k = d(rng.choice([0, -4, 1, 50, 900, 4097], rows), np.int32)
    p = d(rng.choice([0.0, -1.0, 0.5, 0.9, 1.0, 2.0], rows), np.float32)
    m = d(rng.choice([0.0, -1.0, 0.05, 1.0], rows), np.float32)
    compare(ps.sample(z, V, u, temperature=T, top_k=k, top_p=p, min_p=m), z, T, k, p, m, u)
    got = ps.sample(z, V, u, temperature=torch.full_like(T, math.nan), top_k=k, top_p=torch.full_like(p, math.nan), min_p=torch.full_like(m, 7.0))
    compare(got, z, 0.0, 1, 0.0, 1.0, u)


@pytest.mark.parametrize("setting", [dict(), dict(top_k=40), dict(top_p=0.9), dict(min_p=0.05), dict(top_k=3000, top_p=0.97)], ids=str)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [37, 9001, 70001])
def test_masks_and_odd_values(gpu, ps, V, dtype, setting):
    """Rows masked with -inf and with the type's lowest value, one that is masked whole, NaN and +inf, one id, all ids equal to the lowest value."""
    print(f"[case] sample masks V={V} {dtype} {setting}", flush=True)
    z, u = rows_of(12, V, dtype, "normal", V, 1, 1)
    rng = np.random.default_rng(V)
    off = torch.from_numpy(rng.random((12, V)) < 0.875).cuda()
    low = torch.finfo(dtype).min
    z[0] = torch.where(off[0], torch.full_like(z[0], -math.inf), z[0])
    z[1] = torch.where(off[1], torch.full_like(z[1], low), z[1])
    z[2] = -math.inf
    z[3] = math.nan
    z[4, V // 2] = math.nan
    z[5, V // 3] = math.inf
    z[6, V // 3], z[6, V - 1] = math.inf, math.inf
    z[7] = -math.inf
    z[7, V - 1] = -3.0
    z[8] = low
    z[9] = 0.0
    z[9, ::2] = -0.0                                               # (they tie)
    z[10] *= 1000.0
    z[11] = torch.where(off[11], torch.full_like(z[11], math.nan), z[11])
    s = dict(dict(top_k=0, top_p=0.0, min_p=0.0), **setting)
    compare(ps.sample(z, V, u, temperature=0.9, **s), z, 0.9, s["top_k"], s["top_p"], s["min_p"], u)


@pytest.mark.parametrize("setting", [dict(), dict(top_k=50, top_p=0.9), dict(top_k=1000), dict(top_k=4000), dict(top_p=0.9), dict(top_p=0.9, min_p=0.02), dict(min_p=0.02)], ids=str)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("kind", ["normal", "trend"])
def test_the_longest_rows(gpu, ps, kind, dtype, setting):
    print(f"[case] sample longest {kind} {dtype} {setting}", flush=True)
    V = 1 << 20
    z, u = rows_of(2, V, dtype, kind, 6, 1, 1)
    s = dict(dict(top_k=0, top_p=0.0, min_p=0.0), **setting)
    compare(ps.sample(z, V, u, **s), z, 1.0, s["top_k"], s["top_p"], s["min_p"], u)


@pytest.mark.parametrize("top_k,top_p,min_p", [(0, 0.0, 0.0), (50, 0.9, 0.0), (900, 0.9, 0.0), (0, 0.9, 0.0), (0, 0.0, 0.05)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_spread_rows_are_the_unspread_ones(gpu, ps, dtype, top_k, top_p, min_p):
    """With scratch, without it and with too little of it: the same tokens and counts (masses are summed in another order: probabilities to their rounding)."""
    print(f"[case] sample spread {dtype} {top_k} {top_p} {min_p}", flush=True)
    rows, V = 9, 60007
    z, u = rows_of(rows, V, dtype, "normal", 44)
    got = ps.sample(z, V, u, temperature=0.7, top_k=top_k, top_p=top_p, min_p=min_p)
    need = ps.scratch_bytes(ps.CALL_SAMPLE, ps.F32 if dtype == torch.float32 else ps.BF16, rows, 0, V, 0)
    assert need > 0 and need == ps.workspace_bytes(ps.CALL_SAMPLE, ps.F32 if dtype == torch.float32 else ps.BF16, rows, V, 0)
    for size in (0, need - 1):
        ws = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
        o = ps.Sampled(torch.zeros_like(got.tok), torch.zeros_like(got.prob), torch.zeros_like(got.count), torch.zeros_like(got.lse))
        assert ps.lib.picospec_sample(z.data_ptr(), 0 if dtype == torch.float32 else 1, V, rows, V, 0.7, top_k, top_p, min_p, None, None, None, None, u.data_ptr(), o.tok.data_ptr(),
                                      o.prob.data_ptr(), o.count.data_ptr(), o.lse.data_ptr(), ws.data_ptr() if size else None, size, None) == ps.OK
        torch.cuda.synchronize()
        assert torch.equal(o.tok, got.tok) and torch.equal(o.count, got.count)
        assert torch.allclose(o.prob, got.prob, rtol=2.0 ** -23, atol=0.0) and torch.allclose(o.lse, got.lse, rtol=2.0 ** -23, atol=0.0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows", [6, 270])
@pytest.mark.parametrize("top_p,min_p", [(0.9, 0.014), (0.9, 0.0), (0.5, 0.2), (0.99, 0.001), (0.97, 0.3)])
def test_few_ids_far_above_the_rest(gpu, ps, top_p, min_p, rows, dtype):
    """Rows whose largest logits lie far above the rest, at ids that a sample of the row may or may not hold: one to three of them have about 90 % of the mass."""
    print(f"[case] sample outliers rows={rows} {dtype} top_p={top_p} min_p={min_p}", flush=True)
    V = 40003
    z, u = rows_of(rows, V, dtype, "normal", 12)
    z.mul_(0.3).sub_(3.0)
    rng = np.random.default_rng(31)
    for r in range(rows):
        at = rng.choice(V, 3, replace=False)
        z[r, int(at[0])] = 10.0
        z[r, int(at[1])] = float(rng.choice([6.25, 8.0, 9.5]))
        z[r, int(at[2])] = float(rng.choice([-3.0, 5.0, 7.5]))
    compare(ps.sample(z, V, u, top_p=top_p, min_p=min_p), z, 1.0, 0, top_p, min_p, u)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(7, 60001), (56, 40000), (280, 20000)])
def test_min_p_near_the_end_of_a_prefix(gpu, ps, rows, V, dtype):
    """Spread rows whose min-p lies a little above, at, or below the weight of the last entry that top-p keeps."""
    z, u = rows_of(rows, V, dtype, "flat", 77 + rows)
    v = torch.sort(z.double(), dim=1, descending=True).values
    w = torch.exp(v - v[:, :1])
    mass = torch.cumsum(w, 1)
    end = torch.gather(w, 1, (mass < 0.9 * mass[:, -1:]).sum(1, keepdim=True))[:, 0]
    factor = torch.tensor([0.25, 0.9, 0.985, 0.9999, 1.0001, 1.015, 1.1, 4.0], dtype=torch.float64, device=z.device)
    min_p = (end * factor[torch.arange(rows, device=z.device) % 8]).float()
    compare(ps.sample(z, V, u, top_p=0.9, min_p=min_p), z, 1.0, 0, 0.9, min_p, u)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("top,T", [(17.25, 0.6), (16.0, 0.05), (33.5, 0.6), (300.0, 0.6), (1e30, 0.6)])
@pytest.mark.parametrize("rows,V", [(3, 30000), (40, 17001), (270, 9001)])
def test_one_id_above_the_octave_of_the_others(gpu, ps, rows, V, top, T, dtype):
    """A row's largest logit, at a place that a glance at the row may miss, lies one octave of magnitude or many above what the others reach."""
    z, u = rows_of(rows, V, dtype, "normal", 5 + rows)
    z.copy_((z.float() * 1.4).clamp(max=15.75).to(dtype))
    at = torch.randint(0, V, (rows,), device="cuda", generator=torch.Generator("cuda").manual_seed(3))
    z[torch.arange(rows, device="cuda"), at] = top
    for top_p in (0.3, 0.95):
        compare(ps.sample(z, V, u, temperature=T, top_p=top_p), z, T, 0, top_p, 0.0, u)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,V,T,min_p", [(2, 100001, 1.0, 1e-3), (30, 40000, 3.0, 1e-3), (270, 20001, 3.0, 1e-4)])
def test_min_p_that_keeps_thousands(gpu, ps, rows, V, T, min_p, dtype):
    z, u = rows_of(rows, V, dtype, "flat", rows)
    z[0, 5:9] = math.nan
    z[1, ::3] = -math.inf
    compare(ps.sample(z, V, u, temperature=T, min_p=min_p), z, T, 0, 0.0, min_p, u)


@pytest.mark.parametrize("top_p", [0.0, 0.9])
def test_the_ends_of_the_uniforms(gpu, ps, top_p):
    """u = 0 draws the first kept id, the largest u below 1 the last; outside [0, 1): the first and the last."""
    print("[case] sample ends", flush=True)
    z, _ = rows_of(6, 30011, torch.float32, "normal", 4)
    z[:] = z[0]
    u = torch.tensor([0.0, 1.0 - 2.0 ** -24, -0.5, math.nan, 1.0, 3.0], device="cuda")
    got = ps.sample(z, 30011, u, top_p=top_p)
    compare(ps.sample(z[:2], 30011, u[:2], top_p=top_p), z[:2], 1.0, 0, top_p, 0.0, u[:2])
    tok = got.tok.cpu().tolist()
    assert tok[2] == tok[0] and tok[3] == tok[0] and tok[4] == tok[5] and tok[4] >= tok[1]


def test_draws_follow_the_distribution(gpu, ps):
    """4096 draws of one row of 50 ids, at evenly spaced uniforms: frequencies are the probabilities to one and a half draws."""
    print("[case] sample frequencies", flush=True)
    z, _ = rows_of(1, 50, torch.float32, "normal", 8)
    n = 4096
    u = torch.from_numpy(((np.arange(n) + 0.5) / n).astype(np.float32)).cuda()
    got = ps.sample(z.expand(n, 50).contiguous(), 50, u, temperature=1.5)
    torch.cuda.synchronize()
    p = np.exp(z[0].double().cpu().numpy() / 1.5)
    p /= p.sum()
    seen = np.bincount(got.tok.cpu().numpy(), minlength=50) / n
    assert np.abs(seen - p).max() <= 1.5 / n                        # (both ends of an id's share fall between two uniforms)


def test_same_bits_streams_and_graph(gpu, ps):
    print("[case] sample stream and graph", flush=True)
    for rows, V, s in ((3, 20001, dict(top_k=40, top_p=0.9)), (5, 70001, dict(top_p=0.9)), (2, 33001, dict())):
        z, u = rows_of(rows, V, torch.bfloat16, "flat", 3)
        want = ps.sample(z, V, u, **s)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = ps.sample(z, V, u, **s)
        side.synchronize()
        same = lambda a, b: all(torch.equal(x, y) for x, y in ((a.tok, b.tok), (a.prob, b.prob), (a.count, b.count), (a.lse, b.lse)))
        assert same(got, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cap = ps.sample(z, V, u, **s)
        for i in range(3):
            z.copy_(torch.randn_like(z) * (1 + i))
            u.copy_(torch.rand_like(u))
            graph.replay()
            torch.cuda.synchronize()
            now = ps.sample(z, V, u, **s)
            torch.cuda.synchronize()
            assert same(cap, now)


def test_refusals_of_the_binding(gpu, ps):
    z, u = rows_of(4, 100, torch.float32, "normal", 1)
    f = lambda *v: torch.tensor(v, device="cuda")
    for call in (lambda: ps.sample(z, 100, u[:3]), lambda: ps.sample(z, 100, u.double()), lambda: ps.sample(z, 100, u.cpu()), lambda: ps.sample(z, 101, u), lambda: ps.sample(z[:, ::2], 50, u),
                 lambda: ps.sample(z.half(), 100, u), lambda: ps.sample(z, 100, u, temperature=-1.0), lambda: ps.sample(z, 100, u, min_p=2.0),
                 lambda: ps.sample(z, 100, u, temperature=f(1.0, 1.0, 1.0)), lambda: ps.sample(z, 100, u, top_k=f(1.0, 1.0, 1.0, 1.0)),
                 lambda: ps.sample(z, 100, u, top_p=u.cpu())):
        with pytest.raises(ps.PicoSpecError):
            call()
    torch.cuda.synchronize()
