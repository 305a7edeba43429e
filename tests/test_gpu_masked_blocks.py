"""Vocabularies of which whole stretches are masked with a finite value, of which fp32 holds steps of hundreds: what a thread, a wave, a segment or a workgroup's share
of a row sees may be masked altogether, and its reference exponent is then the mask's."""
import dataclasses

import numpy as np
import pytest
import torch

import parity_util as pu
from paper_2603_19133_amd import workloads as W

pytestmark = pytest.mark.gpu

LOW = [-1e9, -1e10, -1e20, -1e30, None]


@pytest.fixture(scope="module")
def ps():
    from paper_2603_19133_amd import binding
    return binding


def _rows(n, V, dtype, low, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    z = torch.randn(n, V, device="cuda", generator=g) * 3
    m = torch.zeros(n, V, dtype=torch.bool, device="cuda")
    m[0::5, : V // 2] = True
    m[1::5, V // 2:] = True
    m[2::5, V // 3: 2 * V // 3] = True
    m[3::5] = True
    m[3::5, V // 2: V // 2 + 500] = False
    m[4::5, : V - 300] = True
    return torch.where(m, torch.full_like(z, torch.finfo(dtype).min if low is None else low), z).to(dtype)


def _close(got, want, rtol, what, atol=0.0):
    assert np.isfinite(got).all(), what                            # (a comparison with NaN is no failure by itself)
    pu.assert_close(got, want, rtol, what, atol)


SHAPES = [(5, 700), (5, 9001), (5, 70001), (60, 40003), (300, 9001), (300, 40003)]
TEMPERATURES = [1.0, 0.7, 2.0]


@pytest.mark.parametrize("low", LOW, ids=str)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T", TEMPERATURES)
def test_row_statistics(gpu, ps, T, dtype, low):
    for n, V in SHAPES:
        print(f"[case] row_stats {n} x {V} {dtype} T={T} {low}", flush=True)
        z = _rows(n, V, dtype, low, n + V)
        want = torch.logsumexp(z.double() / float(np.float32(T)), 1).cpu().numpy()
        mx, sm, lse = ps.row_stats(z, V, T)
        _close(pu.n(lse), want, pu.RTOL_LSE, "lse", atol=1e-6)
        _close(pu.n(mx) / T + np.log(pu.n(sm).astype(np.float64)), want, pu.RTOL_LSE, "max, sum", atol=1e-6)


@pytest.mark.parametrize("low", LOW, ids=str)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T", TEMPERATURES)
def test_records(gpu, ps, T, dtype, low):
    for n, V in SHAPES:
        z = _rows(n, V, dtype, low, n + V)
        y = z.double() / float(np.float32(T))
        want = torch.logsumexp(y, 1)
        for k in (10, 64, 200):
            print(f"[case] compress {n} x {V} k={k} {dtype} T={T} {low}", flush=True)
            c = ps.compress(z, V, T, k)
            assert torch.equal(c.idx.long(), torch.sort(z.double(), dim=1, descending=True, stable=True).indices[:, :k]) and (c.count == k).all()
            _close(pu.n(c.lse), want.cpu().numpy(), pu.RTOL_LSE, "lse", atol=1e-6)
            _close(pu.n(c.prob), torch.exp(y.gather(1, c.idx.long()) - want[:, None]).cpu().numpy(), pu.RTOL, "prob", atol=1e-37)


@pytest.mark.parametrize("low,T", [(-1e10, 1.0), (-1e20, 0.7), (None, 2.0)], ids=str)
@pytest.mark.parametrize("name,scale", [("cfg1", {}), ("cfg2", {"B": 4, "V": 9001}), ("cfg3", {"B": 6, "V": 40003, "k": 200}), ("cfg5", {"B": 60, "V": 20011, "k": 300}),
                                        ("cfg4", {"B": 12, "V": 50021, "k": 500})], ids=str)
def test_rounds(gpu, ps, name, scale, low, T):
    """A round whose draft and target rows are masked in blocks, by its separate calls and as one, with and without the target rows' segment table."""
    print(f"[case] round {name} {scale} {low} T={T}", flush=True)
    w = dataclasses.replace(W.WORKLOADS[name].scaled(**scale), T=T)
    r = W.build_round(w)
    dtype = torch.float32 if w.dtype == "f32" else torch.bfloat16
    fill = np.float32(torch.finfo(dtype).min if low is None else low)
    fill = fill if w.dtype == "f32" else W.to_bf16_bits(np.array([fill], np.float32))[0]
    for a in (r.draft_logits, r.tgt_logits):
        a[:, : w.V // 2] = fill
        a[1::2, 3 * w.V // 4:] = fill
        a[2::3, w.V // 2: w.V // 2 + w.V // 8] = fill
    o = pu.oracle_round(r)

    def compare(g):
        assert all(torch.isfinite(t.float()).all() for t in (g.q.prob, g.q.mass, g.q.lse, g.ver.p_tok, g.ver.q_tok, g.ver.tgt_max, g.ver.tgt_sum, g.ver.tgt_lse, g.res.resid_mass))
        pu.compare_round(g, o, r, max_excluded_frac=0.34)
    for seg in (False, True):
        compare(pu.gpu_round(r, o.tok, gpu, seg=seg))
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(gpu)                                # noqa: E731
    for ws in (None, ps.alloc_workspace(dtype, r.N + r.B, w.V, gpu, ps.CALL_ROUND)):
        q, ver, res = ps.round(pu.to_device(r.draft_logits, gpu), pu.to_device(r.tgt_logits, gpu), w.V, w.T, d(r.seq_off), r.N, d(o.tok), w.k, d(r.uniforms), top_p=w.top_p,
                               workspace=ws)
        compare(pu.GpuRound(q, ver, res))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("at,T", [(0.0, 1.0), (-60.0, 1.0), (-75.0, 1.0), (-100.0, 1.0), (-1e4, 1.0), (-9.0, 0.05), (100.0, 1.0)], ids=str)
def test_records_of_few_allowed_ids_of_low_value(gpu, ps, at, T, dtype):
    """A vocabulary mask (-inf) that leaves a stretch of some ids, none of which a look at the row meets, with logits far below 0."""
    for n, V, k, allowed in ((3, 12331, 19, 20), (8, 128256, 50, 400), (300, 40003, 64, 20), (300, 40003, 300, 200), (256, 128256, 1024, 700)):
        print(f"[case] compress {n} x {V} k={k} {allowed} allowed {dtype} at {at} T={T}", flush=True)
        rng = np.random.default_rng(V + k)
        z = torch.full((n, V), -np.inf, dtype=dtype, device="cuda")
        z[:, V // 2: V // 2 + allowed] = torch.from_numpy(rng.normal(size=(n, allowed)) * 3 * T + at).to(dtype).cuda()
        y = z.double() / float(np.float32(T))
        want = torch.logsumexp(y, 1)
        c = ps.compress(z, V, T, k)
        m = min(k, allowed)
        assert torch.equal(c.idx[:, :m].long(), torch.sort(z.double(), dim=1, descending=True, stable=True).indices[:, :m])
        # (what fp32 holds of the exponents of values at -10^4: 2^-24 of 14427 each)
        far = abs(at) / T * 2.0 ** -24
        _close(pu.n(c.lse), want.cpu().numpy(), pu.RTOL_LSE, "lse", atol=1e-6 + far)
        _close(pu.n(c.prob[:, :m]), torch.exp(y.gather(1, c.idx[:, :m].long()) - want[:, None]).cpu().numpy(), pu.RTOL + far, "prob", atol=1e-37)


def test_a_row_of_low_values_keeps_its_nan(gpu, ps):
    z = torch.full((300, 40003), -np.inf, device="cuda")
    z[:, 20000:20020] = -200.0 + torch.arange(20, device="cuda")
    want = ps.compress(z, 40003, 1.0, 64)
    z[7, 30000] = float("nan")
    got = ps.compress(z, 40003, 1.0, 64)
    torch.cuda.synchronize()
    assert torch.isnan(got.lse[7]) and torch.isfinite(want.lse).all()
    keep = torch.arange(300, device="cuda") != 7
    assert torch.equal(got.lse[keep], want.lse[keep]) and torch.equal(got.prob[keep], want.prob[keep])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,V,k,block", [(30, 199536, 1516, 64), (30, 199536, 1516, 256), (30, 199536, 1400, 256), (60, 151936, 1000, 64), (60, 100003, 700, 256), (90, 128256, 900, 64)])
def test_full_lists(gpu, ps, n, V, k, block, dtype):
    """Rows of which every other block of ids is masked: half of a workgroup's lanes hold nothing, the others more than their share, and some of the lists that the
    workgroups of a row leave are full to the last place."""
    print(f"[case] full lists {n} x {V} k={k} blocks of {block} {dtype}", flush=True)
    g = torch.Generator("cuda").manual_seed(24526895)
    z = torch.randn(n, V, device="cuda", generator=g) * 6.77 + 100
    z = torch.where(torch.arange(V, device="cuda") // block % 2 == 0, torch.full_like(z, -np.inf), z).to(dtype)
    want = torch.sort(z.double(), dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(ps.compress(z, V, 1.0, k).idx.long(), want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,V,k,allowed,values,at", [(56, 142226, 12, 400, "two", 0.0), (56, 142226, 64, 400, "one", 5.0), (64, 131072, 64, 400, "one", 5.0), (8, 51528, 25, 5000, "normal", 1e4),
                                                     (64, 22807, 112, 7000, "normal", -1e4), (300, 40003, 64, 400, "one", 5.0), (300, 128256, 3000, 7000, "two", 0.0)])
def test_ties_among_allowed_ids(gpu, ps, n, V, k, allowed, values, at, dtype):
    """A stretch of allowed ids of few values: more entries of one value than a list holds, of which the lowest ids are kept."""
    print(f"[case] ties {n} x {V} k={k} {allowed} {values} {dtype}", flush=True)
    for seed in range(4):
        g = torch.Generator("cuda").manual_seed(seed)
        t = torch.randn(n, allowed, device="cuda", generator=g)
        t = {"two": torch.where(t > 0, 0.22, -0.22), "one": torch.zeros_like(t), "normal": t * 0.3}[values] + at
        z = torch.full((n, V), -np.inf, dtype=dtype, device="cuda")
        z[:, V // 2: V // 2 + allowed] = t.to(dtype)
        want = torch.sort(z.double(), dim=1, descending=True, stable=True).indices[:, :k]
        for _ in range(2):
            assert torch.equal(ps.compress(z, V, 1.0, k).idx.long(), want)
