"""picospec_clip_grad against the formula in 64 bits.

The norm's squares are summed in 64 bits, so it is off by half a step of fp32 (and some 2^-40).  Factor and products are formed in 64 bits and rounded to fp32, 2^-24, and bf16
tensors from there once more."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

OFF = {torch.float32: 2.0 ** -24 * (1 + 2.0 ** -10), torch.bfloat16: 2.0 ** -8 + 2 * 2.0 ** -24}


@pytest.fixture(scope="module")
def ps():
    from paper_2603_19133_amd import binding
    return binding


def _grads(gpu, shapes, seed=0, scale=1e-2):
    g = torch.Generator(device=gpu).manual_seed(seed)
    kinds = (torch.float32, torch.bfloat16)
    return [(torch.randn(s, device=gpu, generator=g) * scale).to(kinds[(i + seed) % 2]) for i, s in enumerate(shapes)]


def _norm(grads):
    return math.sqrt(math.fsum(float((g.double() ** 2).sum()) for g in grads))


def _check(ps, grads, max_norm, out=None):
    before = [g.clone() for g in grads]
    want = _norm(before)
    factor = min(1.0, torch.tensor(max_norm, dtype=torch.float32).item() / (want + 1e-6))           # (the limit reaches the library as fp32)
    norm = ps.clip_grad(grads, max_norm, out)
    assert norm.shape == (1,) and abs(norm.item() - want) <= want * (2.0 ** -24 + 2.0 ** -36) + 2.0 ** -149
    for g, b, o in zip(grads, before, out or grads):
        if out:
            assert torch.equal(g, b)
        if factor == 1.0:
            assert torch.equal(o, b)
        else:
            ref = b.double() * factor
            tiny = 2.0 ** -149 if b.dtype == torch.float32 else 2.0 ** -133         # (a step of the smallest numbers)
            assert bool(((o.double() - ref).abs() <= OFF[b.dtype] * ref.abs() + tiny).all())


SHAPES = {
    "one": [(1,)],
    "scalar": [(), (3,)],
    "pair": [(4096, 24), (24, 4096)],
    "odd": [(7,), (333, 501), (0,), (1,), (16383,), (16384,), (16385,), (3, 5, 7)],
    "many": [(i % 37 + 1, 11) for i in range(300)],
    "large": [(5_000_001,), (3, 1_000_003)],
    "empty": [(0,), (4, 0)],
}


@pytest.mark.parametrize("name", SHAPES)
@pytest.mark.parametrize("max_norm", [0.5, 1e9, 0.0, float("inf")])
def test_clip(gpu, ps, name, max_norm):
    print(f"[case] clip {name} {max_norm}", flush=True)
    for seed in (0, 1):
        _check(ps, _grads(gpu, SHAPES[name], seed), max_norm)
        grads = _grads(gpu, SHAPES[name], seed)
        _check(ps, grads, max_norm, [torch.full_like(g, 7) for g in grads])


def test_no_tensors(gpu, ps):
    print("[case] clip none", flush=True)
    assert ps.clip_grad([], 1.0).item() == 0.0


def test_views_of_one_buffer(gpu, ps):
    print("[case] clip views", flush=True)
    for dtype in (torch.float32, torch.bfloat16):
        flat = torch.randn(100_003, device=gpu).to(dtype)
        sizes = [1, 2, 3, 17, 40_001, 255, 59_724]
        parts = list(flat.split(sizes))
        _check(ps, parts[1:-1], 0.3)                      # (what lies around them is not touched)
        keep = flat.clone()
        ps.clip_grad(parts[1:-1], 0.1)
        assert torch.equal(flat[:1], keep[:1]) and torch.equal(flat[sum(sizes[:-1]):], keep[sum(sizes[:-1]):])
    t = torch.randn(40, 30, device=gpu).t()               # (dense, in another order of its elements)
    _check(ps, [t], 0.3)
    _check(ps, [t], 0.3, [torch.zeros(40, 30, device=gpu).t()])


def test_large_and_small_values(gpu, ps):
    print("[case] clip values", flush=True)
    for v in (1e30, 3e38, 1e-30, 2.0 ** -149):
        g = torch.full((1000,), v, device=gpu)
        want = _norm([g])
        norm = ps.clip_grad([g], float("inf")).item()
        assert norm == float("inf") if want > 3.4028235e38 else abs(norm - want) <= want * 2.0 ** -24 * (1 + 2.0 ** -10) + 2.0 ** -150
    g = torch.full((1000,), 3e38, device=gpu)             # (a norm beyond fp32 still scales as it should)
    ps.clip_grad([g], 1.0)
    assert abs(g[0].item() - 1000 ** -0.5) <= 3 * 2.0 ** -24
    for bad, then in ((float("inf"), 0.0), (float("nan"), float("nan"))):
        g, h = torch.ones(100, device=gpu), torch.ones(50, device=gpu, dtype=torch.bfloat16)
        g[7] = bad
        norm = ps.clip_grad([g, h], 1.0).item()
        assert norm == bad if bad == math.inf else math.isnan(norm)
        assert all(x == then or (math.isnan(then) and math.isnan(x)) for x in h.tolist() + g.tolist()[:7]) and math.isnan(g[7].item())


def test_without_a_limit_nothing_is_scaled(gpu, ps):
    print("[case] clip without a limit", flush=True)
    g, to = torch.randn(5000, device=gpu), torch.zeros(5000, device=gpu)
    g[3] = float("inf")
    assert ps.clip_grad([g], float("inf"), [to]).item() == float("inf") and torch.equal(g, to)


def test_more_than_32_bits_of_elements(gpu, ps):
    print("[case] clip large offsets", flush=True)
    n = (1 << 31) + 5000
    g = torch.full((n,), 2.0 ** -10, dtype=torch.bfloat16, device=gpu)
    h = torch.ones(7, device=gpu)
    want = math.sqrt(n * 2.0 ** -20 + 7)
    assert abs(ps.clip_grad([g, h], 2.0 ** -10).item() - want) <= want * 2.0 ** -24 * (1 + 2.0 ** -10)
    ref = 2.0 ** -20 / (want + 1e-6)
    for part in (g[:9], g[n // 2:n // 2 + 9], g[-9:]):
        assert bool(((part.double() - ref).abs() <= OFF[torch.bfloat16] * ref).all())
    assert bool((g == g[0]).all())


def test_the_same_bits_every_time(gpu, ps):
    print("[case] clip twice", flush=True)
    grads = _grads(gpu, SHAPES["odd"] + SHAPES["large"])
    outs = [[torch.empty_like(g) for g in grads] for _ in range(2)]
    norms = [ps.clip_grad(grads, 0.1, o) for o in outs]
    assert torch.equal(*norms) and all(torch.equal(a, b) for a, b in zip(*outs))


def test_parameters(gpu, ps):
    print("[case] clip parameters", flush=True)
    from paper_2603_19133_amd import training
    a, b, c = (torch.nn.Parameter(torch.zeros(s, device=gpu)) for s in ((30, 20), (5,), (4,)))
    a.grad, b.grad = torch.randn(30, 20, device=gpu), torch.randn(5, device=gpu)
    want = _norm([a.grad, b.grad])
    assert abs(training.clip_grad_norm(iter([a, b, c]), 1.0).item() - want) <= want * 2.0 ** -23
    assert abs(_norm([a.grad, b.grad]) - 1.0) <= 1e-5
    assert abs(training.clip_grad_norm(b, 100.0).item() - _norm([b.grad])) <= 1e-6
    # what the tape has saved of a tensor that is then scaled is not what it was
    x = torch.randn(5, device=gpu, requires_grad=True)
    y = x * 1.0
    z = (y * y).sum()
    ps.clip_grad([y.detach()], 1e-3)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.backward()


def test_refusals(gpu, ps):
    print("[case] clip refusals", flush=True)
    a, b = torch.randn(100, device=gpu), torch.randn(50, device=gpu)
    for f in (lambda: ps.clip_grad([a, a], 1.0), lambda: ps.clip_grad([a, a[50:]], 1.0), lambda: ps.clip_grad([a, b], 1.0, [a, a[:50]]), lambda: ps.clip_grad([a], 1.0, [a, b]),
              lambda: ps.clip_grad([a, b], 1.0, [torch.empty_like(a), torch.empty_like(a)]), lambda: ps.clip_grad([a[::2]], 1.0), lambda: ps.clip_grad([b.expand(3, 50)], 1.0),
              lambda: ps.clip_grad([a], -1.0), lambda: ps.clip_grad([a], float("nan")), lambda: ps.clip_grad([a, b.cpu()], 1.0), lambda: ps.clip_grad([a.to_sparse()], 1.0),
              lambda: ps.clip_grad([a.view(10, 10)], 1.0, [torch.zeros(10, 10, device=gpu).t()])):
        with pytest.raises(ps.PicoSpecError) as e:
            f()
        assert e.value.code == ps.EINVAL
    for f in (lambda: ps.clip_grad([a.half()], 1.0), lambda: ps.clip_grad([a], 1.0, [a.bfloat16()])):
        with pytest.raises(ps.PicoSpecError) as e:
            f()
        assert e.value.code == ps.EDTYPE
