"""picospec_embed and picospec_embed_grad against the sums in 64 bits.

The gradient's sums are formed in fp32: k rows behind each other, or (k of 64 and more, tokens of more than 1024 positions in all) in pieces of 32 and up to k / 128 rows, at most 128 of them, or
in up to 32 parts.  So a sum of k rows is off by less than (min(k, 127) + k / 64) 2^-24 of the sum of absolute values; the factor rounds once more, the result to the table's type once (an added table: the sum with it, too)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module")
def ps():
    from paper_2603_19133_amd import binding
    return binding


def _tokens(n, V, seed, how):
    g = torch.Generator().manual_seed(seed)
    if how == "spread":
        return torch.randint(0, V, (n,), generator=g, dtype=torch.int32)
    if how == "one":
        return torch.full((n,), V - 1, dtype=torch.int32)
    if how == "none":
        return torch.full((n,), -1, dtype=torch.int32)
    if how == "runs":                                   # (tokens of 1, 2, 3, .. positions, pieces' ends among them)
        t = torch.repeat_interleave(torch.arange(1000, dtype=torch.int32), torch.arange(1000))[:n] % V
        return t[torch.randperm(n, generator=g)]
    if how == "edges":                                  # (127, 128, 129, 191, 192 positions behind each other)
        t = torch.cat([torch.full((k,), v, dtype=torch.int32) for v, k in enumerate([127, 128, 129, 1, 191, 192, 193, 63, 64, 65])])
        return t[torch.randperm(t.numel(), generator=g)] % V
    t = (torch.exp(torch.rand(n, generator=g) * torch.log(torch.tensor(V + 1.0))) - 1).to(torch.int32).clamp(0, V - 1)
    t[torch.rand(n, generator=g) < 0.2] = -1
    t[torch.rand(n, generator=g) < 0.02] = V            # (behind the table)
    return t


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,V,d", [(1, 1, 1), (1, 50, 64), (7, 1000, 33), (300, 5000, 501), (1000, 32000, 1024), (33, 100, 5000), (5, 3, 20011)])
def test_embed(gpu, ps, n, V, d, dtype):
    print(f"[case] embed {n} {V} {d} {dtype}", flush=True)
    g = torch.Generator(device=gpu).manual_seed(n)
    whole = torch.randn((V, d + 3), device=gpu, generator=g).to(dtype)
    tok = _tokens(n, V, 5, "zipf").to(gpu)
    there = ((tok >= 0) & (tok < V)).unsqueeze(1)
    for table in (whole[:, :d], whole[:, :d].contiguous()):
        rows = table[tok.clamp(0, V - 1).long()]
        assert torch.equal(ps.embed(table, tok), torch.where(there, rows, 0))
        for scale in (0.0, -1.0, 3.7):
            s = float(torch.tensor(scale, dtype=torch.float32))
            want = torch.where(there, rows.double() * s, 0.0)
            bound = (HALF[dtype] + (2.0 ** -24 if dtype == torch.bfloat16 else 0.0)) * (1 + 2.0 ** -20) * want.abs()
            assert bool(((ps.embed(table, tok, scale).double() - want).abs() <= bound).all())
    room = torch.full((n, d + 5), 9.0, dtype=dtype, device=gpu)
    ps.embed(table, tok, out=room[:, :d])
    assert torch.equal(room[:, :d], torch.where(there, rows, 0)) and bool((room[:, d:] == 9).all())


def test_embed_takes_tokens_of_any_shape(gpu, ps):
    print("[case] embed shapes", flush=True)
    table = torch.randn(50, 12, device=gpu)
    tok = torch.randint(0, 50, (3, 4, 5), device=gpu, dtype=torch.int32)
    assert torch.equal(ps.embed(table, tok), table[tok.long()])
    assert torch.equal(ps.embed(table, tok[0, 0, 0]), table[tok[0, 0, 0].long()])
    assert ps.embed(table, tok[:0]).shape == (0, 4, 5, 12)
    big = torch.full((4,), float("nan"), device=gpu).view(2, 2)
    assert ps.embed(big, torch.tensor([1, -1], dtype=torch.int32, device=gpu), 2.0).isnan().tolist() == [[True, True], [False, False]]


def _expect(grad, tok, V, scale, old=None):
    """(sums, their bound without the last rounding) in 64 bits."""
    there = (tok >= 0) & (tok < V)
    g = grad.double()[there]
    at = tok[there].long()
    d = grad.shape[1]
    s = torch.zeros((V, d), dtype=torch.float64, device=grad.device).index_add_(0, at, g)
    a = torch.zeros((V, d), dtype=torch.float64, device=grad.device).index_add_(0, at, g.abs())
    k = torch.bincount(at, minlength=V).double().unsqueeze(1)
    scale = float(torch.tensor(scale, dtype=torch.float32))
    bound = ((k.clamp(max=127) + k / 64 + 1) * 2.0 ** -24) * a * abs(scale)
    s = s * scale
    if old is not None:
        s = torch.where(k > 0, s + old.double(), old.double())
        bound = bound + torch.where(k > 0, 2.0 ** -24 * (s.abs() + bound), 0.0)
    return s, bound, k


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16], ids=["to_f32", "to_bf16"])
@pytest.mark.parametrize("n,V,d,how", [(1, 1, 1, "spread"), (1, 257, 64, "spread"), (63, 3, 33, "zipf"), (1000, 5000, 501, "zipf"), (5000, 300, 72, "runs"), (1153, 11, 40, "edges"), (3000, 1000, 16, "one"),
                                       (200, 40, 128, "none"), (20000, 151936, 64, "zipf"), (777, 50001, 100, "spread"), (300, 7, 5000, "zipf"), (4096, 2, 2100, "zipf")])
def test_embed_grad(gpu, ps, n, V, d, how, dtype, out_dtype):
    print(f"[case] embed_grad {n} {V} {d} {how} {dtype} {out_dtype}", flush=True)
    g = torch.Generator(device=gpu).manual_seed(n + d)
    tok = _tokens(n, V, 7, how).to(gpu)
    grad = torch.randn((tok.numel(), d + 1), device=gpu, generator=g).to(dtype)[:, :d]
    scale = 1.7
    s, bound, k = _expect(grad, tok, V, scale)
    bound = bound + HALF[out_dtype] * (s.abs() + bound)
    room = torch.full((V, d + 3), 9.0, dtype=out_dtype, device=gpu)
    out = ps.embed_grad(grad, tok, V, scale, out=room[:, :d])
    assert bool(((out.double() - s).abs() <= bound).all()) and bool((room[:, d:] == 9).all())
    assert bool((out[(k == 0)[:, 0]] == 0).all())
    if out_dtype == dtype:
        again = ps.embed_grad(grad, tok, V, scale)
        assert torch.equal(again, out)
    # added to what is there
    old = torch.randn((V, d), device=gpu, generator=g).to(out_dtype)
    s, bound, k = _expect(grad, tok, V, scale, old)
    bound = bound + HALF[out_dtype] * (s.abs() + bound)
    out = ps.embed_grad(grad, tok, V, scale, out=old.clone(), accumulate=True)
    assert bool(((out.double() - s).abs() <= bound).all())
    assert torch.equal(out[(k == 0)[:, 0]], old[(k == 0)[:, 0]])


def test_more_than_32_bits_of_elements(gpu, ps):
    print("[case] embed large offsets", flush=True)
    V, d = 1 << 20, 2100
    table = torch.zeros((V, d), dtype=torch.bfloat16, device=gpu)
    ids = torch.tensor([0, V - 1, V // 2, V - 2, -1, V, 1], dtype=torch.int32, device=gpu)
    rows = torch.randn(7, d, device=gpu).bfloat16()
    there = torch.tensor([0, 1, 2, 3, 6], device=gpu)
    table[ids[there].long()] = rows[there]
    want = rows.clone()
    want[4:6] = 0
    assert torch.equal(ps.embed(table, ids), want)
    for n in (7, 3000):                                       # (few positions, and many)
        tok = torch.full((n,), -1, dtype=torch.int32, device=gpu)
        tok[-7:] = ids
        g = torch.zeros((n, d), dtype=torch.bfloat16, device=gpu)
        g[-7:] = rows
        table.fill_(5.0)
        ps.embed_grad(g, tok, V, out=table)
        assert torch.equal(table[ids[there].long()], rows[there]) and int((table != 0).any(1).sum()) == 5
    wide = torch.randn((1100000, 2000), device=gpu).bfloat16()          # (and of rows)
    tok = torch.full((wide.shape[0],), 3, dtype=torch.int32, device=gpu)
    tok[:-2] = -1
    got = ps.embed_grad(wide, tok, 9, out=torch.empty((9, 2000), device=gpu))
    assert torch.equal(got[3], wide[-2].float() + wide[-1].float()) and int((got != 0).any(1).sum()) == 1


@pytest.mark.parametrize("V", [255, 256, 257, 262144, 262145, 1 << 20])
def test_vocabularies_around_the_sorts_shares(gpu, ps, V):
    print(f"[case] embed_grad V {V}", flush=True)
    g = torch.Generator(device=gpu).manual_seed(V)
    tok = torch.randint(0, V, (3000,), device=gpu, generator=g, dtype=torch.int32)
    tok[::3] = V - 1
    grad = torch.randn((3000, 9), device=gpu, generator=g)
    s, bound, k = _expect(grad, tok, V, 1.0)
    out = ps.embed_grad(grad, tok, V)
    assert bool(((out.double() - s).abs() <= bound + HALF[torch.float32] * (s.abs() + bound)).all()) and bool((out[(k == 0)[:, 0]] == 0).all())


def test_embed_grad_of_nothing(gpu, ps):
    print("[case] embed_grad nothing", flush=True)
    e = torch.empty((0, 40), device=gpu)
    tok = torch.empty(0, dtype=torch.int32, device=gpu)
    out = torch.full((30, 40), 3.0, device=gpu)
    ps.embed_grad(e, tok, 30, out=out, accumulate=True)
    assert bool((out == 3).all())
    ps.embed_grad(e, tok, 30, out=out)
    assert bool((out == 0).all())


def test_what_the_workspace_holds_does_not_matter(gpu, ps):
    print("[case] embed_grad workspace", flush=True)
    n, V, d = 4000, 500, 64
    tok = _tokens(n, V, 3, "runs").to(gpu)
    grad = torch.randn((n, d), device=gpu)
    need = ps.workspace_bytes(ps.CALL_EMBED_GRAD, ps.F32, n, V, d)
    want = ps.embed_grad(grad, tok, V)
    for fill in (0, 0xFF, 1, 0x7F):
        ws = torch.full((need,), fill, dtype=torch.uint8, device=gpu)
        if fill == 1:
            ws.view(torch.int32)[:] = torch.arange(need // 4, dtype=torch.int32, device=gpu) % V
        out = torch.empty((V, d), device=gpu)
        rc = ps.lib.picospec_embed_grad(grad.data_ptr(), ps.F32, d, n, tok.data_ptr(), V, d, 1.0, 0, out.data_ptr(), ps.F32, d, ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
        assert rc == ps.OK and torch.equal(out, want)


def test_embed_on_the_tape(gpu, ps):
    print("[case] embed on the tape", flush=True)
    from paper_2603_19133_amd import training
    for dtype in (torch.float32, torch.bfloat16):
        table = torch.randn(300, 50, device=gpu).to(dtype).requires_grad_()
        tok = _tokens(400, 300, 9, "zipf").view(20, 20).to(gpu)
        out = training.embed(table, tok, 2.0)
        assert out.shape == (20, 20, 50) and torch.equal(out.detach(), ps.embed(table.detach(), tok, 2.0))
        w = torch.randn(20, 20, 50, device=gpu).to(dtype)
        out.backward(w)
        assert table.grad.dtype == dtype and torch.equal(table.grad, ps.embed_grad(w, tok, 300, 2.0))
        table.grad = None
        training.embed(table, tok).sum().backward()                                  # (one value seen from every place)
        s, bound, k = _expect(torch.ones(400, 50, device=gpu), tok.view(-1), 300, 1.0)
        assert bool(((table.grad.double() - s).abs() <= bound + HALF[dtype] * s.abs()).all())
        with pytest.raises(RuntimeError, match="differentiable once"):
            torch.autograd.grad(training.embed(table, tok).sum(), table, create_graph=True)
    # the formula's gradient against differences: the call is linear in the table
    table = torch.randn(9, 4, device=gpu)
    tok = torch.tensor([1, 5, 1, 1, -1, 8], dtype=torch.int32, device=gpu)
    w = torch.randn(6, 4, device=gpu)
    g = ps.embed_grad(w, tok, 9, 1.5)
    for v in range(9):
        for j in range(4):
            up, down = table.clone(), table.clone()
            up[v, j] += 0.5
            down[v, j] -= 0.5
            diff = ((ps.embed(up, tok, 1.5).double() - ps.embed(down, tok, 1.5).double()) * w).sum().item() / (up[v, j] - down[v, j]).double().item()
            # two roundings (2^-24) of values below 1.5 * 5 for each of up to three positions, times |w| < 5, over a step of 1; and the gradient's own
            assert abs(g[v, j].item() - diff) <= 3 * 2 * 7.5 * 5 * 2.0 ** -24 + 4 * 2.0 ** -24 * 22.5


def test_refusals(gpu, ps):
    print("[case] embed refusals", flush=True)
    table, tok = torch.randn(10, 8, device=gpu), torch.zeros(4, dtype=torch.int32, device=gpu)
    g = torch.randn(4, 8, device=gpu)
    for f in (lambda: ps.embed(table, tok.long()), lambda: ps.embed(table, tok.cpu()), lambda: ps.embed(table.t(), tok), lambda: ps.embed(table[:0], tok), lambda: ps.embed(table, tok, float("nan")),
              lambda: ps.embed(table, tok, out=torch.zeros(4, 9, device=gpu)), lambda: ps.embed(table, tok, out=torch.zeros(3, 8, device=gpu)), lambda: ps.embed(table, tok, out=table[2:6]),
              lambda: ps.embed(table, torch.zeros(8, dtype=torch.int32, device=gpu)[::2]), lambda: ps.embed_grad(g, tok[:3], 10), lambda: ps.embed_grad(g, tok, 0),
              lambda: ps.embed_grad(g, tok, 10, accumulate=True), lambda: ps.embed_grad(g, tok, 10, out=torch.zeros(9, 8, device=gpu)), lambda: ps.embed_grad(g, tok.long(), 10),
              lambda: ps.embed_grad(g, tok, 10, out=torch.zeros(8, 10, device=gpu).t())):
        with pytest.raises(ps.PicoSpecError) as e:
            f()
        assert e.value.code == ps.EINVAL
    for f in (lambda: ps.embed(table.half(), tok), lambda: ps.embed(table, tok, out=torch.zeros(4, 8, device=gpu, dtype=torch.bfloat16)), lambda: ps.embed_grad(g.double(), tok, 10),
              lambda: ps.embed_grad(g, tok, 10, out=torch.zeros(10, 8, device=gpu, dtype=torch.float16))):
        with pytest.raises(ps.PicoSpecError) as e:
            f()
        assert e.value.code == ps.EDTYPE
