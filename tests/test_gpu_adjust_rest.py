"""Rows of a batch that no sequence has: offsets that begin above 0 or end before the last drafted token, as those of a batch that is padded for a graph do.

Rows that a call makes itself are zeros there, whatever their memory held, and so is the logits' gradient; every other row has the bits that it has in rows that the caller brings."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ps():
    from paper_2603_19133_amd import binding
    return binding


def _poisoned(call, like):
    """call() with NaN in the memory that its output of `like`'s size is likely to get."""
    torch.cuda.synchronize()
    dirt = [torch.full_like(like, float("nan")) for _ in range(4)]
    torch.cuda.synchronize()
    del dirt
    return call()


CASES = {
    "ends early": dict(off=[0, 2, 2], N=4, V=100, bonus=True),
    "begins late": dict(off=[3, 5, 5, 9], N=9, V=1001, bonus=True),
    "both": dict(off=[2, 2, 6, 7], N=11, V=5003, bonus=True),
    "draft rows": dict(off=[1, 1, 4], N=9, V=2050, bonus=False),
    "nothing of it": dict(off=[5, 5, 5], N=9, V=70, bonus=False),
    "all of it": dict(off=[0, 4, 9], N=9, V=9000, bonus=True),
    "much behind": dict(off=[0, 1], N=700, V=1300, bonus=True),
    "many": dict(off=[7 + 3 * i for i in range(120)], N=500, V=20001, bonus=True),
    "many draft rows": dict(off=[0] + [2 + 2 * i for i in range(60)], N=400, V=40000, bonus=False),
    "beyond the arrays": dict(off=[-4, 2, 99], N=9, V=300, bonus=True),
}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("cap", [30, 9000])
@pytest.mark.parametrize("name", CASES)
def test_rows_of_no_sequence_are_zeros(gpu, ps, name, cap, dtype):
    print(f"[case] adjust rest {name} {cap} {dtype}", flush=True)
    from paper_2603_19133_amd import training
    c = CASES[name]
    V, N, B = c["V"], c["N"], len(c["off"]) - 1
    rows = N + B * c["bonus"]
    g = torch.Generator(device=gpu).manual_seed(V)
    z = (torch.randn((rows, V), device=gpu, generator=g) * 3).to(dtype)
    grad = torch.randn((rows, V), device=gpu, generator=g).to(dtype)
    hist = ps.History(torch.randint(0, V, (B, cap), device=gpu, generator=g, dtype=torch.int32), torch.randint(0, cap + 1, (B,), device=gpu, generator=g, dtype=torch.int32))
    args = dict(repetition=torch.rand(B, device=gpu, generator=g) + 0.7, seq_off=torch.tensor(c["off"], dtype=torch.int32, device=gpu),
                draft_tok=torch.randint(0, V, (N,), device=gpu, generator=g, dtype=torch.int32))
    clamped = [min(max(x, 0), N) for x in c["off"]]
    own = torch.zeros(rows, dtype=torch.bool, device=gpu)
    own[clamped[0]:clamped[-1] + B * c["bonus"]] = True
    # into rows that the caller brings: those of no sequence stay
    want, want_grad = torch.full_like(z, 5.0), torch.full_like(z, 5.0)
    ps.adjust(z, V, hist, presence=0.3, out=want, **args)
    ps.adjust_grad(grad, z, V, hist, out=want_grad, **args)
    assert bool((want[~own] == 5).all()) and bool((want_grad[~own] == 5).all())
    want[~own] = 0
    want_grad[~own] = 0
    assert torch.equal(_poisoned(lambda: ps.adjust(z, V, hist, presence=0.3, **args), z), want)
    assert torch.equal(_poisoned(lambda: ps.adjust_grad(grad, z, V, hist, **args), z), want_grad)
    z.requires_grad_()
    out = _poisoned(lambda: training.adjust(z, V, hist, presence=0.3, **args), z)
    assert torch.equal(out.detach(), want)
    _poisoned(lambda: out.backward(grad), z)
    assert torch.equal(z.grad, want_grad)


def test_a_captured_batch_whose_offsets_change(gpu, ps):
    print("[case] adjust rest graph", flush=True)
    V, N, B = 3001, 12, 3
    z = torch.randn((N + B, V), device=gpu)
    off = torch.tensor([0, 4, 8, 12], dtype=torch.int32, device=gpu)
    draft = torch.randint(0, V, (N,), device=gpu, dtype=torch.int32)
    call = lambda: ps.adjust(z, V, presence=0.5, seq_off=off, draft_tok=draft)                                          # noqa: E731
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for o in ([0, 4, 8, 12], [0, 1, 1, 3], [2, 3, 9, 9], [0, 0, 0, 0], [0, 4, 8, 12]):
        off.copy_(torch.tensor(o, dtype=torch.int32))
        graph.replay()
        want = call()
        torch.cuda.synchronize()
        assert torch.equal(out, want), o
        assert bool((out[:o[0]] == 0).all()) and bool((out[o[-1] + B:] == 0).all()) and bool((out[o[0]:o[-1] + B] != 0).any(1).all())
