"""picospec_adjust and its gradient value by value where test_gpu_adjust looks at a part: gradients of a sum, and every element of a matrix whose offsets pass 32 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ps():
    from paper_2603_19133_amd import binding
    return binding


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_the_gradient_of_a_sum(gpu, ps, dtype):
    """One value seen from every place: 1 / r above 0, r at 0 and below it for seen tokens, 1 for the others, 0 behind the vocabulary; r a power of two."""
    print(f"[case] adjust sum {dtype}", flush=True)
    from paper_2603_19133_amd import training
    V, pad = 501, 6
    gammas, B = [2, 4, 0], 3
    rows, N = sum(gammas) + B, sum(gammas)
    g = torch.Generator(device=gpu).manual_seed(2)
    z = torch.randn((rows, V + pad), device=gpu, generator=g).to(dtype)
    z[:, ::9] = 0
    z.requires_grad_()
    hist = ps.History(torch.randint(0, V, (B, 60), device=gpu, generator=g, dtype=torch.int32), torch.tensor([60, 0, 33], dtype=torch.int32, device=gpu))
    off = torch.tensor([0, 2, 6, 6], dtype=torch.int32, device=gpu)
    draft = torch.randint(0, V, (N,), device=gpu, generator=g, dtype=torch.int32)
    r = torch.tensor([2.0, 0.5, 1.0], device=gpu)
    training.adjust(z, V, hist, repetition=r, seq_off=off, draft_tok=draft).sum().backward()
    want = torch.zeros_like(z)
    want[:, :V] = 1
    row = 0
    for b in range(B):
        for t in range(gammas[b] + 1):
            met = torch.cat([hist.tok[b, :int(hist.length[b])], draft[int(off[b]):int(off[b]) + t]]).long().unique()
            want[row, met] = torch.where(z.detach()[row, met] > 0, 1 / r[b], r[b]).to(dtype)
            row += 1
    assert torch.equal(z.grad, want)
    ones = torch.ones((rows, V), dtype=dtype, device=gpu)
    assert torch.equal(z.grad[:, :V], ps.adjust_grad(ones, z.detach(), V, hist, repetition=r, seq_off=off, draft_tok=draft))


def test_every_element_beyond_32_bits_of_them(gpu, ps):
    print("[case] adjust every element of 4.5 GB", flush=True)
    B, V = 15000, 150001                                          # (row 14,317 holds element 2^31)
    at = torch.arange(B, device=gpu)
    tok = ((at * 10007) % V).int().view(B, 1)
    hist = ps.History(tok, torch.ones(B, dtype=torch.int32, device=gpu))
    z = torch.zeros((B, V), dtype=torch.bfloat16, device=gpu)
    new = ps.adjust(z, V, hist, presence=2.0)
    assert bool((z == 0).all())
    for out in (new, ps.adjust(z, V, hist, presence=2.0, out=z)):
        assert bool(((out != 0).sum(1) == 1).all()) and bool((out[at, tok[:, 0].long()] == -2).all())
    out = ps.adjust_grad(new, z, V, hist, repetition=4.0)         # (-2 at each row's token, whose logit is below 0)
    assert bool(((out != 0).sum(1) == 1).all()) and bool((out[at, tok[:, 0].long()] == -8).all())
