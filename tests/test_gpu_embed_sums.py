"""How picospec_embed_grad's sums round where rounding counts: rows whose errors all point one way, so that a chain of k additions is off by k of them.

One row of 1 and then rows of just under 2^-24, half a step of fp32 at 1: added to the 1 one by one each of them is lost.  A sum of k rows has to stay within (min(k, 127) + k / 64) 2^-24 of the sum
of absolute values all the same (see test_gpu_embed), whatever the number of positions, the rows' width and what shares them out."""
import pytest
import torch

from test_gpu_embed import HALF, _expect

pytestmark = pytest.mark.gpu

SMALL = (1 - 2.0 ** -8) * 2.0 ** -24          # (a bf16 number, too)


@pytest.fixture(scope="module")
def ps():
    from paper_2603_19133_amd import binding
    return binding


@pytest.mark.parametrize("accumulate", [False, True], ids=["write", "add"])
@pytest.mark.parametrize("share", [1.0, 0.5])
@pytest.mark.parametrize("n", [100, 300, 1024, 1025, 6000])
@pytest.mark.parametrize("dtype,d", [(torch.float32, 20), (torch.float32, 200), (torch.float32, 389), (torch.float32, 1024), (torch.bfloat16, 600), (torch.bfloat16, 1001), (torch.bfloat16, 4096)],
                         ids=lambda x: str(x).replace("torch.", ""))
def test_rows_whose_errors_add_up(gpu, ps, dtype, d, n, share, accumulate):
    print(f"[case] embed_grad sums {dtype} {d} {n} {share} {accumulate}", flush=True)
    V = 300
    tok = torch.randint(0, V, (n,), generator=torch.Generator().manual_seed(n + d), dtype=torch.int32)
    tok[:int(n * share)] = 7
    tok = tok[torch.randperm(n, generator=torch.Generator().manual_seed(1))].to(gpu)
    grad = torch.full((n, d), SMALL, dtype=dtype, device=gpu)
    grad[int(torch.nonzero(tok == 7)[0])] = 1.0
    old = torch.zeros((V, d), device=gpu) if accumulate else None
    s, bound, _ = _expect(grad, tok, V, 1.0, old)
    out = ps.embed_grad(grad, tok, V, out=old.clone() if accumulate else torch.full((V, d), 3.0, device=gpu), accumulate=accumulate)
    off = (out.double() - s).abs()
    assert bool((off <= bound + HALF[torch.float32] * (s.abs() + bound)).all()), float(off.max()) * 2 ** 24
