"""picospec_adjust and its gradient where the launch is nearly as large as one can be."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_sixteen_million_sequences(gpu):
    print("[case] adjust 2^32 threads less a few", flush=True)
    from paper_2603_19133_amd import binding as ps
    B, V = (1 << 24) - 1, 7
    z = torch.arange(B * V, dtype=torch.int32, device=gpu).view(B, V).remainder_(251).float()
    tok = (torch.arange(B, dtype=torch.int32, device=gpu) % V).view(B, 1)
    hist = ps.History(tok, torch.ones(B, dtype=torch.int32, device=gpu))
    met = tok == torch.arange(V, dtype=torch.int32, device=gpu)
    assert torch.equal(ps.adjust(z, V, hist, presence=3.0), torch.where(met, z - 3.0, z))
    g = torch.ones_like(z)
    assert torch.equal(ps.adjust_grad(g, z, V, hist, repetition=2.0), torch.where(met, torch.where(z > 0, 0.5, 2.0), 1.0))
    with pytest.raises(ps.PicoSpecError) as e:
        ps.adjust(torch.zeros((B + 1, V), device=gpu), V, presence=1.0)
    assert e.value.code == ps.EUNSUPPORTED
