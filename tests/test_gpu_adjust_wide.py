"""A vocabulary whose size has more than 32 bits, in calls that hand it on as an int32."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_a_vocabulary_beyond_32_bits_is_refused(gpu):
    print("[case] adjust V beyond 32 bits", flush=True)
    from paper_2603_19133_amd import binding as ps
    from paper_2603_19133_amd import training
    V = (1 << 32) + 100                                       # (100 in 32 bits)
    z = torch.empty((1, V), dtype=torch.bfloat16, device=gpu)
    for f in (lambda: ps.adjust(z, V, presence=1.0), lambda: ps.adjust(z, V, out=z), lambda: ps.adjust_grad(z, z, V, out=z), lambda: training.adjust(z, V)):
        with pytest.raises(ps.PicoSpecError) as e:
            f()
        assert e.value.code == ps.EUNSUPPORTED
    assert ps.adjust(z[:, :100], 100).shape == (1, 100)
