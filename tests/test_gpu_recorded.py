"""Tensors that torch's autograd records, given to calls that it does not learn of: refused while it records, as torch refuses them as `out`."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ps():
    from paper_2603_19133_amd import binding
    return binding


def _refuses(ps, f):
    with pytest.raises(ps.PicoSpecError) as e:
        f()
    assert e.value.code == ps.EINVAL


def test_an_output_that_is_recorded(gpu, ps):
    print("[case] recorded outputs", flush=True)
    V = 50
    x = torch.randn((4, V), device=gpu, requires_grad=True)
    tok = torch.tensor([1, 2, 3, 4], dtype=torch.int32, device=gpu)
    hist = ps.History(tok.view(4, 1), torch.ones(4, dtype=torch.int32, device=gpu))
    table, rows = torch.randn((9, V), device=gpu), torch.randn((4, V), device=gpu)
    calls = [lambda z: ps.adjust(z, V, hist, presence=1.0, out=z), lambda z: ps.adjust(rows, V, hist, presence=1.0, out=z), lambda z: ps.adjust_grad(z, rows, V, hist, repetition=2.0, out=z),
             lambda z: ps.embed(table, tok, out=z), lambda z: ps.embed_grad(rows, tok, 4, out=z), lambda z: ps.embed_grad(rows, tok, 4, out=z, accumulate=True),
             lambda z: ps.clip_grad([rows], 1e-3, out=[z])]
    for call in calls:
        for z in (x * 1.0, x):                          # (a value of the tape, and a leaf)
            before = z.detach().clone()
            _refuses(ps, lambda: call(z))
            assert torch.equal(z.detach(), before)
        with torch.no_grad():                           # (a caller that says so may)
            z = (x * 1.0).requires_grad_()
            call(z)
            assert not torch.equal(z, x)
        z = x.detach().clone()                          # (nor is anything else refused)
        call(z)
        assert not torch.equal(z, x.detach())
    # gradients that are themselves recorded may be clipped in place, as torch's own clipping does
    y = (x * 1.0)
    ps.clip_grad([y], 1e-3)
    assert float(y.detach().norm()) <= 1.01e-3


def test_settings_that_are_recorded(gpu, ps):
    """training.adjust has a gradient for the logits alone."""
    print("[case] recorded settings", flush=True)
    from paper_2603_19133_amd import training
    V = 50
    z = torch.randn((3, V), device=gpu, requires_grad=True)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=gpu)                                                       # noqa: E731
    hist = ps.History(i32(1, 2, 3).view(3, 1), i32(1, 1, 1))
    learnt = torch.full((3,), 1.5, device=gpu, requires_grad=True)
    for kw in (dict(repetition=learnt), dict(presence=learnt), dict(frequency=learnt), dict(bias=ps.Bias(i32(0, 1, 2, 3), i32(4, 5, 6), learnt))):
        _refuses(ps, lambda: training.adjust(z, V, hist, **kw))
        with torch.no_grad():
            want = training.adjust(z, V, hist, **kw)
        for k, v in kw.items():
            kw[k] = ps.Bias(v.off, v.id, v.value.detach()) if k == "bias" else v.detach()
        out = training.adjust(z, V, hist, **kw)
        assert out.requires_grad and torch.equal(out.detach(), want)
