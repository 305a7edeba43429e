"""Backward calls whose saved tensors come back in another form than they went, as a hook on saved tensors may give them: an error that a program can catch."""
import pytest
import torch

pytestmark = pytest.mark.gpu

FORMS = {
    "on the host": lambda t: t.cpu(),
    "by columns": lambda t: t.t().contiguous().t() if t.dim() == 2 else t.repeat_interleave(2)[::2],
    "in halves": lambda t: t.half(),
}


@pytest.fixture(scope="module")
def calls(gpu):
    """name -> (leaf, function of it whose backward reads what it has saved)"""
    from paper_2603_19133_amd import binding as ps
    from paper_2603_19133_amd import training
    V, rows = 300, 8
    z = torch.randn((rows, V), device=gpu, requires_grad=True)
    table = torch.randn((V, 20), device=gpu, requires_grad=True)
    tok = torch.randint(0, V, (rows,), device=gpu, dtype=torch.int32)
    hist = ps.History(torch.randint(0, V, (rows, 30), device=gpu, dtype=torch.int32), torch.full((rows,), 20, dtype=torch.int32, device=gpu))
    rec = ps.compress(torch.randn((rows, V), device=gpu), V, 1.0, 10)
    rounds = ps.History(hist.tok[:2], hist.length[:2])
    off = torch.tensor([0, 3, 6], dtype=torch.int32, device=gpu)
    return {"adjust": (z, lambda: training.adjust(z, V, hist, repetition=torch.full((rows,), 1.5, device=gpu))),
            "adjust round": (z, lambda: training.adjust(z, V, rounds, repetition=1.5, seq_off=off, draft_tok=tok[:6])),
            "embed": (table, lambda: training.embed(table, tok)),
            "distill_loss": (z, lambda: training.distill_loss(z, rec, V, 1.0)[0])}


def _refused(leaf, call, unpack):
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, unpack):
        out = call()
    w = torch.ones_like(out)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(out, leaf, w)
    # (and the next one goes as ever)
    assert torch.autograd.grad(call(), leaf, w)[0].isfinite().all()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("name", ["adjust", "adjust round", "embed", "distill_loss"])
def test_other_forms(gpu, calls, name, form):
    print(f"[case] saved tensors {name} {form}", flush=True)
    _refused(*calls[name], FORMS[form])
