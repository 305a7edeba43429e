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


SIZES = {
    "all of fewer rows": lambda t: t[:-1],
    "all of more rows": lambda t: torch.cat([t, t[:1]]),
    "logits of fewer rows": lambda t: t[:-1] if t.dtype == torch.float32 and t.dim() == 2 and t.shape[1] == 300 else t,
    "logits of more rows": lambda t: torch.cat([t, t[:1]]) if t.dtype == torch.float32 and t.dim() == 2 and t.shape[1] == 300 else t,
    "logits of fewer columns": lambda t: t[:, :-1].contiguous() if t.dtype == torch.float32 and t.dim() == 2 and t.shape[1] == 300 else t,
    "whole numbers on the host": lambda t: t.cpu() if t.dtype == torch.int32 else t,
    "fewer whole numbers": lambda t: t[:-1] if t.dtype == torch.int32 else t,
    "wide numbers on the host": lambda t: t.cpu() if t.dtype == torch.float64 else t,
    "fewer wide numbers": lambda t: t[:-1] if t.dtype == torch.float64 else t,
}


@pytest.mark.parametrize("name,size", [(n, s) for n in ("adjust", "adjust round", "embed", "distill_loss") for s in SIZES
                                       if not (s.startswith("logits") and n == "embed") and not ("wide" in s and n != "distill_loss")])       # (what a call saves)
def test_other_sizes(gpu, calls, name, size):
    print(f"[case] saved tensors {name} {size}", flush=True)
    _refused(*calls[name], SIZES[size])
