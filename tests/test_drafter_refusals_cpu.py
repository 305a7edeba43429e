"""What the calls beside the round refuse before the library is called, without a GPU: the checks run on host tensors (the meta device stands for another one),
and a call that gets past them is seen by a stand-in for the native part."""
import types

import pytest
import torch

from paper_2603_19133_amd import binding as ps

ROWS, V = 4, 100


@pytest.fixture
def calls(monkeypatch):
    """The names of the native calls that were made."""
    made = []
    native = types.SimpleNamespace(
        rows2d=lambda t: (0, t.stride(0), t.shape[0]), scratch=lambda *a: None,
        distill_inputs=lambda z, *a: (0, z.stride(0), z.shape[0]),
        empty=lambda like, codes, *sizes: tuple(torch.empty(s, dtype={"i": torch.int32, "f": torch.float32, "d": torch.float64}[c]) for c, s in zip(codes, sizes)),
        **{name: (lambda *a, name=name: made.append(name) or 0) for name in ("sample", "distill", "distill_grad")})
    monkeypatch.setattr(ps, "_nat", native)
    monkeypatch.setattr(ps, "_stream", lambda: 0)
    return made


def _out(rows=ROWS, **kw):
    o = dict(tok=torch.empty(rows, dtype=torch.int32), prob=torch.empty(rows), count=torch.empty(rows, dtype=torch.int32), lse=torch.empty(rows))
    return ps.Sampled(**{**o, **kw})


def test_sample_refuses_outputs_that_do_not_hold_the_rows(calls):
    z, u = torch.zeros(ROWS, V), torch.zeros(ROWS)
    for name in ("tok", "prob", "count", "lse"):
        t = getattr(_out(), name)
        other = torch.float32 if t.dtype == torch.int32 else torch.int32
        for bad in (t[:-1], t.to(other), torch.empty(2 * ROWS, dtype=t.dtype)[::2], t.to("meta")):
            with pytest.raises(ps.PicoSpecError):
                ps.sample(z, V, u, out=_out(**{name: bad}))
    assert not calls
    for good in (_out(), _out(ROWS + 3)):
        assert ps.sample(z, V, u, out=good) is good
    assert calls == ["sample"] * 2


def test_sample_refuses_tensors_of_another_device(calls):
    z, u = torch.zeros(ROWS, V), torch.zeros(ROWS)
    f, i = torch.ones(ROWS), torch.ones(ROWS, dtype=torch.int32)
    for kw in (dict(uniforms=u.to("meta")), dict(temperature=f.to("meta")), dict(top_k=i.to("meta")), dict(top_p=f.to("meta")), dict(min_p=f.to("meta"))):
        with pytest.raises(ps.PicoSpecError):
            ps.sample(z, V, **{**dict(uniforms=u), **kw})
    assert not calls
    ps.sample(z, V, u, temperature=f, top_k=i, top_p=f, min_p=f)
    assert calls == ["sample"]


def _record(rows=ROWS, k=5):
    return ps.Compressed(torch.zeros(rows, k, dtype=torch.int32), torch.zeros(rows, k), torch.zeros(rows, dtype=torch.int32), torch.zeros(rows), torch.zeros(rows), k)


def test_distill_grad_refuses_statistics_and_outputs_of_another_device(calls):
    z, stats = torch.zeros(ROWS, V), torch.zeros(ROWS, 4, dtype=torch.float64)
    for s, out in ((stats.to("meta"), torch.empty(ROWS, V)), (stats, torch.empty(ROWS, V, device="meta"))):
        with pytest.raises(ps.PicoSpecError):
            ps.distill_grad(z, V, 1.0, _record(), s, out=out)
    assert not calls
    ps.distill_grad(z, V, 1.0, _record(), stats, out=torch.empty(ROWS, V))
    assert calls == ["distill_grad"]


def test_a_vocabulary_wider_than_the_view_is_refused(calls):
    """The last columns of a wider tensor: its rows are as far apart as the vocabulary is long, but the last one ends with the tensor."""
    z = torch.zeros(ROWS, 2 * V)[:, V:]
    assert z.stride(0) >= V + 1
    for call in (lambda v: ps.sample(z, v, torch.zeros(ROWS)), lambda v: ps.distill(z, v, 1.0, _record()),
                 lambda v: ps.distill_grad(z, v, 1.0, _record(), torch.zeros(ROWS, 4, dtype=torch.float64), out=torch.empty(ROWS, 2 * V))):
        with pytest.raises(ps.PicoSpecError):
            call(V + 1)
        call(V)
    assert calls == ["sample", "distill", "distill_grad"]
