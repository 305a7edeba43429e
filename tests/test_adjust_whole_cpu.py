"""picospec_adjust_whole and picospec_adjust_grad_whole, the part without a GPU: they refuse what picospec_adjust and picospec_adjust_grad refuse, and rows in place."""
import pytest

import test_more_operators_cpu as T

B = T.B                                              # (the fixture)


class _Whole:
    """The binding with the two calls in place of those that they are variants of."""

    class _Lib:
        def __init__(self, lib):
            self.picospec_adjust, self.picospec_adjust_grad = lib.picospec_adjust_whole, lib.picospec_adjust_grad_whole

    def __init__(self, binding):
        self.lib = self._Lib(binding.lib)


@pytest.mark.parametrize("kw", T.BAD_ROWS + [dict(pres=float("inf")), dict(freq=float("nan")), dict(off=T.FAKE, n_bias=-1), dict(out=T.FAKE + 4), dict(out=T.FAKE)])
def test_adjust_whole_refuses(B, kw):
    assert T._adjust(_Whole(B), **kw) == B.EINVAL


@pytest.mark.parametrize("kw", T.BAD_ROWS + [dict(grad=None), dict(ld_g=99), dict(out=T.FAKE * 2), dict(out=T.FAKE)])
def test_adjust_grad_whole_refuses(B, kw):
    assert T._adjust_grad(_Whole(B), **kw) == B.EINVAL


def test_no_rows_and_types(B):
    w = _Whole(B)
    assert T._adjust(w, rows=0, seqs=0, logits=None, out=None) == B.OK and T._adjust_grad(w, rows=0, seqs=0, grad=None, logits=None, out=None) == B.OK
    assert T._adjust(w, dtype=9) == B.EDTYPE and T._adjust_grad(w, dtype=9) == B.EDTYPE
