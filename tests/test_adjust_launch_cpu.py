"""Calls of picospec_adjust and picospec_adjust_grad that are larger than a launch can be, 2^32 threads, are refused before anything is launched, whichever shape of a workgroup they take."""
import pytest

import test_more_operators_cpu as T

B = T.B                                              # (the fixture)


@pytest.mark.parametrize("seqs,V,mean,cap", [
    ((1 << 22) + 100, 100, 8, 20000),                # workgroups of 512 threads for a vocabulary of one chunk, a sequence's rows shared out in two
    ((1 << 23) + 100, 100, 1, 20000),                # the same, decoding
    ((1 << 21) + 100, 9000, 8, 100000),              # two chunks
    ((1 << 24) + 100, 100, 1, 0),                    # workgroups of 256 threads
    ((1 << 23) + 100, 100, 8, 0),
], ids=lambda x: str(x))
def test_more_threads_than_a_launch_has(B, seqs, V, mean, cap):
    rows = seqs * mean
    kw = dict(rows=rows, seqs=seqs, V=V, ld=V, ld_out=V, hist=T.FAKE if cap else None, length=T.FAKE if cap else None, cap=cap, ld_hist=cap, out=1 << 60)
    if mean > 1:
        kw.update(seq_off=T.FAKE, n_draft=rows - seqs, draft=T.FAKE)
    assert T._adjust(B, **kw) == B.EUNSUPPORTED
    assert T._adjust_grad(B, ld_g=V, logits=1 << 50, **{k: v for k, v in kw.items()}) == B.EUNSUPPORTED
