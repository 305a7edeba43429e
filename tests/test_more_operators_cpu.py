"""picospec_adjust, picospec_embed, picospec_clip_grad and their gradients, the part without a GPU: every refusal of the C entries, the workspaces' sizes, and that the binding
refuses tensors that are not on a device."""
import ctypes as C

import pytest
import torch

FAKE, FAR = 0x1000, 0x10000000                     # non-null addresses that are never dereferenced


@pytest.fixture(scope="module")
def B():
    from paper_2603_19133_amd import binding
    return binding


def _adjust(B, logits=FAKE, dtype=0, ld=100, rows=2, V=100, seqs=2, n_draft=0, seq_off=None, draft=None, hist=FAKE, ld_hist=8, cap=8, length=FAKE, prompt=None,
            rep=1.1, pres=0.0, freq=0.0, rows_of=(None, None, None), off=None, ids=None, val=None, n_bias=0, mask=None, ld_mask=4, masks=2, mask_row=None, out=FAR, ld_out=100):
    return B.lib.picospec_adjust(logits, dtype, ld, rows, V, seqs, n_draft, seq_off, draft, hist, ld_hist, cap, length, prompt, rep, pres, freq, *rows_of, off, ids, val, n_bias,
                                 mask, ld_mask, masks, mask_row, out, ld_out, None)


def _adjust_grad(B, grad=FAKE, ld_g=100, logits=FAKE * 2, dtype=0, ld=100, rows=2, V=100, seqs=2, n_draft=0, seq_off=None, draft=None, hist=FAKE, ld_hist=8, cap=8, length=FAKE,
                 rep=1.1, rep_rows=None, mask=None, ld_mask=4, masks=2, mask_row=None, out=FAR, ld_out=100):
    return B.lib.picospec_adjust_grad(grad, ld_g, logits, dtype, ld, rows, V, seqs, n_draft, seq_off, draft, hist, ld_hist, cap, length, rep, rep_rows, mask, ld_mask, masks, mask_row,
                                      out, ld_out, None)


BAD_ROWS = [dict(rows=-1), dict(V=0), dict(ld=99), dict(ld_out=99), dict(logits=None), dict(out=None), dict(out=FAR + 2), dict(seqs=3), dict(seqs=-1), dict(n_draft=1),
            dict(seq_off=FAKE, n_draft=3), dict(seq_off=FAKE, n_draft=2, seqs=1), dict(seq_off=FAKE, n_draft=-1, seqs=1), dict(seq_off=FAKE, n_draft=2, seqs=0, draft=FAKE),
            dict(length=None), dict(cap=9), dict(cap=-1), dict(rep=0.0), dict(rep=float("nan")), dict(rep=float("inf")), dict(rep=-1.0),
            dict(mask=FAKE, ld_mask=3), dict(mask=FAKE, masks=1), dict(mask=FAKE, masks=-1, mask_row=FAKE)]


@pytest.mark.parametrize("kw", BAD_ROWS + [dict(pres=float("inf")), dict(freq=float("nan")), dict(off=FAKE, n_bias=-1), dict(off=FAKE, n_bias=2, ids=FAKE),
                                           dict(out=FAKE + 4), dict(out=FAKE, ld_out=101), dict(out=FAKE + 796)])
def test_adjust_refuses(B, kw):
    assert _adjust(B, **kw) == B.EINVAL


@pytest.mark.parametrize("kw", BAD_ROWS + [dict(grad=None), dict(ld_g=99), dict(out=FAKE * 2), dict(out=FAKE + 4), dict(out=FAKE, ld_out=101),
                                           dict(grad=FAKE, logits=FAKE, ld=120, out=FAKE)])
def test_adjust_grad_refuses(B, kw):
    assert _adjust_grad(B, **kw) == B.EINVAL


def test_adjust_refuses_types_and_sizes(B):
    for f in (_adjust, _adjust_grad):
        assert f(B, dtype=7) == B.EDTYPE
        assert f(B, V=(1 << 20) + 1, ld=1 << 21, ld_out=1 << 21, **({"ld_g": 1 << 21} if f is _adjust_grad else {})) == B.EUNSUPPORTED
        big = dict(rows=1 << 22, seqs=1 << 22, V=50000, ld=50000, ld_out=50000, out=1 << 60)
        assert f(B, **big, **({"ld_g": 50000, "logits": 1 << 50} if f is _adjust_grad else {})) == B.EUNSUPPORTED
        assert f(B, rows=0, seqs=0, logits=None, out=None) == B.OK
        assert f(B, rows=0, seqs=3, seq_off=FAKE, logits=None, out=None) == B.OK


def _embed(B, table=FAKE, dtype=0, ld=8, V=10, d=8, tok=FAKE, n=4, scale=1.0, out=FAR, ld_out=8):
    return B.lib.picospec_embed(table, dtype, ld, V, d, tok, n, scale, out, ld_out, None)


@pytest.mark.parametrize("kw", [dict(V=0), dict(d=0), dict(n=-1), dict(ld=7), dict(ld_out=7), dict(scale=float("nan")), dict(scale=float("inf")), dict(table=None), dict(tok=None),
                                dict(out=None), dict(table=FAKE + 2), dict(out=FAR + 2), dict(out=FAKE + 316), dict(out=FAKE - 124)])
def test_embed_refuses(B, kw):
    assert _embed(B, **kw) == B.EINVAL


def _embed_grad(B, grad=FAKE, dtype=0, ld=8, n=4, tok=FAKE, V=10, d=8, scale=1.0, acc=0, out=FAR, dt_out=0, ld_out=8, ws=FAKE, ws_bytes=1 << 20):
    return B.lib.picospec_embed_grad(grad, dtype, ld, n, tok, V, d, scale, acc, out, dt_out, ld_out, ws, ws_bytes, None)


@pytest.mark.parametrize("kw", [dict(V=0), dict(d=0), dict(n=-1), dict(ld=7), dict(ld_out=7), dict(scale=float("nan")), dict(acc=2), dict(grad=None), dict(tok=None), dict(out=None),
                                dict(out=FAR + 2), dict(grad=FAKE + 2), dict(out=FAKE + 124), dict(out=FAKE - 316)])
def test_embed_grad_refuses(B, kw):
    assert _embed_grad(B, **kw) == B.EINVAL


def test_embed_refuses_types_sizes_and_workspaces(B):
    assert _embed(B, dtype=3) == B.EDTYPE and _embed_grad(B, dtype=3) == B.EDTYPE and _embed_grad(B, dt_out=-1) == B.EDTYPE
    assert _embed(B, V=(1 << 20) + 1) == B.EUNSUPPORTED and _embed_grad(B, V=(1 << 20) + 1) == B.EUNSUPPORTED and _embed_grad(B, n=(1 << 26) + 1, out=1 << 50) == B.EUNSUPPORTED
    assert _embed(B, n=0, tok=None, out=None, table=None) == B.OK
    assert _embed_grad(B, n=0, acc=1, tok=None, grad=None, ws=None, ws_bytes=0) == B.OK
    assert B.workspace_bytes(B.CALL_EMBED_GRAD, B.F32, 1024, 10, 8) == 0          # (few positions are looked up where they are)
    need = B.workspace_bytes(B.CALL_EMBED_GRAD, B.F32, 1025, 10, 8)
    assert need >= 4 * 1025 + 8 * 10 + 1025 // 64 * 8 * 4
    many = dict(n=1025, out=1 << 50)
    assert _embed_grad(B, ws=None, **many) == B.EWORKSPACE and _embed_grad(B, ws=FAKE + 8, **many) == B.EWORKSPACE and _embed_grad(B, ws_bytes=need - 1, **many) == B.EWORKSPACE
    # (a token's pieces have a row of sums each)
    assert B.workspace_bytes(B.CALL_EMBED_GRAD, B.BF16, 1 << 20, 1 << 20, 4096) >= (1 << 20) // 64 * 4096 * 4
    assert B.workspace_bytes(B.CALL_EMBED_GRAD, B.F32, 4, 10, 0) == 0
    assert B.scratch_bytes(B.CALL_EMBED_GRAD, B.F32, 1025, 0, 10, 8) == need


def _clip(B, ptrs=(FAKE, FAKE + 4096), numel=(8, 8), dtypes=(0, 1), outs=None, max_norm=1.0, norm=FAR, ws=FAKE, ws_bytes=1 << 20, n=None):
    k = len(ptrs)
    p = (C.c_void_p * k)(*ptrs)
    o = (C.c_void_p * k)(*outs) if outs else None
    return B.lib.picospec_clip_grad(k if n is None else n, p, o, (C.c_int64 * k)(*numel), (C.c_int32 * k)(*dtypes), max_norm, norm, ws, ws_bytes, None)


@pytest.mark.parametrize("kw", [dict(n=-1), dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(norm=None), dict(norm=FAR + 2), dict(numel=(8, -1)), dict(numel=(8, 1 << 45)), dict(ptrs=(FAKE, None)),
                                dict(ptrs=(FAKE + 2, FAKE + 4096)), dict(ptrs=(FAKE, FAKE)), dict(ptrs=(FAKE, FAKE + 31), dtypes=(0, 1)), dict(ptrs=(FAKE + 28, FAKE), dtypes=(0, 0)),
                                dict(outs=(FAKE, None)), dict(outs=(FAKE + 4, FAKE + 4096)), dict(outs=(FAR, FAR + 16)), dict(outs=(FAKE + 4096, FAKE))])
def test_clip_refuses(B, kw):
    assert _clip(B, **kw) == B.EINVAL


def test_clip_refuses_types_and_workspaces(B):
    assert _clip(B, dtypes=(0, 2)) == B.EDTYPE
    assert _clip(B, ws=None) == B.EWORKSPACE and _clip(B, ws=FAKE + 8) == B.EWORKSPACE and _clip(B, ws_bytes=B.workspace_bytes(B.CALL_CLIP_GRAD, 0, 2, 1, 0) - 1) == B.EWORKSPACE
    # the same tensor among many (more than the check keeps on its own stack)
    many = [FAR + 64 * i for i in range(300)]
    assert _clip(B, ptrs=many[:299] + [many[7]], numel=[8] * 300, dtypes=[0] * 300, ws=None) == B.EINVAL
    assert _clip(B, ptrs=many, numel=[8] * 300, dtypes=[0] * 300, ws=None) == B.EWORKSPACE
    assert B.lib.picospec_clip_grad(1, None, None, None, None, 1.0, FAR, FAKE, 1 << 20, None) == B.EINVAL


def test_binding_refuses_tensors_of_the_host(B):
    z, tok = torch.zeros(2, 10), torch.zeros(2, dtype=torch.int32)
    from paper_2603_19133_amd import training as T
    for f in (lambda: B.adjust(z, 10), lambda: B.adjust_grad(z, z, 10), lambda: B.embed(z, tok), lambda: B.embed_grad(z, tok, 5), lambda: B.clip_grad([z], 1.0),
              lambda: T.adjust(z, 10), lambda: T.embed(z, tok)):
        with pytest.raises(B.PicoSpecError) as e:
            f()
        assert e.value.code == B.EINVAL
    with pytest.raises(TypeError):
        B.clip_grad(z, 1.0)
    with pytest.raises(TypeError):
        B.embed(z, 3)
