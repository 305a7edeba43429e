"""picospec_distill / picospec_distill_grad without a GPU: every misuse that the host can see is refused before anything is launched."""
import pytest

FAKE = 0x1000                                    # (never dereferenced: the calls fail their checks first)


@pytest.fixture(scope="module")
def B():
    from paper_2603_19133_amd import binding
    return binding


def _distill(B, z=FAKE, dt=0, ld=100, rows=2, V=100, T=1.0, rec=(FAKE,) * 3, k=10, tail=0, w=None, loss=FAKE, acc=None, stats=None, grad=None, ldg=100, ws=None):
    return B.lib.picospec_distill(z, dt, ld, rows, V, T, *rec, k, tail, w, loss, acc, stats, grad, ldg, ws, 0, None)


def _grad(B, z=FAKE, dt=0, ld=100, rows=2, V=100, T=1.0, rec=(FAKE,) * 3, k=10, tail=0, w=None, stats=FAKE, grad=FAKE, ldg=100):
    return B.lib.picospec_distill_grad(z, dt, ld, rows, V, T, *rec, k, tail, w, stats, grad, ldg, None)


@pytest.mark.parametrize("call", [_distill, _grad])
def test_misuse_is_refused(B, call):
    assert call(B, z=None) == B.EINVAL
    assert call(B, dt=2) == B.EDTYPE
    assert call(B, ld=99) == B.EINVAL
    assert call(B, rows=-1) == B.EINVAL
    assert call(B, V=0) == B.EINVAL
    assert call(B, z=FAKE + 2) == B.EINVAL                       # fp32 base off the 4-byte boundary
    assert call(B, V=(1 << 20) + 1, ld=1 << 21, ldg=1 << 21) == B.EUNSUPPORTED
    for T in (0.0, -1.0, float("nan"), float("inf")):
        assert call(B, T=T) == B.EINVAL
    assert call(B, k=0) == B.EINVAL and call(B, k=101) == B.EINVAL
    assert call(B, V=10000, ld=10000, ldg=10000, k=4097) == B.EUNSUPPORTED
    assert call(B, tail=2) == B.EINVAL and call(B, tail=-1) == B.EINVAL
    for i in range(3):
        rec = [FAKE] * 3
        rec[i] = None
        assert call(B, rec=tuple(rec)) == B.EINVAL
    assert call(B, stats=FAKE + 4) == B.EINVAL                   # four words a row, stored at once
    assert call(B, grad=FAKE, ldg=99) == B.EINVAL
    assert call(B, grad=FAKE + 2) == B.EINVAL


def test_outputs_are_required(B):
    assert _distill(B, ws=FAKE + 4) == B.EWORKSPACE
    assert _distill(B, loss=None) == B.EINVAL
    assert _grad(B, stats=None) == B.EINVAL
    assert _grad(B, grad=None) == B.EINVAL


def test_calls_of_no_rows_do_nothing(B):
    assert _distill(B, z=None, rows=0, rec=(None,) * 3, loss=None) == B.OK
    assert _grad(B, z=None, rows=0, rec=(None,) * 3, stats=None, grad=None) == B.OK


def test_streaming_loads_stay_inside_the_row(B):
    """The kernels' own rule of what their row loads address, evaluated on the host over every lane, look-ahead included."""
    for dtype, esz in ((B.F32, 4), (B.BF16, 2)):
        for V in (1, 2, 7, 8, 9, 255, 256, 257, 1025, 2047, 4096, 8191, 8193, 16384, 16387, 32000, 65537, 131073, 151936, (1 << 20) - 1, 1 << 20):
            for mis in range(0, 16, esz):
                end = B.max_load_byte(B.CALL_DISTILL, dtype, V, mis)
                assert V * esz - 15 <= end <= (mis + V * esz + 15) // 16 * 16 - mis, (dtype, V, mis, end)
    assert B.max_load_byte(B.CALL_DISTILL, B.F32, 0, 0) == -1 and B.max_load_byte(B.CALL_DISTILL, B.BF16, 100, 3) == -1
