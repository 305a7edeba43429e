"""picospec_sample without a GPU: every misuse that the host can see is refused before anything is launched."""
import pytest

FAKE = 0x1000                                    # (never dereferenced: the calls fail their checks first)
NAN = float("nan")


@pytest.fixture(scope="module")
def B():
    from paper_2603_19133_amd import binding
    return binding


def _sample(B, z=FAKE, dt=0, ld=100, rows=2, V=100, T=1.0, k=0, p=0.0, m=0.0, per_row=(None,) * 4, u=FAKE, outs=(FAKE,) * 4, ws=None, ws_bytes=0):
    return B.lib.picospec_sample(z, dt, ld, rows, V, T, k, p, m, *per_row, u, *outs, ws, ws_bytes, None)


def test_misuse_is_refused(B):
    assert _sample(B, z=None) == B.EINVAL
    assert _sample(B, dt=3) == B.EDTYPE
    assert _sample(B, ld=99) == B.EINVAL
    assert _sample(B, rows=-1) == B.EINVAL
    assert _sample(B, V=0) == B.EINVAL
    assert _sample(B, z=FAKE + 1, dt=1) == B.EINVAL              # bf16 base off the 2-byte boundary
    assert _sample(B, V=(1 << 20) + 1, ld=1 << 21) == B.EUNSUPPORTED
    for T in (-1.0, NAN, float("inf")):
        assert _sample(B, T=T) == B.EINVAL
    assert _sample(B, p=NAN) == B.EINVAL
    assert _sample(B, m=NAN) == B.EINVAL and _sample(B, m=1.5) == B.EINVAL
    assert _sample(B, u=None) == B.EINVAL
    for i in range(4):
        outs = [FAKE] * 4
        outs[i] = None
        assert _sample(B, outs=tuple(outs)) == B.EINVAL
    assert _sample(B, ws=FAKE + 8, ws_bytes=1 << 20) == B.EWORKSPACE


def test_a_call_of_no_rows_does_nothing(B):
    assert _sample(B, z=None, rows=0, u=None, outs=(None,) * 4) == B.OK
    assert _sample(B, z=None, rows=0, T=0.0, u=None, outs=(None,) * 4) == B.OK        # (greedy)
    assert _sample(B, z=None, rows=0, T=NAN, p=NAN, m=NAN, per_row=(FAKE, None, FAKE, FAKE), u=None, outs=(None,) * 4) == B.OK   # (per row)


def test_streaming_loads_stay_inside_the_row(B):
    """The kernels' own rule of what their row loads address, evaluated on the host over every lane, look-ahead included."""
    for dtype, esz in ((B.F32, 4), (B.BF16, 2)):
        for V in (1, 2, 7, 8, 9, 255, 256, 257, 1025, 2047, 4096, 8191, 8193, 16384, 16387, 32000, 65537, 131073, 151936, (1 << 20) - 1, 1 << 20):
            for mis in range(0, 16, esz):
                end = B.max_load_byte(B.CALL_SAMPLE, dtype, V, mis)
                assert V * esz - 15 <= end <= (mis + V * esz + 15) // 16 * 16 - mis, (dtype, V, mis, end)
    assert B.max_load_byte(B.CALL_SAMPLE, B.F32, 0, 0) == -1 and B.max_load_byte(B.CALL_SAMPLE, B.BF16, 100, 3) == -1
