"""Outputs at their input's place with other strides (no GPU: every call is refused, or has no row to write): a row would be
written over one that is still to be read."""
import ctypes

import pytest

ROW, SEQ = 16 * 64, 5 * 16 * 64      # a fused projection's rows


@pytest.fixture(scope="module")
def mad():
    import paper_2608_30252_amd as m
    m._load_library()
    return m


def i32(*x):
    return (ctypes.c_int32 * len(x))(*x)


def _norm(mad, which, out, n):
    """mad_qk_norm_rope on rows of 4 or 2 heads of 64, 2 sequences of up to 5 rows."""
    lib, ref = mad._load_library(), ctypes.byref
    x, y = mad._Rows(1 << 24, SEQ, ROW), mad._Rows(1 << 24, *out)
    q, k = ((ref(x), ref(y)), (None, None)) if which == "q" else ((None, None), (ref(x), ref(y)))
    return lib.mad_qk_norm_rope(q[0], k[0], q[1], k[1], None, None, 1e-5, 1e4, i32(0, 9), None, n, 2, 5, 4, 2, 64, mad.MAD_BF16, None)


def _append(mad, which, out, n):
    """mad_kv4_append with the values held; `which` of them at its new rows' place, the other elsewhere."""
    lib, ref = mad._load_library(), ctypes.byref
    view = mad._KV4View(k=1 << 20, v=1 << 21, k_scale=1 << 22, v_scale=1 << 23, seq_stride=2 * 64 * 32, head_stride=64 * 32,
                        scale_seq_stride=2 * 64 * 2, scale_head_stride=64 * 2, cap=64, len=i32(0, 3))
    k, v = mad._Rows(1 << 24, SEQ, ROW), mad._Rows(1 << 25, SEQ, ROW)
    kh = mad._Rows(1 << 24, *out) if which == "k" else mad._Rows(1 << 26, SEQ, ROW)
    vh = mad._Rows(1 << 25, *out) if which == "v" else mad._Rows(1 << 26, SEQ, ROW)
    return lib.mad_kv4_append(ref(k), ref(v), ref(kh), ref(vh), n, 2, 5, 2, 64, mad.MAD_BF16, ref(view), None)


CALLS = {"norm of q": (_norm, "q"), "norm of k": (_norm, "k"), "append, K": (_append, "k"), "append, V": (_append, "v")}


@pytest.mark.parametrize("call", CALLS)
def test_other_strides_in_place_are_refused(mad, call):
    f, which = CALLS[call]
    for out, n in (((5 * 256, 256), None),                  # compact, over the front of the projection
                   ((SEQ, 256), None), ((SEQ, 256), i32(0, 2)), ((2 * SEQ, ROW), None), ((2 * SEQ, 2 * ROW), i32(2, 0)),
                   ((2 * SEQ, ROW), i32(0, 1)), ((5 * 256, 256), i32(1, 1))):
        assert f(mad, which, out, n) == mad.MAD_EINVAL, (out, None if n is None else list(n))
        assert "other strides" in mad._load_library().mad_last_error().decode()


@pytest.mark.parametrize("call", CALLS)
def test_no_rows_to_write_are_no_error(mad, call):
    f, which = CALLS[call]
    for out in ((SEQ, ROW), (5 * 256, 256), (2 * SEQ, ROW)):
        assert f(mad, which, out, i32(0, 0)) == mad.MAD_OK
