"""The verify attentions' limit of T * Hq / Hkv query rows where that product does not fit 32 bits (no GPU: every call fails
validation before anything is launched)."""
import ctypes

import pytest

ROWS = 1 << 30          # of the caches, so that a T of 2^28 is no longer than they are
LEN = (ctypes.c_int32 * 1)(ROWS)


@pytest.fixture(scope="module")
def mad():
    import paper_2608_30252_amd as m
    m._load_library()
    return m


def _verify(mad, T, Hq, vt):
    f = mad._load_library().mad_verify_attn_vt if vt else mad._load_library().mad_verify_attn
    p = ctypes.c_void_p
    if vt:
        return f(p(1 << 24), 1, T, Hq, 1, 64, mad.MAD_BF16, 0.125, p(1 << 20), p(1 << 21), ROWS * 64, ROWS * 64, ROWS, LEN, p(1 << 25),
                 None, p(1 << 26), 1 << 40, None)
    view = mad._KVView(1 << 20, 1 << 21, ROWS * 64, ROWS * 64, ROWS, None, LEN)
    return f(p(1 << 24), 1, T, Hq, 1, 64, mad.MAD_BF16, 0.125, ctypes.byref(view), p(1 << 25), None, p(1 << 26), 1 << 40, None)


def _verify8(mad, T, Hq):
    view = mad._KV8View(k=1 << 20, v=1 << 21, k_scale=1 << 22, v_scale=1 << 23, seq_stride=ROWS * 64, head_stride=ROWS * 64,
                        scale_seq_stride=ROWS // 16, scale_head_stride=ROWS // 16, cap=ROWS, block=16, len=LEN)
    p = ctypes.c_void_p
    return mad._load_library().mad_verify_attn_kv8(p(1 << 24), 1, T, Hq, 1, 64, mad.MAD_BF16, 0.125, ctypes.byref(view), p(1 << 25), None,
                                                   p(1 << 26), 1 << 40, None)


def _verify4(mad, T, Hq):
    view = mad._KV4View(k=1 << 20, v=1 << 21, k_scale=1 << 22, v_scale=1 << 23, seq_stride=ROWS * 32, head_stride=ROWS * 32,
                        scale_seq_stride=ROWS * 2, scale_head_stride=ROWS * 2, cap=ROWS, len=LEN)
    p = ctypes.c_void_p
    return mad._load_library().mad_verify_attn_kv4(p(1 << 24), 1, T, Hq, 1, 64, mad.MAD_BF16, 0.125, ctypes.byref(view), p(1 << 25), None,
                                                   p(1 << 26), 1 << 40, None)


CALLS = {"16 bits": lambda m, T, G: _verify(m, T, G, False), "16 bits, transposed V": lambda m, T, G: _verify(m, T, G, True), "8 bits": _verify8, "4 bits": _verify4}


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("T,G", [((1 << 28) + 1, 16), (1 << 28, 16), ((1 << 29) + 8, 8), (1 << 30, 4), ((1 << 28) - 1, 16), (65, 1), (5, 16)])
def test_products_beyond_32_bits_are_refused(mad, call, T, G):
    assert CALLS[call](mad, T, G) == mad.MAD_EINVAL
    assert "must be in [1, 64]" in mad._load_library().mad_last_error().decode()


@pytest.mark.parametrize("op", ["MAD_OP_VERIFY", "MAD_OP_VERIFY_KV4"])
def test_workspaces_of_such_products(mad, op):
    """More rows than a call takes need no more than the most that one takes."""
    ws = lambda T, Hq: mad.workspace_bytes(getattr(mad, op), 1, Hq, 1, 64, T)   # noqa: E731
    for T in ((1 << 28) + 1, 1 << 28, (1 << 28) - 1, 2 ** 31 - 1):
        assert ws(T, 16) >= ws(4, 16) > 0, T
