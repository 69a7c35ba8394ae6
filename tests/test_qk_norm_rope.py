"""What mad_qk_norm_rope and its binding refuse (no GPU: every call fails validation before anything is launched)."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def mad():
    import paper_2608_30252_amd as m
    m._load_library()
    return m


def _call(mad, **kw):
    rows = lambda at, h: mad._Rows(at, 5 * 16 * 64, 16 * 64)   # noqa: E731
    a = dict(q=rows(1 << 24, 4), k=rows(1 << 25, 2), qo=rows(1 << 26, 4), ko=rows(1 << 27, 2), qg=1 << 20, kg=1 << 21, eps=1e-5, base=1e4,
             start=(ctypes.c_int32 * 2)(0, 9), pos=None, n=None, B=2, n_cap=5, Hq=4, Hkv=2, d=64, dtype=mad.MAD_BF16)
    a.update(kw)
    p = lambda x: ctypes.c_void_p(x) if x else None   # noqa: E731
    ref = lambda r: None if r is None else ctypes.byref(r)   # noqa: E731
    return mad._load_library().mad_qk_norm_rope(ref(a["q"]), ref(a["k"]), ref(a["qo"]), ref(a["ko"]), p(a["qg"]), p(a["kg"]), a["eps"], a["base"],
                                                a["start"], p(a["pos"]), a["n"], a["B"], a["n_cap"], a["Hq"], a["Hkv"], a["d"], a["dtype"], None)


def test_refusals(mad):
    R = mad._Rows
    i32 = lambda *x: (ctypes.c_int32 * len(x))(*x)   # noqa: E731
    row, seq = 16 * 64, 5 * 16 * 64
    for kw in (dict(B=0), dict(B=65), dict(n_cap=0), dict(Hq=0), dict(Hkv=-1), dict(Hq=5000), dict(q=None), dict(ko=None), dict(q=None, k=None, qo=None, ko=None),
               dict(q=R(0, seq, row)), dict(qo=R((1 << 26) + 8, seq, row)), dict(k=R(1 << 25, seq, 2 * 64 - 8)), dict(q=R(1 << 24, seq, row + 4)),
               dict(q=R(1 << 24, seq + 4, row)), dict(q=R(1 << 24, -8, row)), dict(qo=R(1 << 26, row, row)), dict(qo=R(1 << 26, 0, row)),
               dict(ko=R(1 << 27, 4 * row, row)), dict(qg=(1 << 20) + 2), dict(eps=-1e-5), dict(eps=float("nan")), dict(eps=float("inf")), dict(base=1.0),
               dict(base=-2.0), dict(base=float("inf")), dict(base=float("nan")), dict(start=None), dict(pos=1 << 22), dict(start=None, pos=(1 << 22) + 2),
               dict(n=i32(6, 0)), dict(n=i32(0, -1)), dict(start=i32(0, 2 ** 31 - 4)), dict(n_cap=1 << 24, q=R(1 << 24, 1 << 39, row),
               k=R(1 << 24, 1 << 39, row), qo=R(1 << 24, 1 << 39, row), ko=R(1 << 24, 1 << 39, row))):
        assert _call(mad, **kw) == mad.MAD_EINVAL, kw
    assert _call(mad, d=96) == mad.MAD_ENOTSUP and _call(mad, dtype=3) == mad.MAD_ENOTSUP
    none = i32(0, 0)
    for kw in (dict(ko=R(1 << 26, seq, row)), dict(qo=R(1 << 25, seq, row)), dict(ko=R(1 << 24, seq, row))):   # written twice, or while it is read
        assert _call(mad, n=none, **kw) == mad.MAD_EINVAL, kw
    assert _call(mad, n=none) == mad.MAD_OK                                    # nothing to do: nothing is launched
    assert _call(mad, n=none, qo=R(1 << 26, 256, 512)) == mad.MAD_OK           # rows first, the sequences inside a row
    assert _call(mad, n=none, q=R(1 << 24, 0, row)) == mad.MAD_OK              # read only: sequences may share rows
    assert _call(mad, n=none, base=0.0, start=None) == mad.MAD_OK              # no rotation, no positions


def test_binding_refuses(mad):
    q, k, g = torch.zeros(2, 3, 4, 64), torch.zeros(2, 3, 2, 64), torch.zeros(64)
    f = mad.qk_norm_rope
    for args, kw, match in (((None, None, [0, 0]), {}, "neither"), ((q, k[:1], [0, 0]), {}, "alike"), ((q, k.bfloat16(), [0, 0]), {}, "alike"),
                            ((q, k), {}, "needs pos"), ((q, k, [0]), {}, "one first position"), ((q, k, torch.zeros(2, 3)), {}, "int32"),
                            ((q, k, torch.zeros(2, 4, dtype=torch.int32)), {}, "int32"), ((q, k, [0, 0], g[:32]), {}, "q_gamma must be"),
                            ((q, k, [0, 0], None, g.bfloat16()), {}, "k_gamma must be"), ((q, None, [0, 0], None, g), {}, "k_gamma goes with k"),
                            ((q, None, [0, 0], None, None, None, k), {}, "k_out goes with k"), ((q, k, [0, 0]), dict(q_out=k), "q_out must match"),
                            ((q, k, [0, 0]), dict(n=[1]), "one entry per sequence"),
                            ((q.transpose(1, 2).contiguous().transpose(1, 2), k, [0, 0]), {}, "heads must be contiguous")):
        with pytest.raises(ValueError, match=match):
            f(*args, **kw)
    with pytest.raises(TypeError, match="dtype"):
        f(q.half(), k.half(), [0, 0])
