"""The 4-bit cache on the CPU: its plain reference against closed forms, and what the entry points refuse (every call
fails validation before anything is launched)."""
import ctypes

import numpy as np
import pytest
import torch

import kv4_ref


@pytest.fixture(scope="module")
def mad():
    import paper_2608_30252_amd as m
    m._load_library()
    return m


# ------------------------------------------------------------ the reference ----

def test_reference_codes_are_the_nearest():
    x = np.concatenate([np.linspace(-6, 6, 4801), [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -5.0, -0.0]])
    x = np.resize(x, (151, 32))
    x[:, 0] = 6.0                                                       # the scale is 1
    codes, scale = kv4_ref.encode(x)
    assert np.all(scale == 127)
    got = kv4_ref.values(codes, scale)
    every = np.concatenate([kv4_ref.LEVELS, -kv4_ref.LEVELS])
    best = np.abs(x[..., None] - every).min(-1)
    assert np.array_equal(np.abs(got - x), best)
    ties = dict(zip([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0]))   # the even code
    for a, want in ties.items():
        row = np.full(32, a)
        row[0] = 6.0
        assert kv4_ref.values(*kv4_ref.encode(row))[1] == want and kv4_ref.values(*kv4_ref.encode(-row))[1] == -want


@pytest.mark.parametrize("m,want", [(0.0, -100), (6.0, 0), (6.0001, 1), (3.0, -1), (1e-38, -100), (3.4e38, 125), (1.5, -2), (1.50001, -1)])
def test_reference_scale(m, want):
    assert kv4_ref.least_scale(m) == want


def test_reference_bytes():
    x = np.zeros((1, 64))
    x[0, 0], x[0, 1], x[0, 33], x[0, 40] = 6.0, -1.5, 12.0, np.inf
    codes, scale = kv4_ref.encode(x)
    assert codes[0, 0] == 0x07 | (0x0b << 4) and np.all(codes[0, 1:] == 0) and list(scale[0]) == [127, 255]
    v = kv4_ref.values(codes, scale)[0]
    assert v[0] == 6 and v[1] == -1.5 and np.isnan(v[32:]).all()


# ------------------------------------------------------------------ refusals ----

LEN = (ctypes.c_int32 * 64)(*([20] * 64))
p = lambda x: ctypes.c_void_p(x) if x else None   # noqa: E731


def _view(mad, **kw):
    a = dict(k=1 << 20, v=1 << 21, k_scale=1 << 22, v_scale=1 << 23, seq_stride=2 * 64 * 32, head_stride=64 * 32,
             scale_seq_stride=2 * 64 * 2, scale_head_stride=64 * 2, cap=64, len=LEN)
    a.update(kw)
    return mad._KV4View(*[a[f] for f, _ in mad._KV4View._fields_])


def _rows(mad, at=1 << 24, seq=4 * 128, row=128):
    return mad._Rows(at, seq, row)


def _append(mad, view=None, n=None, k=None, v=None, kh=None, vh=None, **kw):
    a = dict(B=2, n_cap=4, Hkv=2, d=64, dtype=mad.MAD_BF16)
    a.update(kw)
    ref = lambda r: None if r is None else ctypes.byref(r)   # noqa: E731
    k = _rows(mad) if k is None else k
    v = _rows(mad, 1 << 25) if v is None else v
    return mad._load_library().mad_kv4_append(ref(k) if k else None, ref(v) if v else None, ref(kh), ref(vh), n, a["B"], a["n_cap"],
                                              a["Hkv"], a["d"], a["dtype"], ref(view), None)


def _verify(mad, view=None, **kw):
    a = dict(q=1 << 24, B=2, T=2, Hq=8, Hkv=2, d=64, dtype=mad.MAD_BF16, scale=0.125, out=1 << 25, lse=0, ws=1 << 26, ws_bytes=1 << 30)
    a.update(kw)
    return mad._load_library().mad_verify_attn_kv4(p(a["q"]), a["B"], a["T"], a["Hq"], a["Hkv"], a["d"], a["dtype"], a["scale"],
                                                   ctypes.byref(view) if view is not None else None, p(a["out"]), p(a["lse"]),
                                                   p(a["ws"]), a["ws_bytes"], None)


BAD_VIEWS = [dict(k=0), dict(v=0), dict(k_scale=0), dict(v_scale=0), dict(k=(1 << 20) + 8), dict(v_scale=(1 << 23) + 1), dict(cap=0),
             dict(len=None), dict(head_stride=64 * 32 - 16), dict(head_stride=64 * 32 + 8), dict(seq_stride=2 * 64 * 32 + 8),
             dict(seq_stride=-16), dict(seq_stride=64 * 32), dict(scale_head_stride=126), dict(scale_head_stride=129),
             dict(scale_seq_stride=-2), dict(scale_seq_stride=128), dict(scale_seq_stride=257), dict(scale_seq_stride=0),
             dict(len=(ctypes.c_int32 * 2)(1, 65)), dict(len=(ctypes.c_int32 * 2)(-1, 5))]


@pytest.mark.parametrize("change", BAD_VIEWS)
def test_both_refuse_a_bad_view(mad, change):
    assert _append(mad, _view(mad, **change)) == mad.MAD_EINVAL
    assert _verify(mad, _view(mad, **change)) == mad.MAD_EINVAL


def test_scales_of_long_rows_are_aligned_to_their_four_bytes(mad):
    base = dict(seq_stride=2 * 64 * 64, head_stride=64 * 64, scale_seq_stride=2 * 64 * 4, scale_head_stride=64 * 4)
    for bad in (dict(k_scale=(1 << 22) + 2), dict(scale_head_stride=64 * 4 + 2), dict(scale_seq_stride=2 * 64 * 4 + 2)):
        assert _verify(mad, _view(mad, **{**base, **bad}), d=128) == mad.MAD_EINVAL, bad


def test_append_refuses(mad):
    v = _view(mad)
    i32 = lambda *x: (ctypes.c_int32 * len(x))(*x)   # noqa: E731
    assert _append(mad, None) == mad.MAD_EINVAL
    for kw in (dict(B=0), dict(B=65), dict(n_cap=0), dict(Hkv=0), dict(k=False), dict(v=False), dict(k=_rows(mad, 0)),
               dict(k=_rows(mad, (1 << 24) + 8)), dict(v=_rows(mad, row=120)), dict(v=_rows(mad, row=132)), dict(k=_rows(mad, seq=-8)),
               dict(k=_rows(mad, seq=516)), dict(k=_rows(mad, row=1 << 41)), dict(kh=_rows(mad)), dict(vh=_rows(mad)),
               dict(kh=_rows(mad), vh=_rows(mad, seq=0)), dict(kh=_rows(mad, seq=3 * 128), vh=_rows(mad))):
        assert _append(mad, v, **kw) == mad.MAD_EINVAL, kw
    assert _append(mad, v, d=96) == mad.MAD_ENOTSUP and _append(mad, v, dtype=3) == mad.MAD_ENOTSUP
    assert _append(mad, v, i32(1, 5)) == mad.MAD_EINVAL          # more than n_cap
    assert _append(mad, v, i32(-1, 1)) == mad.MAD_EINVAL
    assert _append(mad, v, n_cap=45) == mad.MAD_EINVAL           # 20 + 45 > 64
    assert "exceeds cap" in mad._load_library().mad_last_error().decode()
    cap = 1 << 29                                                # 2^24 tiles of 128 rows, K and V of 2 heads
    huge = _view(mad, cap=cap, head_stride=cap * 32, seq_stride=2 * cap * 32, scale_head_stride=cap * 2, scale_seq_stride=cap * 4, len=i32(0, 0))
    assert _append(mad, huge, i32(0, cap), n_cap=cap) == mad.MAD_EINVAL
    assert "more than a call takes" in mad._load_library().mad_last_error().decode()
    shared = _view(mad, seq_stride=0, scale_seq_stride=0)
    assert _append(mad, shared) == mad.MAD_EINVAL                # two sequences write one buffer
    for lay in (dict(), dict(seq=128, row=256)):                 # sequence by sequence, row by row
        kh, vh = _rows(mad, **lay), _rows(mad, 1 << 25, **lay)
        assert _append(mad, v, i32(0, 0), kh=kh, vh=vh) == mad.MAD_OK       # nothing to do: nothing is launched
    # what would be written twice, or written while it is read
    a, b, c = _rows(mad), _rows(mad, 1 << 25), _rows(mad, 1 << 26)
    for kh, vh in ((c, c), (b, c), (c, a)):
        assert _append(mad, v, i32(0, 0), kh=kh, vh=vh) == mad.MAD_EINVAL
    for one in (dict(v=1 << 20), dict(v_scale=1 << 22)):
        assert _append(mad, _view(mad, **one), i32(0, 0)) == mad.MAD_EINVAL


def test_verify_refuses(mad):
    v = _view(mad)
    assert _verify(mad, None) == mad.MAD_EINVAL
    for kw in (dict(B=0), dict(B=65), dict(T=0), dict(T=17), dict(Hq=7), dict(q=0), dict(out=0), dict(q=(1 << 24) + 4),
               dict(out=(1 << 25) + 8), dict(lse=(1 << 27) + 2), dict(scale=0.0), dict(scale=float("nan")), dict(scale=float("inf")),
               dict(ws=(1 << 26) + 8)):
        assert _verify(mad, v, **kw) == mad.MAD_EINVAL, kw
    assert _verify(mad, v, d=96) == mad.MAD_ENOTSUP and _verify(mad, v, dtype=3) == mad.MAD_ENOTSUP
    assert _verify(mad, v, Hq=6) == mad.MAD_ENOTSUP              # group 3
    assert _verify(mad, v, scale=2.0 ** 127 * 1.9) == mad.MAD_EINVAL           # times log2 e beyond fp32
    many = _view(mad, seq_stride=64 * 32 << 20, scale_seq_stride=128 << 20)
    assert _verify(mad, many, Hq=1 << 20, Hkv=1 << 20) == mad.MAD_EINVAL
    assert "more than a call takes" in mad._load_library().mad_last_error().decode()
    assert _verify(mad, v, ws=0) == mad.MAD_EWS
    need = mad.workspace_bytes(mad.MAD_OP_VERIFY_KV4, 2, 8, 2, 64, 2)
    assert _verify(mad, v, ws_bytes=need - 1) == mad.MAD_EWS


def test_binding_refuses(mad):
    q = torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16)
    x = torch.zeros(2, 3, 2, 64, dtype=torch.bfloat16)
    kv = mad.KV4.empty(2, 2, 40, 64, device="cpu")
    assert kv.k.shape == (2, 2, 40, 32) and kv.k_scale.shape == (2, 2, 40, 2)
    bad = lambda **kw: mad.KV4(**{**dict(k=kv.k, v=kv.v, k_scale=kv.k_scale, v_scale=kv.v_scale, length=[3, 3]), **kw})   # noqa: E731
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)   # noqa: E731
    for kw, match in ((dict(k=kv.k.char(), v=kv.v.char()), "uint8"), (dict(k_scale=kv.k_scale[:, :, :39]), "scales must be"),
                      (dict(v=kv.v[:, :1]), "identical strides"), (dict(k_scale=kv.k_scale.float()), "uint8"), (dict(length=[3]), "one entry per row"),
                      (dict(k=u8(2, 2, 40, 64)[..., :32], v=u8(2, 2, 40, 64)[..., :32]), "rows must be contiguous"),
                      (dict(v_scale=u8(2, 2, 44, 2)[:, :, :40]), "identical strides")):
        with pytest.raises(ValueError, match=match):
            mad.verify_attn_kv4(q, bad(**kw))
        with pytest.raises(ValueError, match=match):
            mad.kv4_append(x, x, bad(**kw))
    with pytest.raises(ValueError, match="batch dimension"):
        mad.verify_attn_kv4(q[:1].expand(3, 3, 4, 64).contiguous(), bad(length=[1, 1, 1]))
    with pytest.raises(ValueError, match="head_dim"):
        mad.kv4_append(torch.zeros(2, 3, 2, 128), torch.zeros(2, 3, 2, 128), kv)
    with pytest.raises(ValueError, match="KV heads"):
        mad.kv4_append(x[:, :, :1], x[:, :, :1], kv)
    with pytest.raises(ValueError, match="multiple of the KV heads"):
        mad.verify_attn_kv4(q[:, :, :3].contiguous(), kv)
    with pytest.raises(ValueError, match="match k_new"):
        mad.kv4_append(x, x.float(), kv)
    with pytest.raises(ValueError, match="go together"):
        mad.kv4_append(x, x, kv, k_held=x)
    with pytest.raises(ValueError, match="heads must be contiguous"):
        mad.kv4_append(x.transpose(1, 2).contiguous().transpose(1, 2), x, kv)
    with pytest.raises(ValueError, match="one entry per sequence"):
        mad.kv4_append(x, x, kv, [1])
    with pytest.raises(TypeError, match="dtype"):
        mad.kv4_append(x.half(), x.half(), kv)
