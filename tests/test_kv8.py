"""The 8-bit cache on the CPU: its plain reference against torch's e4m3, and what the entry points refuse (every
call fails validation before anything is launched)."""
import ctypes

import numpy as np
import pytest
import torch

import kv8_ref


@pytest.fixture(scope="module")
def mad():
    import paper_2608_30252_amd as m
    m._load_library()
    return m


# ------------------------------------------------------------ the reference ----

def test_reference_codes_are_torchs():
    c = torch.arange(256, dtype=torch.uint8)
    want = c.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(kv8_ref.decode(c.numpy()), want, equal_nan=True)
    g = torch.Generator().manual_seed(1)
    x = torch.randn(20000, generator=g) * torch.exp(3 * torch.randn(20000, generator=g))
    fine = want[np.isfinite(want)]
    near = np.concatenate([fine, (fine[:-1] + fine[1:]) / 2])          # every value and every midpoint of two codes' values
    x = torch.cat([x.clamp(-448, 448), torch.from_numpy(near).float(), torch.tensor([float("nan"), -0.0, 0.0])])
    got = kv8_ref.encode(x.double().numpy())
    assert np.array_equal(got, x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())


@pytest.mark.parametrize("m,want", [(0.0, 2.0 ** -100), (448.0, 1.0), (448.1, 2.0), (449.0 / 2, 1.0), (224.0, 0.5),
                                    (1e-38, 2.0 ** -100), (3.3e38, 2.0 ** 120), (1.75, 2.0 ** -8), (1.7501, 2.0 ** -7)])
def test_reference_scale(m, want):
    assert kv8_ref.least_scale(m) == want


def test_reference_append_rewrites_a_block_that_outgrows_its_scale():
    codes, scale = np.zeros((1, 32, 64), np.uint8), np.ones((1, 2))
    kv8_ref.append(codes, scale, np.full((3, 1, 64), 1.75), 0, 3, 16)
    assert scale[0, 0] == 2.0 ** -8 and np.all(kv8_ref.values(codes, scale, 16)[0, :3] == 1.75)
    kv8_ref.append(codes, scale, np.full((14, 1, 64), 7.0), 3, 14, 16)     # 13 rows fill the block, one starts the next
    v = kv8_ref.values(codes, scale, 16)[0]
    assert scale[0, 0] == 2.0 ** -6 and scale[0, 1] == 2.0 ** -6
    assert np.all(v[:3] == 1.75) and np.all(v[3:17] == 7.0) and np.all(v[17:] == 0)


# ------------------------------------------------------------------ refusals ----

LEN = (ctypes.c_int32 * 64)(*([20] * 64))


def _view(mad, **kw):
    a = dict(k=1 << 20, v=1 << 21, k_scale=1 << 22, v_scale=1 << 23, seq_stride=2 * 64 * 64, head_stride=64 * 64,
             scale_seq_stride=8, scale_head_stride=4, cap=64, block=16, len=LEN)
    a.update(kw)
    return mad._KV8View(*[a[f] for f, _ in mad._KV8View._fields_])


def _append(mad, view=None, n=None, **kw):
    a = dict(k_new=1 << 24, v_new=1 << 25, B=2, n_cap=4, Hkv=2, d=64, dtype=mad.MAD_BF16)
    a.update(kw)
    p = lambda x: ctypes.c_void_p(x) if x else None   # noqa: E731
    return mad._load_library().mad_kv8_append(p(a["k_new"]), p(a["v_new"]), n, a["B"], a["n_cap"], a["Hkv"], a["d"], a["dtype"],
                                              ctypes.byref(view) if view is not None else None, None)


def _verify(mad, view=None, **kw):
    a = dict(q=1 << 24, B=2, T=2, Hq=8, Hkv=2, d=64, dtype=mad.MAD_BF16, scale=0.125, out=1 << 25, ws=1 << 26, ws_bytes=1 << 30)
    a.update(kw)
    p = lambda x: ctypes.c_void_p(x) if x else None   # noqa: E731
    return mad._load_library().mad_verify_attn_kv8(p(a["q"]), a["B"], a["T"], a["Hq"], a["Hkv"], a["d"], a["dtype"], a["scale"],
                                                   ctypes.byref(view) if view is not None else None, p(a["out"]), None,
                                                   p(a["ws"]), a["ws_bytes"], None)


BAD_VIEWS = [(dict(k=0), "EINVAL"), (dict(v=0), "EINVAL"), (dict(k_scale=0), "EINVAL"), (dict(v_scale=0), "EINVAL"),
             (dict(k=(1 << 20) + 8), "EINVAL"), (dict(v_scale=(1 << 23) + 2), "EINVAL"), (dict(cap=0), "EINVAL"),
             (dict(block=0), "ENOTSUP"), (dict(block=8), "ENOTSUP"), (dict(block=48), "ENOTSUP"), (dict(block=256), "ENOTSUP"),
             (dict(len=None), "EINVAL"), (dict(head_stride=64 * 64 - 16), "EINVAL"), (dict(head_stride=64 * 64 + 8), "EINVAL"),
             (dict(seq_stride=2 * 64 * 64 + 8), "EINVAL"), (dict(seq_stride=-16), "EINVAL"), (dict(seq_stride=64 * 64), "EINVAL"),
             (dict(scale_head_stride=3), "EINVAL"), (dict(scale_seq_stride=-1), "EINVAL"), (dict(scale_seq_stride=4), "EINVAL"),
             (dict(scale_seq_stride=0), "EINVAL"), (dict(len=(ctypes.c_int32 * 2)(1, 65)), "EINVAL"),
             (dict(len=(ctypes.c_int32 * 2)(-1, 5)), "EINVAL")]


@pytest.mark.parametrize("change,code", BAD_VIEWS)
def test_both_refuse_a_bad_view(mad, change, code):
    want = getattr(mad, "MAD_" + code)
    assert _append(mad, _view(mad, **change)) == want
    assert _verify(mad, _view(mad, **change)) == want


def test_append_refuses(mad):
    v = _view(mad)
    i32 = lambda *x: (ctypes.c_int32 * len(x))(*x)   # noqa: E731
    assert _append(mad, None) == mad.MAD_EINVAL
    for kw in (dict(B=0), dict(B=65), dict(n_cap=0), dict(Hkv=0), dict(k_new=0), dict(v_new=0), dict(k_new=(1 << 24) + 8)):
        assert _append(mad, v, **kw) == mad.MAD_EINVAL, kw
    assert _append(mad, v, d=96) == mad.MAD_ENOTSUP and _append(mad, v, dtype=3) == mad.MAD_ENOTSUP
    assert _append(mad, v, i32(1, 5)) == mad.MAD_EINVAL          # more than n_cap
    assert _append(mad, v, i32(-1, 1)) == mad.MAD_EINVAL
    assert _append(mad, v, n_cap=45) == mad.MAD_EINVAL           # 20 + 45 > 64
    assert "exceeds cap" in mad._load_library().mad_last_error().decode()
    assert _append(mad, v, i32(0, 45), n_cap=45) == mad.MAD_EINVAL
    cap = 1 << 26                                                # 2^22 blocks of 2 heads, K and V: 2^24 workgroups
    huge = _view(mad, cap=cap, head_stride=cap * 64, seq_stride=2 * cap * 64, scale_head_stride=cap // 16, scale_seq_stride=cap // 8,
                 len=i32(0, 0))
    assert _append(mad, huge, i32(0, cap), n_cap=cap) == mad.MAD_EINVAL
    assert "more than a call takes" in mad._load_library().mad_last_error().decode()
    shared = _view(mad, seq_stride=0, scale_seq_stride=0)
    assert _append(mad, shared) == mad.MAD_EINVAL                # two sequences write one buffer
    assert _append(mad, v, i32(0, 0)) == mad.MAD_OK              # nothing to do: nothing is launched


def test_verify_refuses(mad):
    v = _view(mad)
    assert _verify(mad, None) == mad.MAD_EINVAL
    for kw in (dict(B=0), dict(B=65), dict(T=0), dict(T=17), dict(Hq=7), dict(q=0), dict(out=0), dict(q=(1 << 24) + 4),
               dict(out=(1 << 25) + 8), dict(scale=0.0), dict(scale=float("nan")), dict(ws=(1 << 26) + 8)):
        assert _verify(mad, v, **kw) == mad.MAD_EINVAL, kw
    assert _verify(mad, v, d=96) == mad.MAD_ENOTSUP and _verify(mad, v, dtype=3) == mad.MAD_ENOTSUP
    assert _verify(mad, v, Hq=6) == mad.MAD_ENOTSUP              # group 3
    assert _verify(mad, v, ws=0) == mad.MAD_EWS
    need = mad.workspace_bytes(mad.MAD_OP_VERIFY, 2, 8, 2, 64, 2)
    assert _verify(mad, v, ws_bytes=need - 1) == mad.MAD_EWS


def _cache(mad, B=2, Hkv=2, cap=40, d=64, block=16):
    return mad.KV8.empty(B, Hkv, cap, d, block, device="cpu")


def test_binding_refuses(mad):
    q = torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16)
    x = torch.zeros(2, 3, 2, 64, dtype=torch.bfloat16)
    kv = _cache(mad)
    assert kv.k.shape == (2, 2, 40, 64) and kv.k_scale.shape == (2, 2, 3)
    bad = lambda **kw: mad.KV8(**{**dict(k=kv.k, v=kv.v, k_scale=kv.k_scale, v_scale=kv.v_scale, length=[3, 3], block=16), **kw})   # noqa: E731
    f8 = torch.float8_e4m3fn
    for kw, match in ((dict(k=kv.k.view(torch.uint8), v=kv.v.view(torch.uint8)), "float8_e4m3fn"), (dict(block=32), "scales must be"),
                      (dict(block=20), "block"), (dict(k_scale=kv.k_scale[:1]), "scales must be"), (dict(v=kv.v[:, :1]), "identical strides"),
                      (dict(k_scale=kv.k_scale.double(), v_scale=kv.v_scale.double()), "float32"), (dict(length=[3]), "one entry per row"),
                      (dict(k=torch.zeros(2, 2, 40, 128, dtype=torch.uint8).view(f8)[..., :64], v=torch.zeros(2, 2, 40, 128, dtype=torch.uint8).view(f8)[..., :64]), "rows must be contiguous")):
        with pytest.raises(ValueError, match=match):
            mad.verify_attn_kv8(q, bad(**kw))
        with pytest.raises(ValueError, match=match):
            mad.kv8_append(x, x, bad(**kw))
    with pytest.raises(ValueError, match="batch dimension"):
        mad.verify_attn_kv8(q[:1].expand(3, 3, 4, 64).contiguous(), bad(length=[1, 1, 1]))
    with pytest.raises(ValueError, match="head_dim"):
        mad.kv8_append(torch.zeros(2, 3, 2, 128), torch.zeros(2, 3, 2, 128), kv)
    with pytest.raises(ValueError, match="KV heads"):
        mad.kv8_append(x[:, :, :1].contiguous(), x[:, :, :1].contiguous(), kv)
    with pytest.raises(ValueError, match="multiple of the KV heads"):
        mad.verify_attn_kv8(q[:, :, :3].contiguous(), kv)
    with pytest.raises(ValueError, match="one type"):
        mad.kv8_append(x, x.float(), kv)
    with pytest.raises(ValueError, match="contiguous"):
        mad.kv8_append(x.transpose(0, 1).contiguous().transpose(0, 1), x, kv)
    with pytest.raises(ValueError, match="one entry per sequence"):
        mad.kv8_append(x, x, kv, [1])
    with pytest.raises(TypeError, match="dtype"):
        mad.kv8_append(x.half(), x.half(), kv)
    with pytest.raises(IndexError):
        mad.verify_attn_kv8(q, bad(length=[3, 3, 3]))
