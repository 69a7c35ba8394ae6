"""Sampling on the CPU: the plain reference against closed forms, and what the entry point refuses."""
import ctypes

import numpy as np
import pytest
import torch

import sample_ref


@pytest.fixture(scope="module")
def mad():
    import paper_2608_30252_amd as m
    m._load_library()
    return m


def test_reference_against_closed_forms():
    x = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    tok, p = sample_ref.row(x, 0.5)
    assert tok in (1, 2) and np.allclose(p, [0.1, 0.4, 0.2, 0.3])   # cumulative 0.1, 0.5: on the edge
    assert sample_ref.row(x, 0.5 + 1e-6)[0] == 2 and sample_ref.row(x, 0.5 - 1e-6)[0] == 1 and sample_ref.row(x, 0.0)[0] == 0
    assert np.allclose(sample_ref.row(x, 0.0, top_k=2)[1], [0, 4 / 7, 0, 3 / 7])
    assert np.allclose(sample_ref.row(x, 0.0, top_p=0.69)[1], [0, 4 / 7, 0, 3 / 7])
    assert np.allclose(sample_ref.row(x, 0.0, top_p=0.71)[1], [0, 4 / 9, 2 / 9, 3 / 9])
    assert np.allclose(sample_ref.row(x, 0.0, min_p=0.49)[1], [0, 4 / 9, 2 / 9, 3 / 9])
    assert np.allclose(sample_ref.row(x, 0.0, top_k=2, top_p=0.57)[1], [0, 1, 0, 0])   # of the top two's mass
    assert np.allclose(sample_ref.row(x, 0.0, temperature=0.5)[1], np.array([1, 16, 4, 9]) / 30)
    assert sample_ref.row(x, 0.9, temperature=0)[0] == 1


def test_reference_ties_and_rows_without_a_distribution():
    x = np.array([1.0, 2.0, 2.0, 2.0, 0.0])
    assert np.allclose(sample_ref.row(x, 0.0, top_k=2)[1], [0, 0.5, 0.5, 0, 0])
    assert np.allclose(sample_ref.row(x, 0.0, temperature=0)[1], [0, 1, 0, 0, 0])
    assert sample_ref.row(np.array([-np.inf, -np.inf]), 0.5)[0] == -1
    assert sample_ref.row(np.array([1.0, np.nan]), 0.5)[0] == -1
    assert np.allclose(sample_ref.row(np.array([np.inf, 1.0, np.inf]), 0.6)[1], [0.5, 0, 0.5])


# ------------------------------------------------------------------ refusals ----

def _call(mad, B=2, T=3, V=1000, dtype=None, logits=1 << 22, u=1 << 20, t=None, k=None, p=None, mp=None, tok=1 << 21,
          probs=1 << 26, ws=1 << 28, ws_bytes=1 << 40):
    q = lambda x: ctypes.c_void_p(x) if x else None   # noqa: E731
    f = lambda v: None if v is None else (ctypes.c_double * len(v))(*v)   # noqa: E731
    i = None if k is None else (ctypes.c_int32 * len(k))(*k)
    return mad._load_library().mad_sample(q(logits), mad.MAD_F32 if dtype is None else dtype, q(u), f(t), i, f(p), f(mp), B, T, V,
                                          q(tok), q(probs), q(ws), ws_bytes, None)


def test_entry_point_refuses(mad):
    nan, inf = float("nan"), float("inf")
    for kw in (dict(B=0), dict(B=65), dict(T=0), dict(T=65), dict(V=0), dict(V=(1 << 20) + 1), dict(logits=0), dict(u=0),
               dict(tok=0, probs=0), dict(logits=(1 << 22) + 2), dict(u=(1 << 20) + 2), dict(tok=(1 << 21) + 1), dict(probs=(1 << 26) + 2),
               dict(t=[1, -1]), dict(t=[nan, 1]), dict(t=[1, inf]), dict(k=[0, -1]), dict(p=[1, 0]), dict(p=[1.5, 1]), dict(p=[nan, 1]),
               dict(mp=[0, -0.1]), dict(mp=[1.1, 0]), dict(mp=[0, nan]), dict(ws=(1 << 28) + 64), dict(probs=(1 << 22) + 4 * 5999)):
        assert _call(mad, **kw) == mad.MAD_EINVAL, kw
    assert _call(mad, dtype=5) == mad.MAD_ENOTSUP
    assert _call(mad, dtype=mad.MAD_BF16, logits=(1 << 22) + 1) == mad.MAD_EINVAL
    assert _call(mad, ws=0) == mad.MAD_EWS
    assert _call(mad, ws_bytes=mad.workspace_bytes(mad.MAD_OP_SAMPLE, 2, T=3, max_keys=1000) - 1) == mad.MAD_EWS


def test_workspace(mad):
    ws = lambda B, T, V: mad.workspace_bytes(mad.MAD_OP_SAMPLE, B, T=T, max_keys=V)   # noqa: E731
    assert ws(1, 1, 1) > (1 << 20) and ws(2, 3, 50000) > ws(2, 3, 8192) > ws(1, 3, 8192)
    assert ws(0, 1, 10) == ws(65, 1, 10) == ws(1, 65, 10) == ws(1, 1, 0) == ws(1, 1, (1 << 20) + 1) == 0


def test_binding_refuses(mad):
    x, u = torch.zeros(2, 3, 10), torch.zeros(2, 3)
    with pytest.raises(ValueError, match="logits must be"):
        mad.sample(x[0], u)
    with pytest.raises(ValueError, match="u must be"):
        mad.sample(x, u[:1])
    with pytest.raises(ValueError, match="needs the uniforms"):
        mad.sample(x, None, tok=torch.zeros(2, 3, dtype=torch.int32))
    with pytest.raises(ValueError, match="tok must be"):
        mad.sample(x, u, tok=torch.zeros(2, 3))
    with pytest.raises(ValueError, match="probs must be"):
        mad.sample(x, u, probs=torch.zeros(2, 3, 9))
    with pytest.raises(ValueError, match="top_k needs one entry"):
        mad.sample(x, u, top_k=[1, 2, 3])
    with pytest.raises(ValueError, match="temperature needs one entry"):
        mad.sample(x, u, temperature=[1.0])
    with pytest.raises(ValueError, match="contiguous"):
        mad.sample(x.transpose(0, 1).contiguous().transpose(0, 1), u)
    with pytest.raises(TypeError, match="dtype"):
        mad.sample(x.half(), u)
