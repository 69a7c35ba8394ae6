"""The log-probability reference against closed forms, and what mad_token_logprobs and its binding refuse (no GPU: every
call fails validation before anything is launched)."""
import ctypes

import numpy as np
import pytest
import torch

import logprobs_ref


@pytest.fixture(scope="module")
def mad():
    import paper_2608_30252_amd as m
    m._load_library()
    return m


def test_reference_closed_forms():
    r = logprobs_ref.row(np.zeros(8), 3, 3, 0.7)
    assert abs(r["logp"] + np.log(8)) < 1e-15 and abs(r["entropy"] - np.log(8)) < 1e-15 and r["rank"] == 3 and list(r["top_tok"]) == [0, 1, 2]
    r = logprobs_ref.row([0.0, np.log(3.0)], 0, 2, 1.0)
    assert abs(r["logp"] - np.log(0.25)) < 1e-15 and r["rank"] == 1 and np.allclose(r["top_logp"], np.log([0.75, 0.25]))
    r = logprobs_ref.row([0.0, 2 * np.log(3.0)], 1, 0, 2.0)
    assert abs(r["logp"] - np.log(0.75)) < 1e-15 and r["rank"] == 0
    r = logprobs_ref.row([1.0, np.inf, -np.inf, np.inf], 3, 3, 1.0)
    assert abs(r["logp"] + np.log(2)) < 1e-15 and list(r["top_tok"]) == [1, 3, 0] and np.isneginf(r["top_logp"][2]) and abs(r["entropy"] - np.log(2)) < 1e-15
    assert logprobs_ref.row([1.0, 2.0], -1, 0, 1.0)["rank"] == 2 and np.isneginf(logprobs_ref.row([1.0, 2.0], 2, 0, 1.0)["logp"])
    for x in ([np.nan, 1.0], [-np.inf, -np.inf]):
        r = logprobs_ref.row(x, 0, 1, 1.0)
        assert np.isnan(r["logp"]) and r["rank"] == -1 and np.isnan(r["entropy"]) and r["top_tok"][0] == -1


def _call(mad, **kw):
    a = dict(logits=1 << 24, dtype=mad.MAD_BF16, seq=3 * 1000, row=1000, tok=1 << 20, temp=None, B=2, T=3, V=1000, top=5, logp=1 << 21, rank=1 << 22,
             entropy=1 << 23, top_tok=1 << 25, top_logp=1 << 26, ws=1 << 28, ws_bytes=1 << 30)
    a.update(kw)
    p = lambda x: ctypes.c_void_p(x) if x else None   # noqa: E731
    return mad._load_library().mad_token_logprobs(p(a["logits"]), a["dtype"], a["seq"], a["row"], p(a["tok"]), a["temp"], a["B"], a["T"], a["V"], a["top"],
                                                  p(a["logp"]), p(a["rank"]), p(a["entropy"]), p(a["top_tok"]), p(a["top_logp"]), p(a["ws"]),
                                                  a["ws_bytes"], None)


def test_refusals(mad):
    f64 = lambda *x: (ctypes.c_double * len(x))(*x)   # noqa: E731
    for kw in (dict(B=0), dict(B=65), dict(T=0), dict(B=64, T=(1 << 16) + 1), dict(V=0), dict(V=(1 << 20) + 1), dict(top=-1), dict(top=65), dict(V=4),
               dict(logits=0), dict(logits=(1 << 24) + 1), dict(logits=(1 << 24) + 2, dtype=mad.MAD_F32), dict(tok=(1 << 20) + 2), dict(top_logp=(1 << 26) + 1),
               dict(seq=-1), dict(row=-1), dict(row=1 << 41), dict(tok=0), dict(top=0), dict(top_tok=0), dict(top_logp=0),
               dict(tok=0, logp=0, rank=0, entropy=0, top=0, top_tok=0, top_logp=0), dict(ws=(1 << 28) + 128),
               dict(temp=f64(1.0, 0.0)), dict(temp=f64(-1.0, 1.0)), dict(temp=f64(1.0, float("nan"))), dict(temp=f64(float("inf"), 1.0))):
        assert _call(mad, **kw) == mad.MAD_EINVAL, kw
    assert _call(mad, dtype=3) == mad.MAD_ENOTSUP
    assert _call(mad, ws=0) == mad.MAD_EWS and _call(mad, ws_bytes=mad.workspace_bytes(mad.MAD_OP_LOGPROBS, 2, T=3, max_keys=1000) - 1) == mad.MAD_EWS


def test_workspace(mad):
    ws = lambda B, T, V: mad.workspace_bytes(mad.MAD_OP_LOGPROBS, B, T=T, max_keys=V)   # noqa: E731
    assert ws(0, 1, 10) == 0 and ws(65, 1, 10) == 0 and ws(1, 0, 10) == 0 and ws(1, 1, 0) == 0 and ws(1, 1, (1 << 20) + 1) == 0
    assert (1 << 20) <= ws(64, 4096, 128256) < (1 << 20) + (1 << 22) and ws(1, 1, 50257) > 1 << 20


def test_binding_refuses(mad):
    x, tok = torch.zeros(2, 3, 100), torch.zeros(2, 3, dtype=torch.int32)
    f = mad.token_logprobs
    for args, kw, match in (((x[0], tok), {}, r"\[B, T, V\]"), ((x.transpose(1, 2), tok[:, :1]), {}, "rows must be contiguous"), ((x, tok[:, :2]), {}, "tok must be"),
                            ((x, tok.long()), {}, "tok must be"), ((x, None), dict(logp=torch.zeros(2, 3)), "need tok"), ((x, tok, 65), {}, "top_n=65"),
                            ((x, tok, -1), {}, "top_n=-1"), ((x[..., :7], tok, 8), {}, "top_n=8"), ((x, tok, 0), dict(top_tok=tok), "need top_n"),
                            ((x, tok, 2), dict(top_tok=torch.zeros(2, 3, 3, dtype=torch.int32)), "top_tok must be"), ((x, tok, 2), dict(entropy=tok), "entropy must be"),
                            ((x, tok, 0, [1.0]), {}, "one entry per sequence"), ((x, torch.zeros(3, 2, dtype=torch.int32).t()), {}, "tok must be contiguous")):
        with pytest.raises(ValueError, match=match):
            f(*args, **kw)
    with pytest.raises(TypeError, match="dtype"):
        f(x.half(), tok, ws=torch.zeros(1 << 22, dtype=torch.uint8))
