"""Sampling on the GPU against plain float64 (sample_ref.py): tokens exactly, probabilities to fp32 rounding, and which
entries stay exactly.  (A draw or a cut could differ only where a uniform or top_p lies within some 1e-13 of an edge.)"""
import numpy as np
import pytest
import torch

import sample_ref

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _mad():
    import paper_2608_30252_amd as mad
    return mad


def _logits(kind, shape, seed):
    g = torch.Generator().manual_seed(seed)
    V = shape[-1]
    x = torch.randn(shape, generator=g)
    if kind == "model":      # a body under a Zipf-like head
        m = min(200, V)
        at = torch.rand(shape, generator=g).topk(m, dim=-1).indices
        head = 15 - 2 * torch.log(torch.arange(1, m + 1).float()) + 0.7 * torch.randn(shape[:-1] + (m,), generator=g)
        return (2.2 * x).scatter_(-1, at, head)
    if kind == "flat":       # thousands of entries to a bin
        return 0.01 * x
    if kind == "body":
        return 0.5 * x
    if kind == "wide":       # a few entries to many bins, most below the window of 32
        return 30 * x
    if kind == "ties":       # eight values only
        return torch.randint(0, 8, shape, generator=g).float()
    if kind == "equal":
        return torch.full(shape, -3.25)
    if kind == "masked":     # a grammar leaves few entries
        keep = torch.rand(shape, generator=g) < max(3.0 / V, 1e-9)
        keep[..., V // 2] = True
        return torch.where(keep, 3 * x, torch.tensor(-float("inf")))
    if kind == "lowest":     # masks of the type's lowest value, one row all of it
        x = torch.where(torch.rand(shape, generator=g) < 0.5, 3 * x, torch.tensor(torch.finfo(torch.bfloat16).min))
        x[0, 0] = torch.finfo(torch.bfloat16).min
        return x
    if kind == "huge":       # beyond the range of the bins, and no two far from equal in weight
        return 1e30 + 1e24 * x
    if kind == "spike":      # one entry 60 above the rest
        x[..., V // 3] = 60.0
        return x
    if kind == "infinite":
        x[..., ::max(1, V // 3)] = float("inf")
        return x
    raise ValueError(kind)


def _check(x, u, tok, probs, T=1, what="", **kw):
    """Every row; kw: a list per sequence or a number for all."""
    B = x.shape[0]
    for b in range(B):
        one = {k: (v[b] if isinstance(v, list) else v) for k, v in kw.items()}
        for t in range(x.shape[1]):
            sample_ref.check_row(x[b, t].double().numpy(), None if u is None else float(u[b, t]),
                                 None if tok is None else int(tok[b, t]), None if probs is None else probs[b, t].numpy(),
                                 f"{what} row ({b}, {t})", **one)


def _run(kind, shape, dtype, seed, probs=True, tok=True, **kw):
    mad = _mad()
    x = _logits(kind, shape, seed).to(TYPES[dtype])
    u = torch.rand(shape[:2], generator=torch.Generator().manual_seed(seed + 1)) if tok else None
    out = torch.full(shape, float("nan"), device="cuda") if probs else None
    got, p = mad.sample(x.cuda(), None if u is None else u.cuda(), probs=out, **kw)
    torch.cuda.synchronize()
    _check(x, u, None if got is None else got.cpu(), None if p is None else p.cpu(), what=kind, **kw)


SETTINGS = [dict(), dict(temperature=0.7), dict(top_k=1), dict(top_k=40), dict(top_k=128, temperature=1.3), dict(top_k=129),
            dict(top_k=3000, top_p=0.97), dict(top_p=0.9), dict(top_p=0.5, temperature=2.0), dict(top_p=1e-9), dict(top_p=0.99999),
            dict(min_p=0.05), dict(min_p=1.0), dict(top_k=50, top_p=0.9, min_p=0.02), dict(top_p=0.95, min_p=0.3), dict(temperature=0),
            dict(top_k=200, min_p=0.01), dict(temperature=0.05, top_k=20)]


@pytest.mark.parametrize("kw", SETTINGS, ids=lambda k: ",".join(f"{a}={b}" for a, b in k.items()) or "none")
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_settings(dtype, kw):
    _run("model", (2, 2, 20000), dtype, 1, **kw)
    _run("model", (1, 3, 9001), dtype, 2, probs=False, **kw)


@pytest.mark.parametrize("kind", ["flat", "wide", "ties", "equal", "masked", "lowest", "huge", "spike", "infinite"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_distributions(dtype, kind):
    for i, kw in enumerate((dict(top_k=40), dict(top_k=100, top_p=0.8), dict(top_k=700, top_p=0.9), dict(top_p=0.9), dict(min_p=0.4),
                            dict(top_p=0.6, min_p=0.2), dict(), dict(temperature=0), dict(temperature=40.0, top_k=60))):
        _run(kind, (2, 1, 17000), dtype, 10 + i, probs=i % 2 == 0, **kw)
        _run(kind, (1, 2, 700), dtype, 30 + i, **kw)


@pytest.mark.parametrize("kind", ["model", "body", "wide", "ties", "masked", "lowest", "spike"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_filters_of_any_strength_together(dtype, kind):
    # top-k of 1 .. V with top-p close to 0, in between and close to 1, and a min-p above and below both
    rng = np.random.default_rng(len(kind))
    for i in range(12):
        V = int(rng.choice([300, 9000, 20000]))
        kw = dict(temperature=float(np.exp(rng.normal(0, 0.7))), top_k=int(np.exp(rng.uniform(0, np.log(V)))),
                  top_p=float(rng.choice([rng.uniform(0, 1), 1 - 10 ** rng.uniform(-6, -2), 10 ** rng.uniform(-6, -2)])),
                  min_p=float(rng.choice([0.0, 10 ** rng.uniform(-6, 0)])))
        _run(kind, (2, 2, V), dtype, 70 + i, probs=i % 2 == 0, **kw)


def test_a_top_k_beyond_32_bits_keeps_all():
    mad = _mad()
    x, u = _logits("model", (2, 1, 5000), 3).cuda(), torch.rand((2, 1), device="cuda")
    want = mad.sample(x, u, probs=torch.empty_like(x))
    for k in (5000, 2 ** 31 - 1, 2 ** 32, 2 ** 32 + 1, [2 ** 40, 0]):
        got = mad.sample(x, u, top_k=k, probs=torch.empty_like(x))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    with pytest.raises(mad.MadError):
        mad.sample(x, u, top_k=-2 ** 32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_entries_to_a_bin_than_are_listed(dtype):
    # thousands within an eighth: the range where a filter ends is searched on in the row, for two filters one after the
    # other; where min-p ends above top-k, top-p is still of top-k's mass
    for i, kw in enumerate((dict(top_p=0.9), dict(top_p=0.6, temperature=0.3), dict(top_k=3000), dict(top_k=3000, top_p=0.8),
                            dict(top_k=3000, top_p=0.8, min_p=0.5), dict(top_k=200, top_p=0.3, min_p=0.9), dict(min_p=0.1), dict(top_k=128))):
        _run("body", (2, 1, 40000), dtype, 50 + i, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 63, 1000, 4096, 4097, 8191, 8192, 8193, 16385, 50257, 128256])
def test_sizes(V, dtype):
    for i, kw in enumerate((dict(top_k=5), dict(top_p=0.9), dict(), dict(top_k=max(1, V - 1)), dict(top_k=V), dict(min_p=0.1), dict(temperature=0))):
        _run("model", (1, 2 if V < 60000 else 1, V), dtype, V + i, probs=i != 3, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_min_p_alone(dtype):
    # few to a chunk; chunks whose own best would leave hundreds, none of which the row keeps; rows that keep thousands;
    # next to all; all but the masked
    for i, (kind, kw) in enumerate((("model", dict(min_p=0.1)), ("model", dict(min_p=0.02, temperature=1.2)), ("model", dict(min_p=1e-3, temperature=1.5)),
                                    ("model", dict(min_p=1e-12)), ("masked", dict(min_p=1e-9)), ("lowest", dict(min_p=1e-300)), ("body", dict(min_p=0.3)),
                                    ("wide", dict(min_p=1e-4, temperature=30.0)), ("infinite", dict(min_p=0.5)), ("huge", dict(min_p=0.01)))):
        _run(kind, (2, 2, 40000), dtype, 120 + i, probs=i % 2 == 0, **kw)


@pytest.mark.parametrize("V", [600001, 1 << 20])
def test_the_largest_vocabularies(V):
    # more chunks than a wave has lanes; all of them
    for i, kw in enumerate((dict(top_k=128, top_p=0.9), dict(top_p=0.95), dict(top_k=1000), dict(top_k=1000, top_p=0.5), dict(min_p=0.01),
                            dict(), dict(temperature=0))):
        _run("model", (1, 1, V), ("bf16", "f32")[i % 2], 90 + i, probs=i % 3 == 0, **kw)
    _run("body", (1, 1, V), "f32", 97, top_p=0.9)


def test_every_sequence_its_own_settings():
    B = 64
    kw = dict(temperature=[0.0 if b % 7 == 0 else 0.5 + 0.02 * b for b in range(B)], top_k=[(0, 30, 200, 1, 5000)[b % 5] for b in range(B)],
              top_p=[(1.0, 0.9, 0.99)[b % 3] for b in range(B)], min_p=[(0.0, 0.05)[b % 2] for b in range(B)])
    _run("model", (B, 1, 9000), "bf16", 50, **kw)
    _run("model", (B, 1, 9000), "f32", 51, probs=False, **kw)
    _run("model", (B, 1, 9000), "f32", 52, tok=False, **kw)


def test_many_rows():
    _run("model", (20, 64, 130), "f32", 53, top_k=10, top_p=0.9)
    _run("model", (20, 64, 130), "bf16", 54, top_p=0.9)


def test_uniforms_at_both_ends():
    mad = _mad()
    x = _logits("model", (1, 4, 30000), 55)
    u = torch.tensor([[0.0, 1 - 2.0 ** -24, 0.5, 2.0 ** -30]])
    for kw in (dict(), dict(top_k=7), dict(top_p=0.9), dict(top_p=0.9, min_p=0.2)):
        tok, p = mad.sample(x.cuda(), u.cuda(), probs=torch.empty(1, 4, 30000, device="cuda"), **kw)
        only, _ = mad.sample(x.cuda(), u.cuda(), **kw)
        torch.cuda.synchronize()
        assert torch.equal(tok, only)
        _check(x, u, tok.cpu(), p.cpu(), **kw)


def test_rows_without_a_distribution():
    mad = _mad()
    V = 20000
    x = _logits("model", (1, 5, V), 56)
    x[0, 1, 12345], x[0, 2], x[0, 4, 0] = float("nan"), -float("inf"), float("nan")
    u = torch.full((1, 5), 0.4)
    for kw in (dict(top_k=20), dict(top_p=0.9), dict(), dict(top_k=3000), dict(min_p=0.1), dict(temperature=0)):
        tok, p = mad.sample(x.cuda(), u.cuda(), probs=torch.full((1, 5, V), 7.0, device="cuda"), **kw)
        alone, _ = mad.sample(x.cuda(), u.cuda(), **kw)
        torch.cuda.synchronize()
        assert tok[0].tolist()[1] == tok[0].tolist()[2] == tok[0].tolist()[4] == -1 and torch.equal(tok, alone)
        _check(x, u, tok.cpu(), p.cpu(), **kw)


def test_unaligned_rows():
    # views that start at any element, rows of odd length
    mad = _mad()
    for dtype in ("bf16", "f32"):
        for off in (1, 3):
            V = 9001
            x = _logits("model", (1, 3, V), 57 + off).to(TYPES[dtype])
            buf = torch.full((3 * V + 8,), 1e9, dtype=TYPES[dtype], device="cuda")
            buf[off:off + 3 * V] = x.flatten().cuda()
            out = torch.full((3 * V + 8,), -1.0, device="cuda")
            u = torch.rand(1, 3, generator=torch.Generator().manual_seed(9))
            for kw in (dict(top_k=9), dict(top_p=0.9)):
                out.fill_(-1.0)
                tok, p = mad.sample(buf[off:off + 3 * V].view(1, 3, V), u.cuda(), probs=out[off:off + 3 * V].view(1, 3, V), **kw)
                torch.cuda.synchronize()
                _check(x, u, tok.cpu(), p.cpu(), **kw)
                assert bool((out[:off] == -1).all() and (out[off + 3 * V:] == -1).all())


def test_the_same_bits_every_time():
    mad = _mad()
    x = _logits("model", (4, 2, 50257), 58).cuda()
    u = torch.rand(4, 2, device="cuda")
    body = _logits("body", (4, 2, 50257), 59).cuda()      # (by passes over the row)
    for x, kw in ((x, dict(top_k=100, top_p=0.9)), (x, dict(top_p=0.95)), (x, dict(top_k=900)), (x, dict()), (x, dict(top_k=900, top_p=0.7)),
                  (body, dict(top_p=0.9)), (body, dict(top_k=9000, top_p=0.9))):
        first = None
        for _ in range(5):
            tok, p = mad.sample(x, u, probs=torch.empty_like(x), **kw)
            torch.cuda.synchronize()
            if first is None:
                first = tok.clone(), p.clone()
            assert torch.equal(first[0], tok) and torch.equal(first[1], p)


def test_graph_replays():
    mad = _mad()
    B, T, V = 3, 2, 30000
    x, u = torch.empty(B, T, V, device="cuda"), torch.empty(B, T, device="cuda")
    kw = dict(temperature=[1.0, 0.8, 0.0], top_k=[50, 0, 0], top_p=[0.9, 0.95, 1.0], min_p=[0.0, 0.0, 0.0])
    nbytes = mad.workspace_bytes(mad.MAD_OP_SAMPLE, B, T=T, max_keys=V)
    graphs = []
    for _ in range(2):   # two graphs, a workspace each
        tok, p, ws = torch.zeros(B, T, dtype=torch.int32, device="cuda"), torch.zeros(B, T, V, device="cuda"), torch.zeros(nbytes, dtype=torch.uint8, device="cuda")
        x.copy_(_logits("model", (B, T, V), 1)), u.fill_(0.3)
        mad.sample(x, u, **kw, tok=tok, probs=p, ws=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            mad.sample(x, u, **kw, tok=tok, probs=p, ws=ws)
        graphs.append((g, tok, p, ws))
    for r in range(4):
        x.copy_(_logits("model", (B, T, V), 60 + r))
        u.copy_(torch.rand(B, T, generator=torch.Generator().manual_seed(r)))
        for g, tok, p, _ in graphs:
            p.fill_(float("nan"))
            g.replay()
        torch.cuda.synchronize()
        want, wp = mad.sample(x, u, **kw, probs=torch.empty_like(x))
        torch.cuda.synchronize()
        for g, tok, p, _ in graphs:
            assert torch.equal(tok, want) and torch.equal(p, wp), f"replay {r}"
        _check(x.cpu(), u.cpu(), want.cpu(), wp.cpu(), **kw)


def test_side_stream_and_both_marshalling_paths(monkeypatch):
    mad = _mad()
    x = _logits("model", (2, 3, 20000), 70).cuda()
    u = torch.rand(2, 3, device="cuda")
    kw = dict(temperature=[0.9, 1.1], top_k=[0, 64], top_p=0.9, min_p=(0.0, 0.01))
    want, wp = mad.sample(x, u, **kw, probs=torch.empty_like(x))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for path in ("native", "ctypes"):
        if path == "ctypes":
            monkeypatch.setattr(mad, "_FAST", mad._CtypesOnly())
        tok, p = torch.zeros_like(want), torch.zeros_like(wp)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            mad.sample(x, u, **kw)          # (the stream's workspace)
            mad.sample(x, u, **kw, tok=tok, probs=p)
        side.synchronize()
        assert torch.equal(tok, want) and torch.equal(p, wp), path


def test_ordinary_calls_take_the_native_path():
    mad = _mad()
    fast = mad._fast()
    x, u = torch.randn(2, 2, 500, device="cuda"), torch.rand(2, 2, device="cuda")
    tok, p = torch.empty(2, 2, dtype=torch.int32, device="cuda"), torch.empty_like(x)
    mad.sample(x, u)
    for args in ((u, 0.7, 20, 0.9, 0.0, tok, p), (u, [0.7, 1.0], [0, 3], (1.0, 0.9), [0.0, 0.1], tok, None), (None, 1, 0, 1, 0, None, p)):
        assert fast.sample(x, *args, None) == mad.MAD_OK
    assert fast.sample(x, u, np.array([1.0, 1.0]), 0, 1.0, 0.0, tok, p, None) is None
    torch.cuda.synchronize()


def test_a_workspace_serves_other_calls_before_and_after():
    mad = _mad()
    V = 20000
    ws = torch.zeros(mad.workspace_bytes(mad.MAD_OP_SAMPLE, 2, T=2, max_keys=V), dtype=torch.uint8, device="cuda")
    x = _logits("model", (2, 2, V), 80).cuda()
    u = torch.rand(2, 2, device="cuda")
    draft = torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    am = x.argmax(-1)
    for _ in range(3):
        na, nt = mad.accept_greedy(x, draft, ws=ws)
        tok, p = mad.sample(x, u, top_p=0.9, probs=torch.empty_like(x), ws=ws)
        na2, nt2 = mad.accept_stochastic(p, p[:, :1].contiguous(), draft, u, ws=ws)
        torch.cuda.synchronize()
        assert torch.equal(nt, torch.where(na == 1, am[:, 1], am[:, 0]).to(torch.int32))
        _check(x.cpu(), u.cpu(), tok.cpu(), p.cpu(), top_p=0.9)
