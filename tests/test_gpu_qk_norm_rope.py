"""Head norms and the rotation on the GPU against float64."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _reference(x, gamma, pos, eps, base, bf16):
    """x [n, H, d] float64, pos [n] ints -> (z, tolerance).  In units e = 2^-24 of the pair's length |y| = |(y_j, y_j+h)|:
    the mean square is a sum of at most 11 roundings (16 products, three exchanges more), the root, the quotient and two
    products 5 more, half of the sum's: 11 e.  The angle: the frequency and the product in fp64, 2^-52 of it, its reduction
    a few 2^-53, then fp32's rounding of a number up to pi, 2 e; sine and cosine 4 e (2 units in the last place, up to 1);
    the rotation 3 e.  Together 20 e, and the output's rounding, 2^-8 (bf16) or e, of z."""
    n, H, d = x.shape
    h = d // 2
    y = x
    if gamma is not None:
        y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gamma
    size = np.hypot(y[..., :h], y[..., h:])
    far = 0.0
    z = y
    if base:
        angle = pos[:, None].astype(np.float64) * base ** (-2.0 * np.arange(h) / d)
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        z = np.concatenate([y[..., :h] * c - y[..., h:] * s, y[..., h:] * c + y[..., :h] * s], -1)
        far = np.abs(angle)[:, None] * 2.0 ** -51
    tol = (20 * 2.0 ** -24 + far) * size
    return z, np.concatenate([tol, tol], -1) + np.abs(z) * (2.0 ** -8 if bf16 else 2.0 ** -24) + 1e-38


def _inputs(B, n_cap, Hq, Hkv, d, dtype, seed, layout):
    g = torch.Generator().manual_seed(seed)
    mk = lambda H: (torch.randn((B, n_cap, H, d), generator=g) * torch.exp(torch.randn((B, n_cap, H, 1), generator=g))).to(TYPES[dtype])   # noqa: E731
    q, k, v = mk(Hq), mk(Hkv), mk(Hkv)
    if layout == "fused":
        q, k, _ = torch.split(torch.cat([q, k, v], 2).cuda(), [Hq, Hkv, Hkv], 2)
        return q, k
    if layout == "rows first":
        return tuple(x.transpose(0, 1).contiguous().cuda().transpose(0, 1) for x in (q, k))
    return q.cuda(), k.cuda()


def _check(B, n_cap, Hq, Hkv, d, dtype, n=None, norm=True, base=1e4, far=5000, rows=False, layout="plain", out="new", seed=0, parts="qk"):
    import paper_2608_30252_amd as mad
    q, k = _inputs(B, n_cap, Hq, Hkv, d, dtype, seed, layout)
    g = torch.Generator().manual_seed(seed + 1)
    gam = [(1 + 0.5 * torch.randn(d, generator=g)).to(TYPES[dtype]) if norm else None for _ in range(2)]
    start = torch.randint(0, far + 1, (B,), generator=g).tolist()
    pos = np.array(start)[:, None] + np.arange(n_cap)
    if rows:
        pos = torch.randint(-far, far + 1, (B, n_cap), generator=g).numpy()
    where = torch.tensor(pos, dtype=torch.int32).cuda() if rows else start
    was = [x.double().cpu().numpy() for x in (q, k)]
    given = {"new": (None, None), "given": tuple(torch.full(x.shape, 5.0, dtype=x.dtype, device="cuda") for x in (q, k)), "in place": (q, k)}[out]
    pick = lambda i, x: x if "qk"[i] in parts else None   # noqa: E731
    got = mad.qk_norm_rope(pick(0, q), pick(1, k), where if base else None, *[pick(i, None if gam[i] is None else gam[i].cuda()) for i in (0, 1)],
                           pick(0, given[0]), pick(1, given[1]), n, 1e-5, base)
    torch.cuda.synchronize()
    for i, x in enumerate(was):
        if pick(i, 1) is None:
            assert got[i] is None
            continue
        res = got[i].double().cpu().numpy()
        for b in range(B):
            m = n_cap if n is None else n[b]
            z, tol = _reference(x[b, :m], None if gam[i] is None else gam[i].double().numpy(), pos[b, :m], 1e-5, base, dtype == "bf16")
            err = np.abs(res[b, :m] - z)
            assert np.all(err <= tol), f"{'qk'[i]} of sequence {b}: {(err / tol).max():.3g} of the bound"
            if out != "new":
                rest = x[b, m:] if out == "in place" else np.full_like(x[b, m:], 5.0)
                assert np.array_equal(res[b, m:], rest)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,n_cap,Hq,Hkv", [(1, 1, 32, 8), (1, 1, 1, 1), (3, 5, 6, 3), (64, 2, 4, 4), (2, 33, 9, 1), (1, 130, 64, 8)])
def test_shapes(B, n_cap, Hq, Hkv, d, dtype):
    _check(B, n_cap, Hq, Hkv, d, dtype)
    _check(B, n_cap, Hq, Hkv, d, dtype, rows=True, seed=3)


@pytest.mark.parametrize("layout", ["plain", "fused", "rows first"])
@pytest.mark.parametrize("out", ["new", "given", "in place"])
def test_layouts_and_uneven_rows(out, layout):
    _check(4, 19, 8, 2, 128, "bf16", n=[19, 0, 1, 7], layout=layout, out=out, seed=5)
    _check(1, 3, 5, 3, 64, "f32", n=[2], layout=layout, out=out, seed=6, rows=True)


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "f32")])
def test_many_tokens(d, dtype):
    # sequences that end anywhere; one round of heads to a wave, two (the last wave of a token one)
    _check(3, 1500, 8, 2, d, dtype, n=[1500, 37, 1111], out="in place", layout="fused", seed=7)
    _check(3, 1500, 64, 3, d, dtype, n=[1500, 37, 1111], out="in place", layout="fused", seed=8)


@pytest.mark.parametrize("parts", ["q", "k"])
@pytest.mark.parametrize("norm,base", [(True, 1e4), (False, 5e5), (True, None), (False, None)])
def test_parts(norm, base, parts):
    _check(2, 6, 8, 2, 128, "bf16", norm=norm, base=base, parts=parts, seed=8)
    _check(2, 6, 8, 2, 64, "f32", norm=norm, base=base, parts=parts, seed=8)


@pytest.mark.parametrize("far", [100_000, 2 ** 31 - 100])
def test_far_positions(far):
    _check(2, 9, 4, 2, 128, "f32", far=far, base=5e5, rows=True, seed=9)
    _check(2, 9, 4, 2, 64, "f32", far=far, base=1.5, seed=10)


def test_zero_rows_and_rows_that_are_not_finite():
    import paper_2608_30252_amd as mad
    x = torch.randn(1, 4, 2, 64, device="cuda")
    x[0, 0] = 0
    x[0, 1, 0, 3] = float("nan")
    x[0, 2, 1] *= 1e-15                      # below eps
    q, _ = mad.qk_norm_rope(x, None, [3], torch.ones(64, device="cuda"))
    assert torch.equal(q[0, 0], torch.zeros(2, 64, device="cuda"))
    assert torch.isnan(q[0, 1, 0]).all() and torch.isfinite(q[0, 1, 1]).all() and torch.isfinite(q[0, 2:]).all()
    z, tol = _reference(x[0, 2:3].double().cpu().numpy(), np.ones(64), np.array([5]), 1e-5, 5e5, False)
    assert np.all(np.abs(q[0, 2:3].double().cpu().numpy() - z) <= tol)
    with pytest.raises(mad.MadError):
        mad.qk_norm_rope(x, None, [3], None, eps=-1.0)


def test_captured_calls_replay():
    import bench
    import paper_2608_30252_amd as mad
    q, k = _inputs(2, 5, 8, 2, 128, "bf16", 11, "fused")
    pos = torch.arange(10, dtype=torch.int32, device="cuda").view(2, 5)
    g = torch.ones(128, dtype=torch.bfloat16, device="cuda")
    qo, ko = torch.empty(q.shape, dtype=q.dtype, device="cuda"), torch.empty(k.shape, dtype=k.dtype, device="cuda")
    step = lambda: mad.qk_norm_rope(q, k, pos, g, g, qo, ko)   # noqa: E731
    step()
    graph = bench.graph_of(torch, step)
    for shift in (0, 1000, 77):              # positions on the device: a replay reads the present ones
        pos.copy_(torch.arange(10, dtype=torch.int32, device="cuda").view(2, 5) + shift)
        want = mad.qk_norm_rope(q, k, pos, g, g)
        qo.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(qo, want[0]) and torch.equal(ko, want[1])
