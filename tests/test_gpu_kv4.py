"""The 4-bit cache on the GPU against plain float64 (kv4_ref.py): appends are exact, codes, scales and the values held;
attention is within kv4_ref.tolerances, derived there."""
import numpy as np
import pytest
import torch

import kv4_ref

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _mad():
    import paper_2608_30252_amd as mad
    return mad


def _rows(shape, seed, spread=1.0):
    """N(0, 1) rows whose size varies by exp(spread N(0, 1))."""
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g) * torch.exp(spread * torch.randn(shape[:-1] + (1,), generator=g))


def _bytes(B, Hkv, cap, d, seed, lo=121, hi=126):
    """A cache full of codes and scale bytes in [lo, hi)."""
    g = torch.Generator().manual_seed(seed)
    mk = lambda n, a, b: torch.randint(a, b, (B, Hkv, cap, n), generator=g, dtype=torch.uint8)   # noqa: E731
    return mk(d // 2, 0, 256), mk(d // 2, 0, 256), mk(d // 32, lo, hi), mk(d // 32, lo, hi)


# ------------------------------------------------------------------ append ----

def _append_case(d, dtype, lens, n, n_cap, Hkv=2, seed=0, edit=None, held="none", layout="plain"):
    mad = _mad()
    B = len(lens)
    cap = max(l + m for l, m in zip(lens, n)) + 3
    k, v, ks, vs = _bytes(B, Hkv, cap, d, seed)
    new = [_rows((B, n_cap, Hkv, d), seed + i).to(TYPES[dtype]) for i in (1, 2)]
    if edit:
        edit(*new)
    if layout == "fused":          # views of one projection: queries of 3 heads first
        whole = torch.cat([torch.zeros(B, n_cap, 3, d, dtype=TYPES[dtype]), *new], 2).cuda()
        kn, vn = whole[:, :, 3:3 + Hkv], whole[:, :, 3 + Hkv:]
    elif layout == "rows first":   # [n_cap, B, Hkv, d]
        kn, vn = (x.transpose(0, 1).contiguous().cuda().transpose(0, 1) for x in new)
    else:
        kn, vn = (x.cuda() for x in new)
    before = [x.clone() for x in (kn, vn)]
    hold = {"none": (None, None), "own": tuple(torch.full((B, n_cap, Hkv, d), 7.0, dtype=TYPES[dtype], device="cuda") for _ in range(2)),
            "in place": (kn, vn)}[held]
    kv = mad.KV4(k.cuda(), v.cuda(), ks.cuda(), vs.cuda(), list(lens))
    mad.kv4_append(kn, vn, kv, None if n == [n_cap] * B else n, *hold)
    torch.cuda.synchronize()
    for name, codes, scale, x, got, got_s, h, b4 in (("k", k, ks, new[0], kv.k, kv.k_scale, hold[0], before[0]),
                                                     ("v", v, vs, new[1], kv.v, kv.v_scale, hold[1], before[1])):
        want, want_s = codes.numpy().copy(), scale.numpy().copy()
        want_h = (torch.full(x.shape, 7.0) if held == "own" else b4.cpu()).double().numpy()
        for b in range(B):
            c, s = kv4_ref.encode(x[b, :n[b]].double().numpy())
            want[b, :, lens[b]:lens[b] + n[b]] = c.transpose(1, 0, 2)
            want_s[b, :, lens[b]:lens[b] + n[b]] = s.transpose(1, 0, 2)
            want_h[b, :n[b]] = kv4_ref.values(c, s)
        assert np.array_equal(got_s.cpu().numpy(), want_s), f"{name}: scales"
        assert np.array_equal(got.cpu().numpy(), want), f"{name}: {int((got.cpu().numpy() != want).sum())} bytes differ"
        if h is not None:
            assert np.array_equal(h.double().cpu().numpy(), want_h, equal_nan=True), f"{name}: values held"
            zero = want_h == 0
            assert np.array_equal(np.signbit(h.double().cpu().numpy())[zero], np.signbit(want_h)[zero])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_append_lengths(d, dtype):
    _append_case(d, dtype, [0, 1, 15, 16, 37, 7, 3], [1, 15, 2, 33, 70, 0, 64], 70, seed=d)


@pytest.mark.parametrize("layout", ["plain", "fused", "rows first"])
@pytest.mark.parametrize("held", ["none", "own", "in place"])
def test_append_layouts(held, layout):
    _append_case(128, "bf16", [0, 5, 9], [20, 0, 7], 20, Hkv=3, seed=3, held=held, layout=layout)
    _append_case(64, "f32", [2], [9], 9, Hkv=1, seed=4, held=held, layout=layout)


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "bf16"), (128, "f32")])
def test_append_many_rows(d, dtype):
    # four pieces to a thread: tiles that end inside, sequences shorter than a tile
    _append_case(d, dtype, [0, 11], [5000, 130], 5000, Hkv=8, seed=5, held="own")


def test_append_64_sequences():
    _append_case(64, "bf16", [(7 * b) % 50 for b in range(64)], [1] * 64, 1, Hkv=8, seed=6)
    _append_case(128, "bf16", [(7 * b) % 50 for b in range(64)], [b % 3 for b in range(64)], 2, Hkv=1, seed=7)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_special_values(dtype):
    def edit(k, v):
        k[0, 0, 0, 3], k[0, 1, 1, 40], k[0, 2, 0, 127] = float("nan"), float("inf"), -float("inf")
        k[0, 3] = 0.0
        k[0, 4] = -0.0
        k[0, 5, 0, :32] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0] * 4)     # ties, scale 1
        k[0, 5, 0, 32:64] = -k[0, 5, 0, :32]
        v[0, 0] = torch.finfo(v.dtype).max
        v[0, 1] = -torch.finfo(v.dtype).max
        v[0, 2] = torch.finfo(v.dtype).tiny
        v[0, 3] = 1e-40 if v.dtype == torch.float32 else 1e-39                               # subnormal
        v[0, 4, 0, 0] = 6 * 2.0 ** -100
        v[0, 4, 0, 1:] = 2.0 ** -101                                                          # half of the least step: to even
        v[0, 5, :, 0] = 1e30                                                                  # beside it nothing is left
    _append_case(128, dtype, [4], [6], 6, seed=9, edit=edit, held="own")


def test_append_borders_of_a_scale():
    def edit(k, v):
        up = lambda x: float(np.nextafter(np.float32(x), np.float32(1e9)))   # noqa: E731
        for i, e in enumerate((-100, -101, -3, 0, 7, 120, 125)):
            k[0, i] = 2.0 ** e
            v[0, i] = 2.0 ** e
            k[0, i, 0, 5], v[0, i, 0, 5] = min(6 * 2.0 ** e, 3.4e38), min(up(6 * 2.0 ** e), 3.4e38)
    _append_case(64, "f32", [0], [7], 7, seed=10, edit=edit)


# --------------------------------------------------------------- attention ----

def _attend(q, kv_bytes, lens, dtype, scale=None, got=None, sharing=False):
    """Runs the call (or takes its results) and compares every sequence and head with the reference."""
    mad = _mad()
    k, v, ks, vs = kv_bytes
    B, T, Hq, d = q.shape
    Hkv, G = k.shape[1], Hq // k.shape[1]
    if got is None:
        dev = [t.cuda() for t in kv_bytes]
        got = mad.verify_attn_kv4(q.cuda(), mad.KV4(*dev, list(lens)), scale=scale)
    out, lse = (t.double().cpu().numpy() for t in got)
    for b in range(B):
        s = 0 if sharing else b
        for h in range(Hkv):
            kk, vv = kv4_ref.values(k[s, h].numpy(), ks[s, h].numpy()), kv4_ref.values(v[s, h].numpy(), vs[s, h].numpy())
            ref = kv4_ref.attend(q[b, :, h * G:(h + 1) * G].double().numpy(), kk, vv, lens[b], d ** -0.5 if scale is None else scale)
            tol, tol_lse = kv4_ref.tolerances(dtype, d, lens[b], *ref)
            o, l = out[b, :, h * G:(h + 1) * G], lse[b, :, h * G:(h + 1) * G]
            bad = ~(np.abs(o - ref[0]) <= tol)
            assert not bad.any(), f"sequence {b} head {h}: {int(bad.sum())} off, {np.nanmax(np.abs(o - ref[0])):.3g} at most, {(np.abs(o - ref[0]) / tol).max():.3g} of the bound"
            none = np.isneginf(ref[1])
            assert np.array_equal(np.isneginf(l), none) and np.all(o[none] == 0)
            assert np.all(np.abs(l[~none] - ref[1][~none]) <= tol_lse[~none]), f"sequence {b} head {h}: lse"
    return got


def _q(B, T, Hq, d, dtype, seed):
    return (0.7 * torch.randn((B, T, Hq, d), generator=torch.Generator().manual_seed(seed))).to(TYPES[dtype])


LENS = [[0, 1, 2, 5], [31, 32, 33, 64], [63, 65, 127, 128], [129, 255, 257, 300], [511, 513, 1000, 7]]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", LENS)
def test_attention_lengths(lens, d, dtype):
    cap = max(lens) + (1 if max(lens) % 2 == 0 else 2)   # an odd capacity: scales of 2-byte rows lie at any even address
    kv = _bytes(len(lens), 2, cap, d, seed=sum(lens))
    for T in (1, 5):
        _attend(_q(len(lens), T, 8, d, dtype, T), kv, lens, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,Hq,Hkv", [(1, 3, 3), (16, 2, 2), (17, 1, 1), (8, 16, 8), (3, 32, 2), (5, 8, 1), (6, 16, 2), (64, 1, 1), (4, 16, 1), (2, 48, 3)])
def test_attention_row_blocks(T, Hq, Hkv, d, dtype):
    lens = [T + 70, 40]
    _attend(_q(2, T, Hq, d, dtype, T), _bytes(2, Hkv, max(lens), d, seed=T), lens, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,Hkv,lens,T,G,d", [
    (1, 8, [9001], 5, 4, 64),          # many pieces of a unit, merged by a second launch
    (1, 1, [20011], 1, 1, 128),        # one row
    (2, 3, [4096, 777], 2, 8, 128),    # units whose pieces are merged in the launch
    (3, 8, [1500, 40, 2600], 6, 8, 128),   # 48 rows
    (64, 2, [17 * b % 600 for b in range(64)], 1, 4, 64)])
def test_attention_pieces(B, Hkv, lens, T, G, d, dtype):
    _attend(_q(B, T, Hkv * G, d, dtype, 3), _bytes(B, Hkv, max(lens) + 3, d, seed=len(lens)), lens, dtype)


@pytest.mark.parametrize("B,Hkv,T,G,d,dtype", [
    (33, 8, 1, 4, 64, "bf16"), (33, 8, 1, 4, 128, "bf16"), (40, 8, 4, 8, 128, "bf16"), (40, 8, 6, 8, 64, "bf16"),
    (33, 8, 8, 8, 128, "bf16"), (33, 8, 8, 8, 64, "bf16"), (33, 8, 8, 8, 128, "f32"),
    (64, 9, 2, 1, 64, "bf16"), (48, 11, 5, 2, 128, "bf16"), (64, 5, 1, 1, 64, "f32")])
def test_attention_more_units_than_cus(B, Hkv, T, G, d, dtype):
    # some sequences cut into pieces, the others whole; (64, 9) and (48, 11): more units than places, all whole
    lens = [b * 13 % 90 if b % 3 else 640 + 11 * b for b in range(B)]
    lens[5] = 4 * 640
    lens = [max(n, T) for n in lens]
    _attend(_q(B, T, Hkv * G, d, dtype, 3), _bytes(B, Hkv, max(lens) + 1, d, seed=1), lens, dtype)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_ignores_what_is_not_seen(d, dtype):
    """Bytes past the length (any scale, NaN too), and NaN rows that only later queries see."""
    T, lens = 4, [70, 33]
    kv = _bytes(2, 2, 96, d, seed=5)
    k, v, ks, vs = kv
    q = _q(2, T, 4, d, dtype, 1)
    want = _attend(q, kv, lens, dtype)
    for b, n in enumerate(lens):
        for t in (k, v, ks, vs):
            t[b, :, n:] = 255
    same = _attend(q, kv, lens, dtype)
    assert all(torch.equal(a, b) for a, b in zip(want, same))
    # row len - 2 (seen by queries T - 2 and T - 1 alone): one V group NaN; row len - 1: a K group NaN
    vs[0, 1, lens[0] - 2, 1] = 255
    ks[1, 0, lens[1] - 1, 0] = 255
    got = _mad().verify_attn_kv4(q.cuda(), _mad().KV4(*[t.cuda() for t in kv], lens))
    for x, y in zip(got, want):
        assert torch.equal(x[0, :T - 2], y[0, :T - 2]) and torch.equal(x[1, :T - 1], y[1, :T - 1])
        assert torch.equal(x[0, :, :2], y[0, :, :2]) and torch.equal(x[1, :, 2:], y[1, :, 2:])   # the other KV head
    o = got[0][0, T - 2:, 2:].float()
    assert torch.isnan(o[..., 32:64]).all() and torch.equal(o[..., :32], want[0][0, T - 2:, 2:, :32].float())
    assert torch.equal(got[1][0], want[1][0])                                    # a V value does not reach the lse
    assert torch.isnan(got[0][1, T - 1, :2]).all() and torch.isnan(got[1][1, T - 1, :2]).all()
    if d == 128:
        assert torch.equal(o[..., 64:], want[0][0, T - 2:, 2:, 64:].float())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_nan_where_every_row_sees_it(dtype):
    kv = _bytes(1, 1, 200, 64, seed=6)
    kv[3][0, 0, 10, 0] = 255
    got, _ = _mad().verify_attn_kv4(_q(1, 2, 4, 64, dtype, 1).cuda(), _mad().KV4(*[t.cuda() for t in kv], [200]))
    assert torch.isnan(got[..., :32]).all() and torch.isfinite(got[..., 32:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_scales_of_any_size(d, dtype):
    """V scales 2^90 apart from row to row and group to group, K rows of weight 0 with the largest V, scores far below 0."""
    k, v, ks, vs = _bytes(2, 2, 260, d, seed=7)
    g = torch.Generator().manual_seed(8)
    vs[0] = torch.randint(80, 170, vs[0].shape, generator=g, dtype=torch.uint8)
    ks[1, :, ::3], vs[1, :, ::3] = 130, 60          # some keys take the whole weight ...
    ks[1, :, 1::3], vs[1, :, 1::3] = 27, 200        # ... beside large weightless values
    _attend(_q(2, 3, 8, d, dtype, 9), (k, v, ks, vs), [260, 251], dtype)


def test_attention_equal_scores_and_growing_maxima():
    k, v, ks, vs = _bytes(1, 1, 600, 64, seed=10)
    k[:], ks[:] = 0x22, 127                          # every key the same: the mean of V
    _attend(_q(1, 1, 4, 64, "f32", 1), (k, v, ks, vs), [600], "f32")
    ks[0, 0] = (100 + torch.arange(600) // 16).to(torch.uint8)[:, None]   # scores that double every 16 keys
    q = torch.ones(1, 1, 4, 64) * 0.3
    _attend(q, (k, v, ks, vs), [600], "f32", scale=1e-3)


def test_attention_strided_and_shared_caches():
    mad = _mad()
    k, v, ks, vs = _bytes(3, 4, 90, 128, seed=11)
    q = _q(3, 2, 4, 128, "bf16", 1)
    pad = lambda t: torch.cat([t, torch.full_like(t[:, :, :6], 255)], 2).cuda()[1:, 1:3, :90]   # noqa: E731   heads 1, 2 of sequences 1, 2
    got = mad.verify_attn_kv4(q[1:, :, :4].cuda(), mad.KV4(pad(k), pad(v), pad(ks), pad(vs), [90, 50]))
    cut = [t[1:, 1:3].contiguous() for t in (k, v, ks, vs)]
    _attend(q[1:], cut, [90, 50], "bf16", got=got)
    one = [t[:1, :1].contiguous() for t in (k, v, ks, vs)]
    _attend(q, one, [90, 3, 64], "bf16", sharing=True)       # three queries of one sequence


def test_attention_beyond_32_bit_offsets():
    mad = _mad()
    cap, far = 64, (1 << 32) + (1 << 20)
    k, v, ks, vs = _bytes(2, 1, cap, 128, seed=12)
    big = [torch.empty(far + cap * 64, dtype=torch.uint8, device="cuda") for _ in range(2)]
    views = [t.as_strided((2, 1, cap, 64), (far, cap * 64, 64, 1)) for t in big]
    for t, x in zip(views, (k, v)):
        t.copy_(x.cuda())
    q = _q(2, 2, 4, 128, "bf16", 2)
    got = mad.verify_attn_kv4(q.cuda(), mad.KV4(*views, ks.cuda(), vs.cuda(), [64, 61]))
    _attend(q, (k, v, ks, vs), [64, 61], "bf16", got=got)
    new = _rows((2, 3, 1, 128), 13).to(torch.bfloat16)
    mad.kv4_append(new.cuda(), new.cuda(), mad.KV4(*views, ks.cuda(), vs.cuda(), [9, 61]))
    c, _ = kv4_ref.encode(new[1, :, 0].double().numpy())
    assert np.array_equal(views[0][1, 0, 61:64].cpu().numpy(), c) and np.array_equal(views[1][1, 0, 61:64].cpu().numpy(), c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_calls_repeat_bit_for_bit_on_streams_and_in_graphs(dtype):
    import bench
    mad = _mad()
    kv = [t.cuda() for t in _bytes(3, 8, 3100, 128, seed=14)]
    q = _q(3, 5, 32, 128, dtype, 3).cuda()
    new = _rows((3, 5, 8, 128), 15).to(TYPES[dtype]).cuda()
    c = mad.KV4(*kv, [3005, 77, 800])
    after = mad.KV4(*kv, [3010, 82, 805])
    out, lse, hk, hv = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda"), torch.empty_like(new), torch.empty_like(new)

    def step():
        mad.kv4_append(new, new, c, k_held=hk, v_held=hv)
        mad.verify_attn_kv4(q, after, out, lse)

    step()
    torch.cuda.synchronize()
    eager = [t.clone() for t in (out, lse, hk, hv)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        two = mad.verify_attn_kv4(q, after)
    step()
    torch.cuda.synchronize()
    assert torch.equal(two[0], eager[0]) and torch.equal(two[1], eager[1])
    graph = bench.graph_of(torch, step)
    for _ in range(3):
        for t in (out, lse, hk, hv):
            t.fill_(float("nan"))
        kv[0][0, :, 3005:] = 0
        torch.randn(1 << 20, device="cuda").sum().item()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, lse, hk, hv), eager))


def test_four_wave_calls_repeat_bit_for_bit_on_streams_and_in_graphs():
    import bench
    mad = _mad()
    B, T = 33, 6
    lens = [T + 97 * b % 700 for b in range(B)]
    lens[3] = 3000                                                                  # cut into pieces
    kv = mad.KV4(*[t.cuda() for t in _bytes(B, 8, 3001, 128, seed=16)], lens)
    q = [_q(B, T, 64, 128, "bf16", s).cuda() for s in (4, 5)]
    want = [mad.verify_attn_kv4(x, kv) for x in q]
    for x, w in zip(q, want):
        _attend(x.cpu(), [t.cpu() for t in (kv.k, kv.v, kv.k_scale, kv.v_scale)], lens, "bf16", got=w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    nbytes = mad.workspace_bytes(mad.MAD_OP_VERIFY_KV4, B, 64, 8, 128, T)
    ws = [torch.zeros(nbytes, dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):                                                              # two calls at once, a workspace each
        with torch.cuda.stream(side):
            a = mad.verify_attn_kv4(q[0], kv, ws=ws[0])
        b = mad.verify_attn_kv4(q[1], kv, ws=ws[1])
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((*a, *b), (*want[0], *want[1])))
    out, lse = torch.empty_like(q[0]), torch.empty(q[0].shape[:3], device="cuda")
    graphs = [bench.graph_of(torch, lambda x=x: mad.verify_attn_kv4(x, kv, out=out, lse=lse, ws=ws[0])) for x in q]   # one workspace
    for i in (0, 1, 1, 0):
        out.fill_(float("nan"))
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1])
