"""The 8-bit cache on the GPU against plain float64 (kv8_ref.py): appends are exact, codes and scales; attention is
within kv8_ref.out_tolerance and parity.lse_tol, both derived there."""
import numpy as np
import pytest
import torch

import kv8_ref
from parity import lse_tol

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
F8 = torch.float8_e4m3fn


def _mad():
    import paper_2608_30252_amd as mad
    return mad


def _rows(shape, seed, spread=1.0):
    """N(0, 1) rows whose size varies by exp(spread N(0, 1))."""
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g) * torch.exp(spread * torch.randn(shape[:-1] + (1,), generator=g))


def _cache(B, Hkv, cap, d, block, seed, scales="pow2"):
    """A cache full of codes (never NaN) with scales in place: uint8 [B, Hkv, cap, d] and float32 on the CPU."""
    g = torch.Generator().manual_seed(seed)
    nb = -(-cap // block)
    k, v = (torch.randint(0, 127, (B, Hkv, cap, d), generator=g, dtype=torch.uint8) |
            (torch.randint(0, 2, (B, Hkv, cap, d), generator=g, dtype=torch.uint8) << 7) for _ in range(2))
    mk = lambda: (torch.exp2(torch.randint(-9, -4, (B, Hkv, nb), generator=g).float()) if scales == "pow2"   # noqa: E731
                  else torch.rand((B, Hkv, nb), generator=g) * 0.02 + 1e-4)
    return k, v, mk(), mk()


def _kv(mad, k, v, ks, vs, length, block):
    return mad.KV8(k.cuda().view(F8), v.cuda().view(F8), ks.cuda(), vs.cuda(), list(length), block)


# ------------------------------------------------------------------ append ----

def _append_case(d, block, dtype, lens, n, n_cap, Hkv=2, seed=0, scales="pow2", edit=None):
    mad = _mad()
    B = len(lens)
    cap = max(l + m for l, m in zip(lens, n)) + 3
    k, v, ks, vs = _cache(B, Hkv, cap, d, block, seed, scales)
    kn, vn = (_rows((B, n_cap, Hkv, d), seed + i).to(TYPES[dtype]) for i in (1, 2))
    if edit:
        edit(kn, vn)
    kv = _kv(mad, k, v, ks, vs, lens, block)
    mad.kv8_append(kn.cuda(), vn.cuda(), kv, None if n == [n_cap] * B else n)
    torch.cuda.synchronize()
    for name, codes, scale, new, got, got_s in (("k", k, ks, kn, kv.k, kv.k_scale), ("v", v, vs, vn, kv.v, kv.v_scale)):
        want, want_s = codes.numpy().copy(), scale.numpy().copy()
        for b in range(B):
            kv8_ref.append(want[b], want_s[b], new[b].double().numpy(), lens[b], n[b], block)
        assert np.array_equal(got_s.cpu().numpy(), want_s), f"{name}: scales"
        got = got.view(torch.uint8).cpu().numpy()
        nan = (want & 127) == 127
        assert np.array_equal((got & 127) == 127, nan), f"{name}: NaN codes"
        assert np.array_equal(got[~nan], want[~nan]), f"{name}: {int((got[~nan] != want[~nan]).sum())} codes differ"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("d", [64, 128])
def test_append_lengths(d, block, dtype):
    # starts at, inside, one before and one past a block's border; ends inside a later block; none at all
    lens = [0, 1, block - 1, block, 2 * block + 5, 7, 3]
    n = [1, block - 1, 2, 1, 3 * block + 1, 0, 2 * block]
    _append_case(d, block, dtype, lens, n, 3 * block + 1, seed=block + d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_every_row(dtype):
    _append_case(128, 32, dtype, [0, 31, 40], [70, 70, 70], 70, Hkv=3, seed=5)


def test_append_64_sequences_and_one_token():
    _append_case(64, 16, "bf16", [(7 * b) % 50 for b in range(64)], [1] * 64, 1, Hkv=8, seed=6)
    _append_case(64, 16, "bf16", [(7 * b) % 50 for b in range(64)], [b % 3 for b in range(64)], 2, Hkv=1, seed=7)


@pytest.mark.parametrize("scales", ["pow2", "any"])
def test_append_beside_small_and_large_rows(scales):
    # earlier rows far larger than the new ones (the scale stays), and far smaller (they are written again)
    for size in (1e-6, 1.0, 1e3, 1e30):
        _append_case(64, 32, "f32", [5, 20, 31], [9, 4, 40], 40, seed=8, scales=scales,
                     edit=lambda k, v: (k.mul_(size), v.mul_(size)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_what_is_not_finite(dtype):
    def edit(k, v):
        k[0, 0, 0, 3], k[0, 1, 1, 0], k[1, 2, 0, 5] = float("nan"), float("inf"), -float("inf")
        v[0] = float("nan")            # a block with nothing finite
        v[1, :, 0] = 0.0               # and one of zeros
        k[1, 3] = -0.0
        v[1, 3, 1] = 1e-40             # below the least scale
    _append_case(64, 16, dtype, [0, 13], [6, 6], 6, seed=9, edit=edit)


def test_append_values_on_the_border_of_a_scale():
    # 448 2^k fits scale 2^k, the next number up does not
    def edit(k, v):
        k[...] = 1.0
        k[0, 0, 0, 0], k[0, 0, 1, 0] = 448 * 2.0 ** -4, float(np.nextafter(np.float32(448 * 2.0 ** -4), np.float32(1e9)))
        v[...] = 3e38
        v[0, 0, 1] = 2.0 ** -130
    _append_case(64, 16, "f32", [0], [1], 1, seed=10, edit=edit)


def test_append_into_strided_buffers():
    # heads of a larger buffer, rows before and after the view; scales as a slice of a larger table
    mad = _mad()
    B, Hkv, cap, d, block = 2, 2, 50, 64, 16
    big = torch.full((B, Hkv, 3, cap + 14, d), 0x55, dtype=torch.uint8, device="cuda")
    tab = torch.full((B, Hkv, 3, 9), 2.0 ** -20, device="cuda")
    k, v = big[:, :, 0, 7:7 + cap], big[:, :, 2, 7:7 + cap]
    kv = mad.KV8(k.view(F8), v.view(F8), tab[:, :, 0, 1:5], tab[:, :, 2, 1:5], [17, 30], block)
    kn, vn = (_rows((B, 20, Hkv, d), s).bfloat16() for s in (1, 2))
    want = {n: (t.cpu().numpy().copy(), s.cpu().numpy().copy()) for n, t, s in (("k", k, kv.k_scale), ("v", v, kv.v_scale))}
    mad.kv8_append(kn.cuda(), vn.cuda(), kv, [20, 11])
    torch.cuda.synchronize()
    for n, t, s, new in (("k", k, kv.k_scale, kn), ("v", v, kv.v_scale, vn)):
        for b in range(B):
            kv8_ref.append(want[n][0][b], want[n][1][b], new[b].double().numpy(), kv.length[b], [20, 11][b], block)
        assert np.array_equal(t.cpu().numpy(), want[n][0]) and np.array_equal(s.cpu().numpy(), want[n][1])
    assert bool((big[:, :, 1] == 0x55).all() and (big[:, :, :, :7] == 0x55).all() and (big[:, :, :, 7 + cap:] == 0x55).all())
    assert bool((tab[:, :, 1] == 2.0 ** -20).all() and (tab[:, :, :, 0] == 2.0 ** -20).all() and (tab[:, :, :, 5:] == 2.0 ** -20).all())


def test_rollback_and_append_again():
    # a rejected block's rows are written over; the scale they raised stays
    mad = _mad()
    B, Hkv, cap, d, block = 1, 2, 64, 128, 32
    k, v, ks, vs = _cache(B, Hkv, cap, d, block, 3)
    kv = _kv(mad, k, v, ks, vs, [37], block)
    big, small = _rows((B, 5, Hkv, d), 4) * 100, _rows((B, 2, Hkv, d), 5)
    mad.kv8_append(big.cuda(), big.cuda(), kv)
    mad.kv8_append(small.cuda(), small.cuda(), kv)       # the length was not raised: the same rows again
    torch.cuda.synchronize()
    for codes, scale, got, got_s in ((k, ks, kv.k, kv.k_scale), (v, vs, kv.v, kv.v_scale)):
        c, s = codes[0].numpy().copy(), scale[0].numpy().copy()
        kv8_ref.append(c, s, big[0].double().numpy(), 37, 5, block)
        raised = s.copy()
        kv8_ref.append(c, s, small[0].double().numpy(), 37, 2, block)
        assert np.array_equal(raised, s)
        assert np.array_equal(got[0].view(torch.uint8).cpu().numpy(), c) and np.array_equal(got_s[0].cpu().numpy(), s)


# --------------------------------------------------------------- attention ----

def _attend_case(B, T, Hq, Hkv, d, block, dtype, lens, seed=0, scales="pow2", qsize=1.0, edit=None, kv=None, scale=None):
    mad = _mad()
    cap = max(max(lens), 1) + 2
    k, v, ks, vs = _cache(B, Hkv, cap, d, block, seed, scales)
    q = (qsize * _rows((B, T, Hq, d), seed + 1, 0.2)).to(TYPES[dtype])
    if edit:
        edit(q, k, v, ks, vs)
    out, lse = mad.verify_attn_kv8(q.cuda(), _kv(mad, k, v, ks, vs, lens, block), scale=scale)
    torch.cuda.synchronize()
    _compare(q, k, v, ks, vs, lens, block, out, lse, dtype == "bf16", scale)


def _compare(q, k, v, ks, vs, lens, block, out, lse, bf16, scale=None):
    d = q.shape[3]
    scale = d ** -0.5 if scale is None else scale
    for b, n in enumerate(lens):
        K = kv8_ref.values(k[b].numpy(), ks[b].numpy(), block)
        V = kv8_ref.values(v[b].numpy(), vs[b].numpy(), block)
        o, l, mean, A, m = kv8_ref.attend(q[b].double().numpy(), K, V, n, scale)
        vmax = np.abs(V[:, :max(n, 1)]).max()
        kv8_ref.check_out(out[b].double().cpu().numpy(), o, kv8_ref.out_tolerance(o, mean, A, m, d, vmax, bf16), f"b {b}, {n} keys")
        got = lse[b].double().cpu().numpy()
        assert np.array_equal(np.isneginf(got), np.isneginf(l))
        fin = np.isfinite(l)
        assert np.all(np.abs(got[fin] - l[fin]) <= lse_tol(A, l, d)[fin]), f"b {b}: lse off by {np.abs(got[fin] - l[fin]).max()}"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d,T", [(8, 8, 64, 1), (8, 2, 128, 1), (32, 8, 64, 5), (16, 2, 128, 4), (16, 1, 64, 3),
                                        (16, 1, 128, 4), (12, 3, 128, 6), (16, 16, 64, 2)])
def test_attention_shapes(Hq, Hkv, d, T, dtype):
    _attend_case(2, T, Hq, Hkv, d, 16, dtype, [517, 130], seed=Hq + T)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_lengths(d, dtype):
    # nothing, less than T rows, around a block, a 32-key step and a slab (128 or 256 keys), several slabs
    lens = [0, 1, 2, 3, 15, 16, 17, 31, 32, 33, 127, 128, 129, 255, 256, 257, 511, 513, 700, 1025]
    _attend_case(len(lens), 3, 8, 2, d, 32, dtype, lens, seed=d)


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_blocks_and_any_scales(d, block):
    _attend_case(2, 5, 8, 2, d, block, "bf16", [700, 333], seed=block, scales="any")
    _attend_case(2, 2, 8, 2, d, block, "f32", [700, 333], seed=block + 1, scales="any")


def test_attention_scales_that_differ_by_far():
    # V scales over 60 binades, growing and falling along the keys; K scales of 0
    def edit(q, k, v, ks, vs):
        nb = vs.shape[2]
        vs[0] = torch.exp2(torch.linspace(-50, 10, nb).round())
        vs[1] = torch.exp2(torch.linspace(10, -50, nb).round())
        ks[:, :, ::3] = 0.0
        vs[:, :, 1::5] = 0.0
    for dtype in ("bf16", "f32"):
        _attend_case(2, 3, 8, 2, 128, 32, dtype, [900, 870], seed=11, edit=edit)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_peaky(dtype):
    # queries along one key's row: nearly all of the weight on it
    def edit(q, k, v, ks, vs):
        ks.fill_(2.0 ** -8)
        K = kv8_ref.values(k.numpy(), ks.numpy(), 16)
        for b in range(2):
            for h in range(8):
                q[b, :, h] = torch.from_numpy(K[b, h // 4, 100 * b + 7 * h]).to(q.dtype) * 40
    _attend_case(2, 2, 8, 2, 64, 16, dtype, [400, 390], seed=12, edit=edit)


def test_attention_many_pieces_and_ragged():
    # runs over unit borders, pieces merged in the launch and by the second launch
    rng = np.random.RandomState(3)
    _attend_case(9, 2, 8, 4, 128, 64, "bf16", [int(x) for x in rng.randint(1, 3000, 9)], seed=13)
    _attend_case(3, 4, 16, 2, 64, 64, "bf16", [6000, 10, 2500], seed=14)
    _attend_case(1, 5, 8, 1, 128, 64, "f32", [9000], seed=15)
    _attend_case(1, 8, 8, 1, 128, 64, "bf16", [9000], seed=16)


def test_attention_more_units_than_workgroups():
    _attend_case(64, 1, 8, 8, 64, 16, "bf16", [(5 * b) % 300 for b in range(64)], seed=17)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_hidden_and_unused_rows_hold_anything(dtype):
    # NaN codes: K and V rows from len on, and the last new token's, which only the last query sees
    mad = _mad()
    B, T, Hq, Hkv, d, block, n = 1, 3, 8, 2, 128, 32, 300
    k, v, ks, vs = _cache(B, Hkv, 340, d, block, 18)
    q = _rows((B, T, Hq, d), 19, 0.2).to(TYPES[dtype])
    clean = mad.verify_attn_kv8(q.cuda(), _kv(mad, k, v, ks, vs, [n], block))
    k[:, :, n:], v[:, :, n:] = 127, 255
    ks[:, :, -(-n // block):], vs[:, :, -(-n // block):] = float("nan"), float("inf")
    got = mad.verify_attn_kv8(q.cuda(), _kv(mad, k, v, ks, vs, [n], block))
    torch.cuda.synchronize()
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])
    for row in ("k", "v"):
        k2, v2 = k.clone(), v.clone()
        (k2 if row == "k" else v2)[:, 0, n - 1, 5] = 127
        out, lse = mad.verify_attn_kv8(q.cuda(), _kv(mad, k2, v2, ks, vs, [n], block))
        torch.cuda.synchronize()
        out, lse, o0, l0 = out.float(), lse, clean[0].float(), clean[1]
        # the other KV head (query heads 4 ..) and the first T - 1 queries: untouched, but for roundings (one
        # accumulation less, the taken-out code being 0)
        assert torch.equal(out[:, :, 4:], o0[:, :, 4:]) and torch.equal(lse[:, :, 4:], l0[:, :, 4:])
        assert torch.equal(out[:, :2, :4], o0[:, :2, :4]) and torch.equal(lse[:, :2, :4], l0[:, :2, :4])
        if row == "k":
            assert bool(torch.isnan(out[:, 2, :4]).all() and torch.isnan(lse[:, 2, :4]).all())
        else:
            bad = torch.isnan(out[:, 2, :4])
            assert bool(bad[..., 5].all()) and int(bad.sum()) == 4 and torch.equal(lse[:, 2, :4], l0[:, 2, :4])


def test_attention_sees_nan():
    # a visible NaN in a slab that every query sees whole, and in one of many pieces
    mad = _mad()
    for n, at in ((600, 10), (9000, 5000)):
        k, v, ks, vs = _cache(1, 1, n, 64, 16, 20)
        k[0, 0, at, 0] = 255
        out, lse = mad.verify_attn_kv8(_rows((1, 2, 4, 64), 21).bfloat16().cuda(), _kv(mad, k, v, ks, vs, [n], 16))
        torch.cuda.synchronize()
        assert bool(torch.isnan(out).all() and torch.isnan(lse).all())


def test_attention_views_of_larger_buffers_and_shared_sequences():
    mad = _mad()
    Hkv, cap, d, block = 2, 260, 64, 32
    k, v, ks, vs = _cache(1, Hkv, cap, d, block, 22)
    q = _rows((3, 2, 8, d), 23).bfloat16()
    lens = [260, 100, 17]
    # batch dimension 1: every row reads sequence 0
    out, lse = mad.verify_attn_kv8(q.cuda(), _kv(mad, k, v, ks, vs, lens, block))
    # the same as slices of larger buffers
    big = torch.full((2, 1, Hkv, cap + 32, d), 0x77, dtype=torch.uint8, device="cuda")
    big[0, :, :, 16:16 + cap], big[1, :, :, 16:16 + cap] = k.cuda(), v.cuda()
    tab = torch.full((2, 1, Hkv, 20), float("nan"), device="cuda")
    tab[0, :, :, 3:12], tab[1, :, :, 3:12] = ks.cuda(), vs.cuda()
    kv = mad.KV8(big[0, :, :, 16:16 + cap].view(F8), big[1, :, :, 16:16 + cap].view(F8), tab[0, :, :, 3:12], tab[1, :, :, 3:12], lens, block)
    out2, lse2 = mad.verify_attn_kv8(q.cuda(), kv)
    torch.cuda.synchronize()
    assert torch.equal(out, out2) and torch.equal(lse, lse2)
    three = lambda t: t.expand(3, -1, -1, *[-1] * (t.dim() - 3))   # noqa: E731
    _compare(q, three(k), three(v), three(ks), three(vs), lens, block, out, lse, True)


def test_attention_agrees_with_the_bf16_cache():
    # codes times a power of two are exact in bf16: the bf16 verify attention over the values is the same function
    mad = _mad()
    B, T, Hq, Hkv, d, block, lens = 2, 4, 16, 4, 128, 64, [1500, 2100]
    k, v, ks, vs = _cache(B, Hkv, 2104, d, block, 24)
    q = _rows((B, T, Hq, d), 25).bfloat16()
    out, lse = mad.verify_attn_kv8(q.cuda(), _kv(mad, k, v, ks, vs, lens, block))
    val = lambda c, s: torch.from_numpy(kv8_ref.values(c.numpy(), s.numpy(), block)).bfloat16().cuda()   # noqa: E731
    out2, lse2 = mad.verify_attn(q.cuda(), mad.KV(val(k, ks), val(v, vs), lens))
    torch.cuda.synchronize()
    _compare(q, k, v, ks, vs, lens, block, out, lse, True)
    # the bf16 kernel rounds probabilities to bf16 (2^-8 of the weighted mean of |v| < 4) and both outputs to bf16
    assert float((out.float() - out2.float()).abs().max()) <= 2.0 ** -8 * 4 + 2.0 ** -7 * float(out.float().abs().max())
    assert float((lse - lse2).abs().max()) <= 1e-3


def test_rows_past_two_gigabytes():
    # one head of 17.2 million rows of 128 bytes: offsets past 2^31 in the append, the keys and the scales
    mad = _mad()
    d, block, n = 128, 128, (1 << 31) // 128 + 400_000
    kv = mad.KV8.empty(1, 1, n + 4, d, block)
    kv.k_scale.fill_(1.0), kv.v_scale.fill_(0.5)
    new = torch.zeros(1, 3, 1, d)
    new[0, :, 0, :] = torch.tensor([[7.0], [14.0], [28.0]])
    kv.length = [n]
    mad.kv8_append(torch.zeros_like(new).cuda(), new.cuda(), kv)
    kv.length = [n + 3]
    torch.cuda.synchronize()
    s = kv.v_scale[0, 0, n // block:].cpu()
    assert float(s[0]) == (0.5 if n % block else 2.0 ** -4)
    got = kv.v[0, 0, n:n + 3].float().cpu() * float(s[0])
    assert torch.equal(got, new[0, :, 0])
    # all keys are zero: every row has the same weight, and only the last three values count
    out, lse = mad.verify_attn_kv8(torch.ones(1, 2, 1, d, device="cuda"), kv)
    torch.cuda.synchronize()
    want = torch.tensor([21.0 / (n + 2), 49.0 / (n + 3)])
    # sums of n equal terms in fp32 (within a 32-key step's lane n / 8192 of them one by one): 1e-3 relative is far above
    assert float((out[0, :, 0, :].cpu() / want[:, None] - 1).abs().max()) <= 1e-3
    assert float((lse[0, :, 0].cpu() - torch.log(torch.tensor([n + 2.0, n + 3.0]))).abs().max()) <= 1e-3


# ------------------------------------------------- streams, graphs, workspaces ----

def test_graph_replays_of_append_and_attention():
    # captured once, replayed with other inputs in the same buffers between eager work; two graphs, a workspace each
    mad = _mad()
    B, T, Hq, Hkv, d, block, lens = 4, 3, 16, 4, 128, 32, [300, 65, 1000, 33]
    k, v, ks, vs = _cache(B, Hkv, 1040, d, block, 26)
    cache = [_kv(mad, k, v, ks, vs, lens, block) for _ in range(2)]
    kn, vn = torch.empty(B, T, Hkv, d, device="cuda"), torch.empty(B, T, Hkv, d, device="cuda")
    q = torch.empty(B, T, Hq, d, device="cuda", dtype=torch.bfloat16)
    nbytes = mad.workspace_bytes(mad.MAD_OP_VERIFY, B, Hq, Hkv, d, T)
    res = [(torch.empty_like(q), torch.empty(B, T, Hq, device="cuda")) for _ in range(2)]
    grown = [l + T for l in lens]

    def step(i, ws):
        kv = cache[i]
        mad.kv8_append(kn, vn, mad.KV8(kv.k, kv.v, kv.k_scale, kv.v_scale, lens, block))
        mad.verify_attn_kv8(q, mad.KV8(kv.k, kv.v, kv.k_scale, kv.v_scale, grown, block), *res[i], ws=ws)

    graphs = []
    for i in range(2):
        ws = torch.zeros(nbytes, dtype=torch.uint8, device="cuda")
        kn.normal_(), vn.normal_(), q.normal_()
        step(i, ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(i, ws)
        graphs.append((g, ws))
    for r in range(4):
        for i in range(2):
            for t, src in ((cache[i].k.view(torch.uint8), k), (cache[i].v.view(torch.uint8), v), (cache[i].k_scale, ks), (cache[i].v_scale, vs)):
                t.copy_(src)
        g = torch.Generator(device="cuda").manual_seed(r)
        for t in (kn, vn, q):
            t.normal_(generator=g)
        graphs[0][0].replay()
        graphs[1][0].replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in res[0]]
        assert torch.equal(got[0], res[1][0]) and torch.equal(got[1], res[1][1])
        assert torch.equal(cache[0].k.view(torch.uint8), cache[1].k.view(torch.uint8)) and torch.equal(cache[0].k_scale, cache[1].k_scale)
        for t, src in ((cache[0].k.view(torch.uint8), k), (cache[0].v.view(torch.uint8), v), (cache[0].k_scale, ks), (cache[0].v_scale, vs)):
            t.copy_(src)
        step(0, None)   # eagerly, on the default workspace
        torch.cuda.synchronize()
        assert torch.equal(got[0], res[0][0]) and torch.equal(got[1], res[0][1]), f"replay {r}"


def test_side_stream_and_both_marshalling_paths(monkeypatch):
    mad = _mad()
    B, T, Hq, Hkv, d, block, lens = 2, 5, 32, 8, 64, 16, [3000, 700]
    k, v, ks, vs = _cache(B, Hkv, 3010, d, block, 27)
    kv = _kv(mad, k, v, ks, vs, lens, block)
    q = _rows((B, T, Hq, d), 28).bfloat16().cuda()
    kn = _rows((B, T, Hkv, d), 29).cuda()
    out, lse = mad.verify_attn_kv8(q, kv)
    mad.kv8_append(kn, kn, kv, [5, 3])
    torch.cuda.synchronize()
    after = [t.clone() for t in (kv.k.view(torch.uint8), kv.v_scale)]
    side = torch.cuda.Stream()
    for path in ("native", "ctypes"):
        if path == "ctypes":
            monkeypatch.setattr(mad, "_FAST", mad._CtypesOnly())
        kv2 = _kv(mad, k, v, ks, vs, lens, block)
        o2, l2 = torch.zeros_like(out), torch.zeros_like(lse)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            mad.verify_attn_kv8(q, kv2)                 # (the stream's workspace)
            mad.verify_attn_kv8(q, kv2, o2, l2)
            mad.kv8_append(kn, kn, kv2, [5, 3])
        side.synchronize()
        assert torch.equal(out, o2) and torch.equal(lse, l2), path
        assert torch.equal(after[0], kv2.k.view(torch.uint8)) and torch.equal(after[1], kv2.v_scale), path


def test_ordinary_calls_take_the_native_path():
    mad = _mad()
    fast = mad._fast()
    k, v, ks, vs = _cache(2, 2, 64, 64, 16, 30)
    kv = _kv(mad, k, v, ks, vs, [30, 20], 16)
    q = torch.zeros(2, 2, 4, 64, device="cuda")
    mad.verify_attn_kv8(q, kv)
    assert fast.verify8(q, kv, torch.empty_like(q), torch.empty(2, 2, 4, device="cuda"), None, None) == mad.MAD_OK
    assert fast.kv8_append(q[:, :, :2].contiguous(), q[:, :, :2].contiguous(), kv, [1, 2]) == mad.MAD_OK
    assert fast.kv8_append(q[:, :, :2].contiguous(), q[:, :, :2].contiguous(), kv, np.array([1, 2])) is None
    torch.cuda.synchronize()
