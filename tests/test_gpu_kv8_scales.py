"""The 8-bit verify attention where V scales differ by far between blocks: what a row adds up counts against what it
sees and weighs, not against the largest scale around."""
import math

import numpy as np
import pytest
import torch

import kv8_ref
from test_gpu_kv8 import TYPES, _cache, _kv, _mad, _rows

pytestmark = pytest.mark.gpu


def _check(q, k, v, ks, vs, lens, block, out, bf16):
    """Every element, within: the output's own rounding; the probabilities' (fp16: 2^-11 of each, in two terms 2^-22) and
    fp32's (kv8_ref.out_tolerance) of the weighted mean of |v|; and fp16's least step: p v_scale, a row's largest of which
    is brought to 2^10 at least, is off by 2^-25 at most, i.e. by 2^-35 of that largest, times a code of 448, for every key."""
    d = q.shape[3]
    G = q.shape[2] // k.shape[1]
    for b, n in enumerate(lens):
        K = kv8_ref.values(k[b].numpy(), ks[b].numpy(), block)
        V = kv8_ref.values(v[b].numpy(), vs[b].numpy(), block)
        S = np.repeat(vs[b].double().numpy(), block, axis=-1)
        Q = q[b].double().numpy()
        o, l, mean, A, m = kv8_ref.attend(Q, K, V, n, d ** -0.5)
        tol = kv8_ref.out_tolerance(o, mean, A, m, d, 0.0, bf16)
        T = q.shape[1]
        for t in range(T):
            for h in range(q.shape[2]):
                see = n - T + t + 1
                p = np.exp(d ** -0.5 * (K[h // G, :see] @ Q[t, h]) - l[t, h])
                tol[t, h] += see * 2.0 ** -35 * 448 * (p * S[h // G, :see]).max()
        kv8_ref.check_out(out[b].double().cpu().numpy(), o, tol, f"b {b}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,T,Hq", [(64, 2, 8), (128, 6, 64), (128, 8, 64)])
def test_a_hidden_block_of_large_values(d, T, Hq, dtype):
    # the newest row alone in its block, 2^40 times the others': the queries before the last do not see it
    mad = _mad()
    Hkv, block, n = (2, 16, 17 + 16 * 4) if Hq == 8 else (8, 16, 17 + 16 * 4)
    k, v, ks, vs = _cache(1, Hkv, n, d, block, 5)
    q = _rows((1, T, Hq, d), 6, 0.2).to(TYPES[dtype])
    base, _ = mad.verify_attn_kv8(q.cuda(), _kv(mad, k, v, ks, vs, [n], block))
    for up in (20, 40, 100):
        vs2 = vs.clone()
        vs2[:, :, (n - 1) // block] *= 2.0 ** up
        out, _ = mad.verify_attn_kv8(q.cuda(), _kv(mad, k, v, ks, vs2, [n], block))
        torch.cuda.synchronize()
        assert torch.equal(out[:, :T - 1], base[:, :T - 1]), f"2^{up}"
        _check(q, k, v, ks, vs2, [n], block, out, dtype == "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,T,Hq", [(64, 2, 8), (128, 5, 64), (128, 8, 64)])
@pytest.mark.parametrize("n", [300, 5000])
def test_large_values_of_no_weight(n, d, T, Hq, dtype):
    # a block whose values are 2^30 (2^60) times the others' but whose keys weigh e^-40 (e^-80): what it adds is little,
    # and the rest is as exact as without it; and blocks in between
    mad = _mad()
    Hkv, block = Hq // 8 if Hq == 64 else 2, 16     # (two blocks and more to what a wave reads at a time)
    k, v, ks, vs = _cache(2, Hkv, n, d, block, 7)
    q = torch.zeros(2, T, Hq, d, dtype=TYPES[dtype])
    q[..., 0] = math.sqrt(d)                       # a key's score is its feature 0
    ks.fill_(1.0)
    kk = torch.zeros(k.shape)
    kk[..., 0] = torch.rand(k.shape[:3], generator=torch.Generator().manual_seed(8))
    nb = vs.shape[2]
    for j, (drop, up) in enumerate(((40.0, 30), (80.0, 60), (20.0, 28), (8.0, 11))):
        at = (j * nb) // 4 if n > 400 else 4 * j
        kk[:, :, at * block:(at + 1) * block, 0] -= drop
        vs[:, :, at] *= 2.0 ** up
    k = kk.to(torch.float8_e4m3fn).view(torch.uint8)
    lens = [n, n - 37]
    out, lse = mad.verify_attn_kv8(q.cuda(), _kv(mad, k, v, ks, vs, lens, block))
    torch.cuda.synchronize()
    _check(q, k, v, ks, vs, lens, block, out, dtype == "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales_from_the_least_to_the_largest(dtype):
    # V scales over all of fp32's normal numbers, growing and falling along the keys, zeros among them: a row of equal weights
    # is the mean of what it sees, to which the largest block alone contributes
    mad = _mad()
    d, Hkv, block, n, T, Hq = 128, 2, 16, 1600, 3, 8
    k, v, ks, vs = _cache(2, Hkv, n, d, block, 9)
    nb = vs.shape[2]
    e = torch.linspace(-126, 110, nb).round()
    vs[0], vs[1] = torch.exp2(e), torch.exp2(e.flip(0))
    vs[:, :, 1::7] = 0.0
    q = (0.05 * _rows((2, T, Hq, d), 10)).to(TYPES[dtype])
    ks.fill_(2.0 ** -6)
    lens = [n, n - 5]
    out, lse = mad.verify_attn_kv8(q.cuda(), _kv(mad, k, v, ks, vs, lens, block))
    torch.cuda.synchronize()
    _check(q, k, v, ks, vs, lens, block, out, dtype == "bf16")
