"""Sampling where a filter ends among entries of tiny weight: which of them stay, and the draw among them, are
decided by masses many binades below the row's largest weight.  The expected ends are counted, not summed: rows of
one high entry over a tail of one or two values, top_p half an entry's weight past a chosen one."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _mad():
    import paper_2608_30252_amd as mad
    return mad


def _sample(x, u, **kw):
    mad = _mad()
    p = torch.full(x.shape, float("nan"), device="cuda")
    tok, p = mad.sample(x.cuda(), u.cuda(), probs=p, **kw)
    torch.cuda.synchronize()
    return tok.cpu().numpy(), p.double().cpu().numpy()


def _kept(p, want, what):
    got = p > 0
    assert np.array_equal(got, want), f"{what}: {int(got.sum())} entries stay, expected {int(want.sum())}"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [700, 3000, 9001, 128256])
@pytest.mark.parametrize("gap", [22.0, 28.0])
def test_top_p_ends_in_a_flat_tail(gap, V, dtype):
    # The weights' and sums' roundings, 2^-45 relative at the outside, and top_p's own, 2^-53 of the whole, are below
    # 2^-45 V + 2^-53 e^28 < 2^-12 entries here; the end is half an entry away.
    spike, w = V // 3, math.exp(-gap)
    x = torch.zeros(1, 1, V)
    x[..., spike] = gap
    u = torch.full((1, 1), 0.5)
    for n in (0, 5, V // 7, V // 2, V - 3):
        top_p = (1 + (n + 0.5) * w) / (1 + (V - 1) * w)
        tok, p = _sample(x.to(TYPES[dtype]), u, top_p=top_p)
        tail = np.delete(np.arange(V), spike)
        want = np.zeros(V, bool)
        want[spike] = True
        want[tail[:n + 1]] = True
        _kept(p[0, 0], want, f"top_p {top_p!r}")
        assert tok[0, 0] == spike


@pytest.mark.parametrize("gap", [22.0, 28.0])
def test_top_p_behind_a_large_top_k_in_a_flat_tail(gap):
    V, k = 128256, 100000
    spike, w = V // 3, math.exp(-gap)
    x = torch.zeros(1, 1, V)
    x[..., spike] = gap
    tail = np.delete(np.arange(V), spike)
    for n in (5, 30000, k - 10):
        top_p = (1 + (n + 0.5) * w) / (1 + (k - 1) * w)
        tok, p = _sample(x, torch.full((1, 1), 0.5), top_k=k, top_p=top_p)
        want = np.zeros(V, bool)
        want[spike] = True
        want[tail[:n + 1]] = True
        _kept(p[0, 0], want, f"{n}")


@pytest.mark.parametrize("base", [0.0, 2.0 ** 20])
def test_top_p_ends_below_another_flat_part(base):
    # Two values in turn under the high entry; the end is in the lower one, so all of the upper one's mass lies above it.
    # At 2^20 no bins are counted and the row is decided by passes over it.
    V = 128256
    spike, w1, w2 = V // 3, math.exp(-23.5), math.exp(-24.0)
    at = np.arange(V)
    high = at % 2 == 0
    x = np.where(high, base + 0.5, base)
    x[spike] = base + 24.0
    high[spike] = False
    low = np.nonzero(~high & (at != spike))[0]
    for n in (0, 777, len(low) - 2):
        top_p = (1 + high.sum() * w1 + (n + 0.5) * w2) / (1 + high.sum() * w1 + len(low) * w2)
        tok, p = _sample(torch.from_numpy(x).float()[None, None], torch.full((1, 1), 0.5), top_p=top_p)
        want = high.copy()
        want[spike] = True
        want[low[:n + 1]] = True
        _kept(p[0, 0], want, f"{n}")


@pytest.mark.parametrize("kw,kept", [(dict(min_p=1e-14), 400), (dict(top_p=1 - 2e-12), 379)], ids=["min_p", "top_p"])
def test_the_draw_among_tiny_weights(kw, kept):
    # 400 entries of e^-30 lead the row (behind a masked chunk), the first 379 of them up to top_p: 2e-12 are 21.4.  The
    # uniform, (i + 1/2) of their weight, is rounded to fp32 by 2^-25 of itself: less than 400 2^-25 entries.
    V, n, w = 20000, 400, math.exp(-30.0)
    x = torch.full((1, 4, V), -float("inf"))
    x[..., 8200:8200 + n] = 0.0
    x[..., 17000] = 30.0
    z = 1 + kept * w
    want = [0, 7, 200, kept - 1]
    u = torch.tensor([[(i + 0.5) * w / z for i in want]])
    tok, p = _sample(x, u, **kw)
    stay = np.zeros(V, bool)
    stay[8200:8200 + kept] = stay[17000] = True
    for t in range(4):
        _kept(p[0, t], stay, f"{kw}")
    assert tok[0].tolist() == [8200 + i for i in want]
    assert np.all(np.abs(p[0, :, 8200:8200 + kept] / (w / z) - 1) <= 2.0 ** -23)
