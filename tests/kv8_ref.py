"""The 8-bit cache in plain float64 (CPU): what mad_kv8_append stores, what mad_verify_attn_kv8 computes, and how
far a kernel may be from the latter.

Values of e4m3 (sign, 4 exponent bits of bias 7, 3 mantissa bits; 0x7f and 0xff NaN) are written out here, and a
code is found by comparing against the midpoints of neighbouring values.
"""
import math

import numpy as np

CODES = np.array([np.nan if c == 127 else (c % 8) * 2.0 ** -9 if c < 8 else (1 + c % 8 / 8) * 2.0 ** (c // 8 - 7)
                  for c in range(128)])
MAX = 448.0


def decode(codes):
    """uint8 codes -> float64 values."""
    c = np.asarray(codes)
    return np.where(c >= 128, -1.0, 1.0) * CODES[c & 127]


def encode(x):
    """float64 values within 448 or NaN -> uint8 codes, to nearest, ties to the even code."""
    x = np.asarray(x, dtype=np.float64)
    mid = (CODES[:126] + CODES[1:127]) / 2               # between code c and c + 1
    a = np.abs(x)
    c = np.searchsorted(mid, a, side="left")             # a <= mid[c]: code c or, on the midpoint, the even one
    c = np.where((c < 126) & (a == mid[np.minimum(c, 125)]) & (c % 2 == 1), c + 1, c)
    c = np.where(np.isnan(x), 127, c)
    return (c | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def least_scale(m):
    """Least 2^k, k >= -100, with m <= 448 2^k."""
    k = -100
    if m > 0:
        k = max(k, math.frexp(m / MAX)[1] - 2)
        while m > MAX * 2.0 ** k:
            k += 1
    return 2.0 ** k


def append(codes, scale, new, length, n, block):
    """codes [Hkv, cap, d] uint8 and scale [Hkv, blocks] of one sequence and tensor, new [n_cap, Hkv, d]: changed in
    place, element types kept."""
    H = codes.shape[0]
    for h in range(H):
        for j in range(length // block, (length + n - 1) // block + 1 if n else 0):
            r0, r1 = max(j * block, length), min((j + 1) * block, length + n)
            x = np.asarray(new[r0 - length:r1 - length, h], dtype=np.float64)
            fine = np.isfinite(x)
            s = least_scale(np.abs(x[fine]).max() if fine.any() else 0.0)
            if r0 > j * block:
                old = float(scale[h, j])
                if old >= s:
                    s = old
                else:
                    v = decode(codes[h, j * block:r0]) * old
                    codes[h, j * block:r0] = encode(np.float32(v).astype(np.float64) / s)
            # the quotient as the fp32 division rounds it (exact for powers of two)
            with np.errstate(invalid="ignore"):
                q = (x.astype(np.float32) / np.float32(s)).astype(np.float64)
            codes[h, r0:r1] = encode(np.where(fine, q, np.nan))
            scale[h, j] = s


def values(codes, scale, block):
    """[..., rows, d] codes and [..., blocks] scales -> float64 values."""
    s = np.repeat(np.asarray(scale, dtype=np.float64), block, axis=-1)[..., :codes.shape[-2], None]
    return decode(codes) * s


def attend(q, K, V, length, scale):
    """q [T, Hq, d], K and V [Hkv, >= length, d] of one sequence -> out, lse, and for the tolerance per (t, head) the
    weighted mean of |v| [T, Hq, d], A = scale * max_j |q| . |k_j| and the number of keys."""
    T, Hq, d = q.shape
    G = Hq // K.shape[0]
    out, mean = np.zeros((T, Hq, d)), np.zeros((T, Hq, d))
    lse, A, n = np.full((T, Hq), -np.inf), np.zeros((T, Hq)), np.zeros((T, Hq))
    for t in range(T):
        m = length - T + t + 1
        if m <= 0:
            continue
        for h in range(Hq):
            k, v = K[h // G, :m], V[h // G, :m]
            s = scale * (k @ q[t, h])
            top = s.max()
            w = np.exp(s - top)
            z = w.sum()
            out[t, h], mean[t, h] = w @ v / z, w @ np.abs(v) / z
            lse[t, h] = top + np.log(z)
            A[t, h], n[t, h] = scale * (np.abs(k) @ np.abs(q[t, h])).max(), m
    return out, lse, mean, A, n


def out_tolerance(out, mean, A, n, d, vmax, bf16):
    """Per element.  The output's own rounding, half a step (2^-8 relative in bf16, 2^-24 in fp32); the
    probabilities' (fp16: 2^-11 of each, in two terms 2^-22); a score's error E = 2^-24 (2 sqrt(d) A + 8 A + 8),
    the rounding of a d-term fp32 sum with a factor 2 of margin, of its scaling and of the exponential's argument
    and result, which moves each weight by E and their sum too; fp32 sums over n keys, 2^-24 * 2 sqrt(n); and fp16's
    smallest step, 2^-25 of p' = 2^11 p (p the weight against a maximum that is no larger than the row's), on every key."""
    u = 2.0 ** -24
    E = u * (2 * math.sqrt(d) * A + 8 * A + 8)
    rel = (2.0 ** -11 if bf16 else 2.0 ** -22) + 2 * E + u * (4 + 2 * np.sqrt(n))
    return (2.0 ** -8 if bf16 else u) * np.abs(out) + rel[..., None] * mean + (n * 2.0 ** -36 * vmax)[..., None] + 1e-30


def check_out(got, out, tol, what=""):
    got = np.asarray(got, dtype=np.float64)
    assert got.shape == out.shape and np.all(np.isfinite(got)), f"{what}: shape or values not finite"
    err = np.abs(got - out)
    i = int(np.argmax(err - tol))
    assert np.all(err <= tol), f"{what}: off by {err.flat[i]:.3e}, {tol.flat[i]:.3e} allowed at |out| {abs(out.flat[i]):.3e}"
