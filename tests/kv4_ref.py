"""The 4-bit cache in plain numpy float64, written from its definition: codes 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign in
bit 3, two to a byte (the even feature's low), a scale byte s = 2^(s - 127) for each row and 32 features, 255 NaN."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
GROUP = 32


FITS = 6.0 * 2.0 ** np.arange(-100, 126)   # the largest value of each scale


def least_scale(m):
    """The least k, -100 <= k <= 125, with m <= 6 * 2^k (125 for anything larger)."""
    return np.minimum(np.searchsorted(FITS, m, side="left"), 225) - 100


def encode(x):
    """x [..., 32 g] float64 -> (codes uint8 [..., 16 g], scale bytes uint8 [..., g])."""
    x = np.asarray(x, np.float64)
    g = x.reshape(x.shape[:-1] + (x.shape[-1] // GROUP, GROUP))
    fine = np.isfinite(g).all(-1)
    k = least_scale(np.where(fine, np.where(np.isfinite(g), np.abs(g), 0).max(-1), 0.0))
    a = np.where(fine[..., None], np.minimum(np.abs(np.where(np.isfinite(g), g, 0)) / 2.0 ** k[..., None], 6.0), 0.0)
    lo = np.searchsorted(LEVELS, a, side="right") - 1                  # the last level not above
    hi = np.minimum(lo + 1, 7)
    below, above = a - LEVELS[lo], LEVELS[hi] - a
    code = np.where((above < below) | ((above == below) & (hi % 2 == 0)), hi, lo)
    code = np.where(fine[..., None], code + 8 * np.signbit(g), 0).astype(np.uint8)
    pairs = code.reshape(x.shape[:-1] + (x.shape[-1] // 2, 2))
    return pairs[..., 0] | (pairs[..., 1] << 4), np.where(fine, k + 127, 255).astype(np.uint8)


def values(codes, scale):
    """The float64 values of codes [..., d/2] and scale bytes [..., d/32]."""
    c = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (codes.shape[-1] // 16, GROUP))
    s = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    x = np.where(c & 8, -1.0, 1.0) * LEVELS[c & 7] * s[..., None]
    return x.reshape(codes.shape[:-1] + (2 * codes.shape[-1],))


def attend(q, k, v, n, scale):
    """q [T, G, d], k and v [cap, d]; query t sees rows 0 .. n - T + t.  Returns out [T, G, d], lse [T, G], the sums of
    weight times |value| [T, G, d], and the largest score bound sum |q k| scale [T, G]."""
    T, G, d = q.shape
    out, lse = np.zeros((T, G, d)), np.full((T, G), -np.inf)
    mass, big = np.zeros((T, G, d)), np.zeros((T, G))
    for t in range(T):
        m = n - T + t + 1
        if m <= 0:
            continue
        s = (q[t] @ k[:m].T) * scale                                   # [G, m]
        top = s.max(1, keepdims=True)
        p = np.exp(s - top)
        z = p.sum(1, keepdims=True)
        p /= z
        out[t], mass[t] = p @ v[:m], p @ np.abs(v[:m])
        lse[t] = (top + np.log(z))[:, 0]
        big[t] = ((np.abs(q[t]) @ np.abs(k[:m]).T) * scale).max(1)
    return out, lse, mass, big


def tolerances(dtype, d, n, out, lse, mass, big):
    """Bounds for out and lse.  With e = 2^-24: a score's products are exact or (fp32: three bf16 terms each way) lose e, and
    are summed in at most d + 3 roundings of what the sum of |q k| bounds, then one product and one difference in log2
    units: ds = (d + 6) e big; a probability is off by ds + 4 e (the power, its argument), in sums of n / 32 matrix steps'
    results and 64 joins by another (n / 32 + 64) e.  The numerator carries that twice (values, then weights of the sum
    below) and bf16 rounds each probability by 2^-8, the output by 2^-8; fp32's three bf16 terms lose e, the output e."""
    e = 2.0 ** -24
    ds = (d + 6) * e * big
    chain = (n / 32 + 64) * e
    p = 2 * (ds + 4 * e + chain)[..., None] + (2.0 ** -8 if dtype == "bf16" else 2 * e)
    tol_out = p * mass + (2.0 ** -8 if dtype == "bf16" else e) * np.abs(out) + 1e-37
    tol_lse = ds + 4 * e + chain + 4 * e * np.abs(np.where(np.isfinite(lse), lse, 0))
    return tol_out, tol_lse
