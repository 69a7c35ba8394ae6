"""Token log probabilities in plain numpy float64, a row at a time, with bounds for what fp32 arithmetic may lose."""
import numpy as np

E = 2.0 ** -24


def row(x, tok, top_n, temperature):
    """x [V] float64 -> dict of (value, tolerance) or exact values.

    Bounds, e = 2^-24, d = (x - max) / temperature in natural units: a term exp(d) has an argument with two roundings
    (difference, product, |d| 2 e) and one of the factor (|d| e), and the power's own (2 e); sums of at most 16 terms in
    fp32 (16 e), then fp64.  So the mass is off by sum p (3 |d| + 18) e = S, with it every log p; log p's own difference and
    product are fp64 on the rounded factor (|d| e), the result is rounded once (e |log p|).  The entropy sums p d: each
    term's error times |d|, and that of the mass; the product e d and its sum add 18 e |d| more."""
    x = np.asarray(x, np.float64)
    V = len(x)
    none = np.isnan(x).any() or np.isneginf(x).all()
    at = np.argsort(-np.where(np.isnan(x), 0, x), kind="stable")[:top_n]
    if none:
        return dict(logp=np.nan, rank=-1, entropy=np.nan, top_tok=np.full(top_n, -1), top_logp=np.full(top_n, np.nan), S=0.0, tol_entropy=0.0)
    m = x.max()
    with np.errstate(invalid="ignore", divide="ignore"):
        d = np.where(x == m, 0.0, -np.inf) if np.isposinf(m) else (x - m) / temperature
        p = np.exp(d)
        z = p.sum()
        p /= z
        lp = d - np.log(z)
    live = p > 0
    a = np.abs(np.where(live, d, 0))
    S = (p * (3 * a + 18)).sum() * E
    got = dict(entropy=-(p[live] * lp[live]).sum(), top_tok=at, top_logp=lp[at], S=S,
               tol_entropy=(p * a * (3 * a + 36)).sum() * E + S * (1 + (p * a).sum()) + E * (p * a).sum())
    got["tol_entropy"] += E * abs(got["entropy"])
    if 0 <= tok < V:
        got.update(logp=lp[tok], rank=int(((x > x[tok]) | ((x == x[tok]) & (np.arange(V) < tok))).sum()))
    else:
        got.update(logp=-np.inf, rank=V)
    return got


def close(got, want, S):
    """log probabilities within the bound; infinities and NaN alike."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    fin = np.isfinite(want)
    with np.errstate(invalid="ignore"):
        return np.array_equal(got[~fin], want[~fin], equal_nan=True) and bool(np.all(np.abs(got - want)[fin] <= (S + 3 * E * np.abs(want) + E * 2)[fin] if np.ndim(want) else (not fin or abs(got - want) <= S + 3 * E * abs(want) + 2 * E)))
