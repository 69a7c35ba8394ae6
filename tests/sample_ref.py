"""Sampling in plain float64 (numpy): what mad_sample computes for one row."""
import numpy as np


def row(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """x [V] float64 -> (token, probabilities float64 [V]); (-1, zeros) for a row without a distribution."""
    V = len(x)
    p = np.zeros(V)
    if np.isnan(x).any() or x.max() == -np.inf:
        return -1, p
    order = np.argsort(-x, kind="stable")
    if temperature == 0:
        order, w = order[:1], np.ones(1)
    else:
        if 0 < top_k < V:
            order = order[:top_k]
        top = x[order[0]]
        with np.errstate(invalid="ignore"):
            w = np.where(x[order] == top, 1.0, np.exp((x[order] - top) / temperature))
        part = np.cumsum(w)
        n = len(order)
        if top_p < 1:
            n = int((part - w < top_p * part[-1]).sum())
        n = min(n, int((w >= min_p).sum()))
        order, w = order[:n], w[:n]
    p[order] = w
    part = np.cumsum(p)
    p /= part[-1]
    if u is None:
        return None, p
    over = np.nonzero(part > float(u) * part[-1])[0]
    return int(over[0]) if len(over) else int(np.nonzero(p > 0)[0][-1]), p


def near_edge(x, u, tol=1e-9, **kw):
    """Whether u lies within tol of a bin edge of the row's distribution (the draw may then fall to either side)."""
    _, p = row(x, u, **kw)
    c = np.cumsum(p)
    return bool((np.abs(c - float(u)) < tol).any())


def check_row(x, u, tok, probs, what="", **kw):
    """tok and probs (None: not asked for) of a kernel against the reference: the token exactly, every probability to
    half an fp32 step (2^-24 relative) with a factor 2 for the sums behind it."""
    want, p = row(x, u, **kw)
    if tok is not None:
        assert tok == want, f"{what}: token {tok}, expected {want} ({kw})"
    if probs is not None:
        probs = np.asarray(probs, dtype=np.float64)
        assert np.array_equal(probs > 0, np.float32(p) > 0), f"{what}: {int(((probs > 0) != (np.float32(p) > 0)).sum())} entries in or out ({kw})"
        err = np.abs(probs - p)
        assert np.all(err <= 2.0 ** -23 * p + 2.0 ** -149), f"{what}: off by {(err / np.maximum(p, 1e-300)).max():.2e} relative ({kw})"
