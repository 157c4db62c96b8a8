"""Linears, routing and MoE layers in 8-bit integers, in numpy and 64 bits.

A row's scale is fp32(max |v| / 127), its codes round-half-even(v / scale) of the exact quotient (of two binary32
numbers it is at least 2^-33 of itself away from a tie that it is not, so the 64-bit quotient decides alike).
"""
import numpy as np

MIN_SCALE = np.float32(2.0 ** -126)


def quantize_rows(v):
    """v [R, K] of at most 32 bits -> (codes int8 [R, K], scales fp32 [R])."""
    v = np.asarray(v, dtype=np.float32)
    with np.errstate(all="ignore"):
        top = np.max(np.abs(v), axis=1) if v.shape[1] else np.zeros(v.shape[0], np.float32)
        scale = (top / np.float32(127)).astype(np.float32)
        q = np.rint(v.astype(np.float64) / scale.astype(np.float64)[:, None])
    bad = ~np.isfinite(top)
    small = ~bad & (scale < MIN_SCALE)
    scale = np.where(bad, np.float32(np.nan), np.where(small, np.float32(0), scale)).astype(np.float32)
    q = np.where((bad | small)[:, None], 0, q)
    return q.astype(np.int8), scale


def w8a8_linear(X, codes, scales):
    """[M, N] in fp64 from X [M, K] and the codes [N, K], scales [N] of a weight."""
    xq, xs = quantize_rows(X)
    acc = xq.astype(np.float64) @ codes.astype(np.float64).T        # whole numbers below 2^31: exact
    return acc * xs.astype(np.float64)[:, None] * scales.astype(np.float64)[None, :]


def moe_route(X, Wg, topk, renormalize, n_shared):
    logits = np.asarray(X, np.float64) @ np.asarray(Wg, np.float64).T
    T, E = logits.shape
    nan = np.isnan(logits)
    order = np.argsort(np.where(nan, np.inf, -logits), axis=1, kind="stable")
    # (a NaN behind the infinities that stand for -inf logits)
    order = np.stack([np.concatenate([o[~n[o]], o[n[o]]]) for o, n in zip(order, nan)])
    ids = order[:, :topk]
    with np.errstate(all="ignore"):
        w = np.exp(logits - np.take_along_axis(logits, ids[:, :1], 1))
        gates = np.take_along_axis(w, ids, 1)
        gates = gates / (gates if renormalize else w).sum(1, keepdims=True)
    gates[nan.any(1)] = np.nan
    ids = np.concatenate([ids, np.tile(np.arange(E, E + n_shared), (T, 1))], 1)
    return ids.astype(np.int32), np.concatenate([gates, np.ones((T, n_shared))], 1)


def w8a8_moe(X, experts, ids, gates, border=0.0):
    """experts: list of ((codes, scales) of w1, w3, w2).  Returns (Y, doubt, terms): the layer's output, how far it moves if
    every code of the SwiGLU rows whose quotient lies within `border` of a border between two codes takes the other one, and
    the sum of the magnitudes of the pairs' terms."""
    T, H = X.shape
    Y, doubt, terms = np.zeros((T, H)), np.zeros((T, H)), np.zeros((T, H))
    for e, (w1, w3, w2) in enumerate(experts):
        rows = np.nonzero((ids == e).any(1))[0]
        if not len(rows):
            continue
        g = np.where(ids[rows] == e, gates[rows].astype(np.float64), 0.0).sum(1)[:, None]
        a, b = w8a8_linear(X[rows], *w1), w8a8_linear(X[rows], *w3)
        with np.errstate(all="ignore"):
            h = a / (1.0 + np.exp(-a)) * b
            top = np.max(np.abs(h), axis=1, keepdims=True)
            step = top / 127.0
            u = np.where(step > 0, h / step, 0.0)
        q = np.rint(u)
        near = np.abs(np.abs(u - np.floor(u)) - 0.5) <= border
        c2, s2 = w2[0].astype(np.float64), w2[1].astype(np.float64)[None, :]
        term = (q @ c2.T) * step * s2 * g
        Y[rows] += term
        terms[rows] += np.abs(term)
        doubt[rows] += (near.astype(np.float64) @ np.abs(c2).T) * step * s2 * np.abs(g)
    return Y, doubt, terms
