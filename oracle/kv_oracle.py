"""The key-value cache's operators in 64 bits, from their definitions (numpy; shares nothing with the library).

Caches are [pages, heads, page_size, D] arrays; an 8-bit cache is given as codes with their scales, or as the values that they stand for.
"""
from __future__ import annotations

import numpy as np


def angles(positions, freqs, sections):
    """[tokens, pairs] angles, reduced to a turn with 64 bits of mantissa."""
    positions = np.atleast_2d(np.asarray(positions))
    axis = np.repeat(np.arange(len(sections)), sections)
    a = positions[axis].T.astype(np.longdouble) * np.asarray(freqs, dtype=np.longdouble)
    turn = 2 * np.longdouble("3.14159265358979323846264338327950288")
    return (a - turn * np.rint(a / turn)).astype(np.float64)


def rotary(x, positions, freqs, sections=None, adjacent=False, inverse=False):
    """[tokens, heads, D] with each pair turned by its angle."""
    pairs = len(freqs)
    a = angles(positions, freqs, sections if sections is not None else (pairs,))[:, None, :]
    if inverse:
        a = -a
    y = np.array(x, dtype=np.float64)
    first, second = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if adjacent else (slice(0, pairs), slice(pairs, 2 * pairs))
    u, v = np.array(y[..., first]), np.array(y[..., second])
    y[..., first] = u * np.cos(a) - v * np.sin(a)
    y[..., second] = u * np.sin(a) + v * np.cos(a)
    return y


def quantize(y):
    """(scale, exact quotients) of rows: codes are the quotients rounded.  Rows that are not finite: scale NaN, quotients 0."""
    with np.errstate(invalid="ignore", divide="ignore"):
        top = np.abs(y).max(-1)
        bad = ~np.isfinite(y).all(-1)
        v = np.where((top > 0)[..., None] & ~bad[..., None], 127 * y / np.where(top > 0, top, 1)[..., None], 0.0)
        return np.where(bad, np.nan, top / 127), v


def attention(q, k_cache, v_cache, table, lengths, alpha, softcap=0.0, slopes=None, window=0, max_length=None):
    """(out, lse, weight) of q [sequences, tokens, heads, D]: weight = (sum_n p |v|, largest |score| of a visible position, largest sum_d |alpha q k|, largest |v|), what bounds of
    rounding errors are proportional to."""
    B, T, Hq, D = q.shape
    pages, H, page_size, _ = k_cache.shape
    G = Hq // H
    out, lse = np.zeros(q.shape), np.full(q.shape[:3], -np.inf)
    mass, peak, dot, most = np.zeros(q.shape), np.zeros(q.shape[:3]), np.zeros(q.shape[:3]), np.zeros(q.shape[:3])
    room = min(table.shape[1] * page_size, max_length or 1 << 62)
    for b in range(B):
        length = min(max(int(lengths[b]), 0), room)
        n = np.arange(length)
        page = table[b, n // page_size]
        there = (page >= 0) & (page < pages)
        for h in range(H):
            k = k_cache[np.where(there, page, 0), h, n % page_size]
            v = v_cache[np.where(there, page, 0), h, n % page_size]
            for t in range(T):
                at = length - T + t
                see = there & (n <= at) & ((n > at - window) if window > 0 else True)
                if not see.any():
                    continue
                ks, vs, gap = k[see], v[see], n[see] - at
                for i in range(h * G, (h + 1) * G):
                    s = alpha * (ks @ q[b, t, i])
                    if softcap > 0:
                        s = softcap * np.tanh(s / softcap)
                    if slopes is not None:
                        s = s + slopes[i] * gap
                    top = s.max()
                    e = np.exp(s - top)
                    p = e / e.sum()
                    out[b, t, i] = p @ vs
                    lse[b, t, i] = top + np.log(e.sum())
                    mass[b, t, i] = p @ np.abs(vs)
                    # (positions that weigh nothing do not count)
                    near = p > 1e-12
                    peak[b, t, i] = np.abs(s[near]).max() + (np.abs(slopes[i] * gap[near]).max() if slopes is not None else 0)
                    most[b, t, i] = np.abs(vs).max()
                    dot[b, t, i] = abs(alpha) * (np.abs(ks[near]) @ np.abs(q[b, t, i])).max()
    return out, lse, (mass, peak, dot, most)
