"""Plain fp64 CPU oracle for rotary positions, the paged key-value cache and attention over it.  TEST INFRASTRUCTURE ONLY.

Everything is the definition written out, row by row: angles from the formula of the frequencies, e4m3 as the table of its 256
codes with the nearest one searched for, attention as a full softmax over the positions a query sees.
"""
from __future__ import annotations

import math

import numpy as np

__all__ = ["rotary_frequencies", "rotate_rows", "e4m3_values", "e4m3_encode", "cached_attention"]


def rotary_frequencies(rot, base=10000.0, scaling="none", factor=1.0, trained_length=4096.0):
    """(radians per position of the rot/2 pairs, amplitude)."""
    if scaling == "base" and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    f = np.array([base ** (-2.0 * i / rot) for i in range(rot // 2)])
    if scaling == "linear":
        f = f / factor
    if scaling == "blend":
        turns = trained_length * f / (2 * math.pi)
        keep = np.clip((turns - 1.0) / 31.0, 0.0, 1.0)
        f = keep * f + (1.0 - keep) * f / factor
    return f, (1.0 + 0.1 * math.log(factor) if scaling == "blend" else 1.0)


def rotate_rows(x, positions, freqs, amplitude=1.0, interleaved=False, back=False):
    """x [rows, heads, d]: the first 2 len(freqs) elements of a row turned in pairs by positions[row] * freqs."""
    x = np.asarray(x, dtype=np.float64)
    out = x.copy()
    n = len(freqs)
    for row, p in enumerate(np.asarray(positions).reshape(-1).tolist()):
        for i in range(n):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
            w = math.fmod(p * freqs[i], 2 * math.pi) * (-1.0 if back else 1.0)
            c, s = math.cos(w), math.sin(w)
            out[row, :, a] = amplitude * (x[row, :, a] * c - x[row, :, b] * s)
            out[row, :, b] = amplitude * (x[row, :, a] * s + x[row, :, b] * c)
    return out


def e4m3_values():
    """The value of each of the 256 codes: sign, 4 exponent bits (bias 7), 3 mantissa bits; both codes of all ones are NaN."""
    out = np.empty(256)
    for code in range(256):
        sign, e, m = (-1.0 if code & 128 else 1.0), (code >> 3) & 15, code & 7
        out[code] = math.nan if e == 15 and m == 7 else sign * (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return out


def e4m3_encode(row):
    """(codes, e): the smallest whole e >= -126 with the largest finite |x| 2^-e at most 448, and each x 2^-e as the code of the nearest
    value under 2^128, the even code of two equally near ones; NaN and infinities as a NaN code (0x7f)."""
    row = np.asarray(row, dtype=np.float64)
    finite = np.isfinite(row)
    amax = np.abs(row[finite]).max() if finite.any() else 0.0
    e = -126
    while amax * 2.0 ** -e > 448.0:
        e += 1
    grid = e4m3_values()[:127]                   # the non-negative ones, ascending
    codes = np.empty(row.size, dtype=np.uint8)
    for i, x in enumerate(row):
        if not np.isfinite(x):
            codes[i] = 0x7F
            continue
        y = abs(x) * 2.0 ** -e
        j = min(int(np.searchsorted(grid, y)), 126)
        if j > 0:
            lo, hi = y - grid[j - 1], grid[j] - y
            if lo < hi or (lo == hi and (j - 1) % 2 == 0):
                j -= 1
        if grid[j] * 2.0 ** e >= 2.0 ** 128:     # finite values stay finite: 240 * 2^120 is the largest stored
            j -= 1
        codes[i] = j | (128 if np.signbit(x) else 0)
    return codes, e


def cached_attention(Q, K, V, lens, visible=None):
    """Q [B, N, G, h, d]; K[b], V[b] [length, h, d] of each sequence; query n sits at position lens[b] - N + n.  `visible` [B][length] can
    hide positions altogether.  Returns O [B, N, G, h, d] and LSE [B, N, G, h]; queries that see nothing give zeros and -inf."""
    Q = np.asarray(Q, dtype=np.float64)
    B, N, G, h, d = Q.shape
    O, L = np.zeros(Q.shape), np.full(Q.shape[:-1], -np.inf)
    for b in range(B):
        for n in range(N):
            p = int(lens[b]) - N + n
            seen = [t for t in range(p + 1) if visible is None or visible[b][t]]
            if not seen:
                continue
            for hh in range(h):
                k, v = (np.asarray(x[b], dtype=np.float64)[seen, hh] for x in (K, V))
                s = k @ Q[b, n, :, hh].T / math.sqrt(d)              # [seen, G]
                m = s.max(axis=0)
                m = np.where(m == -np.inf, 0.0, m)
                w = np.exp(s - m)
                z = w.sum(axis=0)
                for g in range(G):
                    if z[g] > 0:
                        O[b, n, g, hh] = (w[:, g] / z[g]) @ v
                        L[b, n, g, hh] = m[g] + math.log(z[g])
    return O, L
