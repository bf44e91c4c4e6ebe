"""Plain fp64 CPU oracle for the block around the experts: the gate by scores, the norm of the residual stream, rows in 8 bits and the experts'
products on them.  TEST INFRASTRUCTURE ONLY.

Definitions written out: the gate token by token, e4m3 by a search in the table of its values, products expert by expert.
"""
from __future__ import annotations

import math

import numpy as np

from .cache_oracle import e4m3_values

__all__ = ["score_gate", "score_gate_bwd", "add_norm", "add_norm_bwd", "pack8", "unpack8", "plinear8", "mlp8"]


def _softmax(x):
    """Of a row without NaN; +inf entries share the weight, as all do where every entry is -inf."""
    top = x.max()
    w = np.exp(np.where(x == top, 0.0, x - (top if np.isfinite(top) else 0.0))) if np.isfinite(top) else (x == top).astype(float)
    return w / w.sum()


def _log_sigmoid(x):
    return np.minimum(x, 0.0) - np.log1p(np.exp(-np.abs(x)))


def _row(logits):
    x = np.asarray(logits, dtype=np.float64).copy()
    x[np.isnan(x)] = -np.inf
    return x


def score_gate(logits, k, score="softmax", bias=None, groups=1, kept_groups=1, group_best=1, renormalise=True, scale=1.0):
    """(expert_idxs [T, k], gates [T, k])."""
    T, E = logits.shape
    idx, gates = np.zeros((T, k), dtype=np.int32), np.zeros((T, k))
    per = E // groups
    for t in range(T):
        x = _row(logits[t])
        if score == "softmax":
            s = _softmax(x)
        else:
            with np.errstate(over="ignore"):
                s = 1.0 / (1.0 + np.exp(-x))
        with np.errstate(invalid="ignore"):
            rank = s + (0.0 if bias is None else np.asarray(bias, dtype=np.float64))
        rank[np.isnan(rank) | (x == -np.inf)] = -np.inf
        if bias is None and (group_best == 1 or kept_groups == groups):
            rank = x                                            # exact scores compared: 64 bits do not hold those next to 1 or 0 apart
        worth = []
        for g in range(groups):
            live = sorted((r for r in rank[g * per:(g + 1) * per] if r > -np.inf), reverse=True)[:group_best]
            worth.append(sum(live) if live else -np.inf)
        kept = sorted(range(groups), key=lambda g: (-worth[g], g))[:kept_groups]
        inside = [e for e in range(E) if e // per in kept]
        chosen = sorted(inside, key=lambda e: (-rank[e], e))[:k]
        idx[t] = chosen
        if renormalise:
            w = _softmax(x[chosen]) if score == "softmax" else _softmax(np.where(x[chosen] == -np.inf, -np.inf, _log_sigmoid(x[chosen])))
        else:
            w = s[chosen]
        gates[t] = scale * w
    return idx, gates


def score_gate_bwd(logits, idx, dgates, score="softmax", renormalise=True, scale=1.0):
    """dlogits: of every slot's weight as a function of the logits, slot by slot."""
    T, E = logits.shape
    out = np.zeros((T, E))
    for t in range(T):
        x = _row(logits[t])
        slots = [j for j in range(idx.shape[1]) if 0 <= idx[t, j] < E and x[idx[t, j]] > -np.inf]
        e = [int(idx[t, j]) for j in slots]
        dw = np.array([scale * dgates[t, j] for j in slots])
        if not slots:
            continue
        with np.errstate(over="ignore"):
            s = 1.0 / (1.0 + np.exp(-x))
            rest = 1.0 / (1.0 + np.exp(x))
        if renormalise:
            w = _softmax(x[e]) if score == "softmax" else _softmax(_log_sigmoid(x[e]))
            d = w * (dw - (w * dw).sum())
            if score == "sigmoid":
                d = d * rest[e]
        elif score == "sigmoid":
            d = dw * s[e] * rest[e]
        else:
            p = _softmax(x)
            d = dw * p[e]
            out[t] -= np.where(x == -np.inf, 0.0, p) * d.sum()
        for j, q in enumerate(e):
            out[t, q] += d[j]
    return out


def add_norm(x, r, weight, eps):
    """(s, y, rstd)."""
    s = np.asarray(x, dtype=np.float64) + (0.0 if r is None else np.asarray(r, dtype=np.float64))
    rstd = 1.0 / np.sqrt((s * s).mean(-1) + eps)
    return s, s * rstd[..., None] * np.asarray(weight, dtype=np.float64), rstd


def add_norm_bwd(dy, ds, s, weight, rstd):
    """(dx, dweight) with rstd as it was kept, a function of s."""
    dy, s, w = (np.asarray(a, dtype=np.float64) for a in (dy, s, weight))
    u = s * np.asarray(rstd, dtype=np.float64)[..., None]
    g = dy * w
    dx = np.asarray(rstd, dtype=np.float64)[..., None] * (g - u * (g * u).mean(-1, keepdims=True))
    return dx + (0.0 if ds is None else np.asarray(ds, dtype=np.float64)), (dy * u).reshape(-1, s.shape[-1]).sum(0)


def pack8(x):
    """x [rows, d] -> (codes [rows, P], exponent bytes [rows, P / 32]), P whole 128s, the padding packed as zeros: cache_oracle's e4m3_encode of
    every block, all at once."""
    rows, d = x.shape
    P = -(-d // 128) * 128
    full = np.zeros((rows, P))
    full[:, :d] = x
    blocks = full.reshape(rows, P // 32, 32)
    finite = np.isfinite(blocks)
    size = np.where(finite, np.abs(blocks), 0.0)
    top = size.max(-1)
    e = np.full(top.shape, -126)
    mantissa, exponent = np.frexp(top)                       # top = mantissa 2^exponent, 448 = 0.875 * 2^9
    e = np.where(top > 0, np.maximum(exponent - 9 + (mantissa > 0.875), -126), -126)
    grid = e4m3_values()[:127]
    y = np.ldexp(size, -e[..., None])
    hi = np.minimum(np.searchsorted(grid, y), 126)
    lo = np.maximum(hi - 1, 0)
    down, up = y - grid[lo], grid[hi] - y
    code = np.where((hi > 0) & ((down < up) | ((down == up) & (lo % 2 == 0))), lo, hi)
    code = np.where(np.ldexp(grid[code], e[..., None]) >= 2.0 ** 128, code - 1, code)
    code = np.where(finite, code | np.where(np.signbit(blocks), 128, 0), 0x7F).astype(np.uint8)
    return code.reshape(rows, P), (e + 127).astype(np.uint8)


def unpack8(codes, exps, d):
    values = e4m3_values()[codes] * np.repeat(2.0 ** (exps.astype(np.float64) - 127), 32, axis=-1)
    return values[..., :d]


def _activation(h, act):
    if act == 2:
        gate, up = np.split(h, 2, axis=-1)
        return gate / (1.0 + np.exp(-gate)) * up
    return np.array([0.5 * v * math.erfc(-v / math.sqrt(2)) for v in h.ravel()]).reshape(h.shape)


def plinear8(X, W, idx, gates=None):
    """X [T, d_in] and W [E, d_in, d_out] as the values they stand for, idx [T, k].  Per slot [T * k, d_out], or weighted sums [T, d_out]."""
    T, k = idx.shape
    y = np.stack([X[t] @ W[idx[t, j]] for t in range(T) for j in range(k)])
    return y if gates is None else (y.reshape(T, k, -1) * np.asarray(gates, dtype=np.float64)[..., None]).sum(1)


def mlp8(X, W1, W2, idx, gates, act, slack=None, rounding=0.0):
    """(Y [T, d_model], tolerance [T, d_model]): Alg. 3 with the hidden rows packed to 8 bits.  `slack`(x, W) bounds the error of a product x W before
    it is rounded; the tolerance is what it does to Y: hidden values that it moves to another code, and the second product's own, whose rows
    may then be rounded once, by `rounding` of a value, or 2^-8 of that of the largest, at most."""
    T, k = idx.shape
    Y, tol = np.zeros((T, W2.shape[2])), np.zeros((T, W2.shape[2]))
    for t in range(T):
        for j in range(k):
            e = idx[t, j]
            pre = X[t] @ W1[e]
            h = _activation(pre, act)
            d = h.shape[0]
            q = unpack8(*pack8(h[None]), d)[0]
            y = q @ W2[e]
            Y[t] += gates[t, j] * y
            if slack is None:
                continue
            err = slack(X[t], W1[e])
            # the activation moves by its derivative, at most 1.13 times, and by 8 roundings of fp32
            if act == 2:
                gate, up = np.split(np.abs(pre), 2)
                eg, eu = np.split(err, 2)
                moved = 1.13 * eg * (up + eu) + eu * (gate + eg) + 2.0 ** -21 * np.abs(h)
            else:
                moved = 1.13 * err + 2.0 ** -21 * np.abs(pre)
            lo, hi = (unpack8(*pack8((h + s * moved)[None]), d)[0] for s in (-1, 1))
            # a block whose largest value is that near to a power's border may be stored in steps of the next power
            a = np.abs(h) + moved
            b = np.maximum(np.abs(h) - moved, 0)
            P = -(-d // 32) * 32
            top = lambda v: np.pad(v, (0, P - d)).reshape(-1, 32).max(1)
            other = np.ceil(np.log2(np.maximum(top(a), 2.0 ** -200) / 448)) != np.ceil(np.log2(np.maximum(top(b), 2.0 ** -200) / 448))
            step = np.maximum(np.abs(h) * 2.0 ** -3, np.repeat(top(a), 32)[:d] * 2.0 ** -17)
            dq = np.maximum(np.maximum(np.abs(lo - q), np.abs(hi - q)), np.where(np.repeat(other, 32)[:d], step, 0.0))
            off = dq @ np.abs(W2[e]) + slack(np.abs(q) + dq, W2[e])
            tol[t] += abs(gates[t, j]) * (off + rounding * (np.abs(y) + off + 2.0 ** -8 * (np.abs(y) + off).max()))
    return Y, tol
