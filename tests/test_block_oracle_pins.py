"""Pins of the oracle for the gate by scores, the norm and the products in 8 bits: hand values, library functions, differences (CPU)."""
import math

import numpy as np
import pytest
import torch

import oracle


def test_gate_by_hand():
    """Four experts, two groups.  Sigmoid of ln 3 is 3/4, of 0 1/2, of -ln 3 1/4, of -ln 9 1/10."""
    x = np.array([[0.0, math.log(3), -math.log(3), -math.log(9)]])
    idx, w = oracle.score_gate(x, 2, "sigmoid")
    assert idx.tolist() == [[1, 0]] and np.allclose(w, [[0.6, 0.4]])
    idx, w = oracle.score_gate(x, 2, "sigmoid", bias=np.array([0.0, 0.0, 0.3, 0.7]), renormalise=False, scale=2.0)     # ranks 0.5, 0.75, 0.55, 0.8
    assert idx.tolist() == [[3, 1]] and np.allclose(w, [[0.2, 1.5]])
    # groups (0, 1) and (2, 3): bests 0.75 and 0.8 by one, 1.25 and 1.35 by two
    idx, _ = oracle.score_gate(x, 2, "sigmoid", bias=np.array([0.0, 0.0, 0.3, 0.7]), groups=2, kept_groups=1, group_best=2)
    assert idx.tolist() == [[3, 2]]
    idx, w = oracle.score_gate(np.log(np.array([[1.0, 4.0, 2.0, 3.0]])), 2, "softmax", renormalise=False)
    assert idx.tolist() == [[1, 3]] and np.allclose(w, [[0.4, 0.3]])


def test_gate_is_the_plain_one_for_renormalised_softmax():
    x = np.random.default_rng(0).normal(size=(20, 16))
    for a, b in zip(oracle.score_gate(x, 4), oracle.topk_gate(x.astype(np.float64), 4)):
        assert np.allclose(a, b)


def test_masked_experts_and_rows():
    inf = math.inf
    x = np.array([[-inf, 1.0, math.nan, 2.0], [-inf] * 4, [inf, 0.0, inf, 1.0]])
    idx, w = oracle.score_gate(x, 3, "softmax", bias=np.array([9.0, 0.0, 9.0, 0.0]))
    assert idx[0].tolist() == [3, 1, 0] and w[0, 2] == 0 and idx[1].tolist() == [0, 1, 2] and np.allclose(w[1], 1 / 3)
    assert np.allclose(w[2, :2].sum(), 1.0)
    _, w = oracle.score_gate(x, 3, "sigmoid", renormalise=False)
    assert w[1].tolist() == [0, 0, 0]
    _, w = oracle.score_gate(np.full((1, 3), -800.0) + np.array([0.0, math.log(2), math.log(5)]), 3, "sigmoid")
    assert np.allclose(w, [[5 / 8, 2 / 8, 1 / 8]])              # ratios stay where the scores underflow


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [False, True])
def test_gate_gradient_by_differences(score, renormalise):
    g = np.random.default_rng(1)
    x, dw, k = g.normal(size=(3, 9)), g.normal(size=(3, 4)), 4
    rule = dict(score=score, renormalise=renormalise, scale=1.7)
    idx, _ = oracle.score_gate(x, k, **rule)
    got = oracle.score_gate_bwd(x, idx, dw, **rule)
    for t in range(3):
        for e in range(9):
            d = np.zeros_like(x)
            d[t, e] = 1e-6
            up, down = ((oracle.score_gate(x + s * d, k, **rule)[1] * dw).sum() for s in (1, -1))
            assert abs((up - down) / 2e-6 - got[t, e]) < 1e-8


def test_norm_against_the_library_and_differences():
    g = np.random.default_rng(2)
    x, r, w, dy, ds = g.normal(size=(4, 7)), g.normal(size=(4, 7)), g.normal(size=7), g.normal(size=(4, 7)), g.normal(size=(4, 7))
    s, y, rstd = oracle.add_norm(x, r, w, 1e-3)
    want = torch.nn.functional.rms_norm(torch.from_numpy(x + r), (7,), torch.from_numpy(w), 1e-3).numpy()
    assert np.allclose(y, want)
    dx, dweight = oracle.add_norm_bwd(dy, ds, s, w, rstd)
    loss = lambda x_, w_: sum((a * b).sum() for a, b in zip(oracle.add_norm(x_, r, w_, 1e-3)[:2], (ds, dy)))
    for i in range(4):
        for j in range(7):
            d = np.zeros_like(x)
            d[i, j] = 1e-6
            assert abs((loss(x + d, w) - loss(x - d, w)) / 2e-6 - dx[i, j]) < 1e-7
    for j in range(7):
        d = np.zeros(7)
        d[j] = 1e-6
        assert abs((loss(x, w + d) - loss(x, w - d)) / 2e-6 - dweight[j]) < 1e-7


def test_packed_rows_by_hand():
    x = np.zeros((1, 40))
    x[0, :3], x[0, 33] = [448.0, -1.0, 0.1], 449.0
    codes, exps = oracle.pack8(x)
    assert codes.shape == (1, 128) and exps.tolist() == [[127, 128, 1, 1]]
    back = oracle.unpack8(codes, exps, 40)
    assert back[0, 0] == 448 and back[0, 1] == -1 and back[0, 2] == 0.1015625 and back[0, 33] == 448     # 449 / 2 = 224.5, to 224
    assert (codes[0, 40:] == 0).all()


def test_packed_rows_are_the_caches_block_by_block():
    """e4m3 with a power of two, as the oracle of the cache searches it out one value at a time."""
    g = np.random.default_rng(5)
    x = g.normal(size=(40, 64)) * np.exp(g.normal(size=(40, 1)) * 20)
    x[0] = 0
    x[1, 3], x[2, 4], x[3] = math.nan, -math.inf, math.inf
    x[4] *= 2.0 ** -150
    x[5] = np.sign(x[5]) * 1.96 * 2.0 ** 127
    x[6, 0], x[6, 1:] = 448.0, 2.0 ** -10 * np.arange(63)
    x[7, 0], x[7, 1:] = 448.0, 16 + 0.5 * np.arange(63)
    x[8] = -0.0
    codes, exps = oracle.pack8(x)
    for i in range(40):
        for b in range(2):
            want, e = oracle.e4m3_encode(x[i, 32 * b:32 * b + 32])
            assert np.array_equal(codes[i, 32 * b:32 * b + 32], want) and exps[i, b] == e + 127, (i, b)


def test_packed_products_are_the_plain_ones_on_exact_values():
    """Small whole numbers are exact in 8 bits, also as hidden rows of an activation that keeps them (GELU far from 0 is the identity)."""
    g = np.random.default_rng(3)
    X, W = g.integers(-3, 4, size=(5, 33)).astype(float), g.integers(-2, 3, size=(3, 33, 8)).astype(float)
    assert (oracle.unpack8(*oracle.pack8(X), 33) == X).all()
    idx = np.array([[0, 1], [2, 0], [1, 2], [0, 2], [1, 0]])
    gates = g.random(size=(5, 2))
    want = np.stack([sum(gates[t, j] * (X[t] @ W[idx[t, j]]) for j in range(2)) for t in range(5)])
    assert np.allclose(oracle.plinear8(X, W, idx, gates), want)
    W1, W2 = np.abs(W[:, :, :4]) + 1, g.integers(-2, 3, size=(3, 4, 6)).astype(float)
    X = np.full((5, 33), 1.0)
    got, _ = oracle.mlp8(X, W1, W2, idx, gates, 1)
    h = [oracle.unpack8(*oracle.pack8((X[0] @ W1[e])[None]), 4)[0] for e in range(3)]
    want = np.stack([sum(gates[t, j] * (h[idx[t, j]] @ W2[idx[t, j]]) for j in range(2)) for t in range(5)])
    assert np.allclose(got, want)


def test_a_planted_mistake_shows():
    """A gate that lets the bias into its weights, and hidden rows that are not packed, differ from the oracle by more than any tolerance."""
    g = np.random.default_rng(4)
    x, b = g.normal(size=(6, 8)), 0.3 * g.normal(size=8)
    idx, w = oracle.score_gate(x, 2, "sigmoid", bias=b)
    s = 1 / (1 + np.exp(-x)) + b
    wrong = np.take_along_axis(s, idx, 1)
    assert np.abs(wrong / wrong.sum(1, keepdims=True) - w).max() > 1e-3
    X, W1, W2 = g.normal(size=(6, 32)), g.normal(size=(8, 32, 64)) / 6, g.normal(size=(8, 32, 8)) / 6
    Y, tol = oracle.mlp8(X, W1, W2, idx, w, 2, slack=lambda x, W: np.full(W.shape[1], 1e-6))
    pre = np.stack([[X[t] @ W1[e] for e in idx[t]] for t in range(6)])
    h = pre[..., :32] / (1 + np.exp(-pre[..., :32])) * pre[..., 32:]
    plain = np.stack([sum(w[t, j] * (h[t, j] @ W2[idx[t, j]]) for j in range(2)) for t in range(6)])
    assert (np.abs(plain - Y) > tol).any() and np.abs(plain - Y).max() > 1e-3
