"""The gate by scores, the norm of the residual stream, rows in 8 bits and the experts' products on them, against the fp64 oracle."""
import sys

import numpy as np
import pytest
import torch

import oracle

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}     # what a rounding is off by at most, relative to the value
EPS32 = 2.0 ** -24
ROW = 2.0 ** -11                    # rows of a weighted sum may be held in fp16, with a power of two for 128 of them


def _log(*a):
    print(*a, flush=True, file=sys.stderr)


@pytest.fixture(scope="module")
def smoe():
    import paper_2403_08245_amd as m
    return m


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _normal(shape, seed, dtype=torch.bfloat16, std=1.0):
    return (torch.randn(*shape, generator=_gen(seed), dtype=torch.float32) * std).to(dtype)


def _f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def _near(got, want, tol, what=""):
    got, want = _f64(got), np.asarray(want)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert np.isfinite(got).all(), what
    over = np.abs(got - want) - tol
    assert (over <= 0).all(), f"{what}: {int((over > 0).sum())} of {over.size} over the bound, worst by {over.max():.3e}"


# --------------------------------------------------------------------------------------------------------------- gate
# Weights: an exponential of a difference rounded to 2^-24 of it, good to 2 units of 2^-24 (expf), the same for those it is divided by, their sum
# over six cross-lane steps and up to 16 of a lane's own, a division and a product.  Sigmoids: two exponentials and two divisions instead.
def _weight_units(x):
    live = np.where(np.isfinite(x), x, 0.0)
    return (2 * np.abs(live).max() + 2 * (live.max() - live.min()) + 40) * EPS32


GATES = [  # T, E, k, score, bias, groups, kept, best, renormalise, scale
    (1, 1, 1, "softmax", False, 1, 1, 1, True, 1.0), (5, 8, 2, "softmax", False, 1, 1, 1, False, 1.0), (33, 64, 8, "softmax", True, 1, 1, 1, True, 2.5),
    (7, 60, 6, "sigmoid", True, 5, 2, 2, True, 16.0), (130, 256, 8, "sigmoid", True, 8, 4, 2, True, 2.5), (9, 256, 8, "sigmoid", False, 8, 3, 1, False, 1.0),
    (6, 96, 5, "softmax", False, 8, 2, 2, False, 1.0), (4, 1000, 16, "sigmoid", True, 4, 1, 2, True, 1.0), (3, 1024, 64, "softmax", False, 1, 1, 1, False, 3.0),
    (5, 512, 12, "softmax", True, 16, 5, 1, True, 1.0), (8, 64, 64, "sigmoid", True, 64, 64, 1, True, 1.0), (11, 160, 7, "sigmoid", True, 5, 1, 2, False, 0.5),
    (2500, 256, 8, "sigmoid", True, 8, 4, 2, True, 2.5), (1501, 64, 6, "softmax", True, 1, 1, 1, False, 1.0), (999, 128, 16, "sigmoid", False, 16, 5, 2, True, 1.0), (700, 160, 5, "softmax", True, 5, 3, 1, True, 1.0),
    (800, 512, 8, "sigmoid", True, 8, 4, 2, True, 2.5), (300, 60, 6, "softmax", True, 5, 2, 2, True, 1.0), (200, 120, 4, "sigmoid", True, 3, 2, 2, True, 1.0), (200, 48, 3, "sigmoid", False, 4, 3, 2, False, 1.0),
    (150, 384, 12, "sigmoid", True, 4, 2, 1, True, 1.0), (4, 3, 3, "sigmoid", False, 3, 3, 2, True, 1.0), (2, 2, 1, "sigmoid", True, 2, 1, 2, True, 1.0), (6, 65, 3, "softmax", True, 13, 4, 2, True, -1.0),
]


@pytest.mark.parametrize("T,E,k,score,bias,groups,kept,best,renormalise,scale", GATES)
def test_gate_and_its_gradient(smoe, T, E, k, score, bias, groups, kept, best, renormalise, scale):
    _log(f"gate {(T, E, k, score, bias, groups, kept, best, renormalise, scale)}")
    x, b = _normal((T, E), 1, torch.float32, 2.0), _normal((E,), 2, torch.float32, 0.2) if bias else None
    rule = smoe.gate_rule(score, groups, kept, best, renormalise, scale)
    want = dict(score=score, renormalise=renormalise, scale=scale)
    idx, w = oracle.score_gate(_f64(x), k, bias=None if b is None else _f64(b), groups=groups, kept_groups=kept, group_best=best, **want)
    X = x.cuda()
    got, gates = smoe.score_gate(X, k, rule, None if b is None else b.cuda())
    assert np.array_equal(got.cpu().numpy(), idx)
    u = _weight_units(_f64(x))
    _near(gates, w, u * np.abs(w), "gates")
    dw = _normal((T, k), 3, torch.float32)
    dx = smoe.score_gate_bwd(X, got, dw.cuda(), rule)
    # every term of a gradient is a weight times a gradient of a gate, k of them in a mean (in the row's softmax: E small ones)
    kept_sum = np.abs(_f64(dw) * w).sum(1, keepdims=True)
    whole = np.abs(scale) * np.abs(_f64(dw)).sum(1, keepdims=True)
    _near(dx, oracle.score_gate_bwd(_f64(x), idx, _f64(dw), **want), 4 * (u + k * EPS32) * (kept_sum + whole * np.exp(_f64(x) - _f64(x).max(1, keepdims=True))), "dlogits")


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("E,groups,kept,best", [(8, 1, 1, 1), (12, 4, 2, 2), (60, 5, 3, 2), (64, 8, 4, 2), (256, 8, 3, 1), (480, 5, 2, 2)])
def test_gate_of_masked_infinite_and_equal_logits(smoe, score, renormalise, bias, E, groups, kept, best):
    _log(f"gate edges {score} {renormalise} {bias} {E}")
    inf, nan, k = float("inf"), float("nan"), 3
    x = _normal((10, E), 4, torch.float32)
    x[0] = -inf                                   # nothing to choose
    x[1] = nan
    x[2, :] = 0.25                                # ties everywhere
    x[3, 1:] = -inf                               # one expert
    x[4, 2] = inf
    x[5, [1, 3, 4]] = inf
    x[6, ::2] = nan
    x[7, : E - 2] = -inf
    x[8] = -0.0
    x[8, 1::2] = 0.0
    x[9] -= 300.0                                 # sigmoids that underflow
    b = None
    if bias:
        b = _normal((E,), 5, torch.float32, 0.5)
        b[1], b[2], b[5] = nan, -inf, inf
    rule = smoe.gate_rule(score, groups, kept, best, renormalise, 1.5)
    want = dict(score=score, renormalise=renormalise, scale=1.5)
    idx, w = oracle.score_gate(_f64(x), k, bias=None if b is None else _f64(b), groups=groups, kept_groups=kept, group_best=best, **want)
    X = x.cuda()
    got, gates = smoe.score_gate(X, k, rule, None if b is None else b.cuda())
    assert np.array_equal(got.cpu().numpy(), idx)
    u = 2 * 300 * EPS32 + _weight_units(_f64(x)[:9])
    _near(gates, w, u * np.abs(w) + 1e-37, "gates")                 # 1e-37: under it fp32 has fewer bits
    dw = _normal((10, k), 6, torch.float32)
    finite = [0, 1, 2, 3, 6, 7, 8, 9]
    dx = smoe.score_gate_bwd(X, got, dw.cuda(), rule)
    assert torch.isfinite(dx).all()
    ref = oracle.score_gate_bwd(_f64(x), idx, _f64(dw), **want)
    _near(dx[finite], ref[finite], 8 * u * (np.abs(_f64(dw)) * 1.5).sum(1)[finite, None], "dlogits")
    assert (dx[0] == 0).all() and (dx[1] == 0).all()


def test_gate_chooses_as_64_bits_do(smoe):
    """Ranks that fp32 cannot tell apart: scores under a bias of 4096, where fp32 has steps of 2^-11."""
    T, E, k = 200, 128, 6
    x = _normal((T, E), 7, torch.float32, 0.02)
    b = torch.full((E,), 4096.0)
    for score in ("sigmoid", "softmax"):
        idx, w = oracle.score_gate(_f64(x), k, score, bias=_f64(b), groups=4, kept_groups=2, group_best=2)
        got, gates = smoe.score_gate(x.cuda(), k, smoe.gate_rule(score, 4, 2, 2), b.cuda())
        assert np.array_equal(got.cpu().numpy(), idx), score
        _near(gates, w, _weight_units(_f64(x)) * w)


def test_gate_gradient_of_repeated_and_foreign_experts(smoe):
    """Choices that did not come from the gate: an expert named twice gets both gradients, one that does not exist none."""
    x, dw = _normal((4, 10), 8, torch.float32), _normal((4, 3), 9, torch.float32)
    idx = torch.tensor([[2, 2, 5], [-1, 3, 10], [9, 9, 9], [2 ** 31 - 1, -2 ** 31, 0]], dtype=torch.int32)
    for score in ("softmax", "sigmoid"):
        for renormalise in (False, True):
            got = smoe.score_gate_bwd(x.cuda(), idx.cuda(), dw.cuda(), smoe.gate_rule(score, renormalise=renormalise))
            want = oracle.score_gate_bwd(_f64(x), idx.numpy(), _f64(dw), score, renormalise)
            _near(got, want, 100 * EPS32 * np.abs(_f64(dw)).sum(1, keepdims=True), f"{score} {renormalise}")


@pytest.mark.parametrize("T,E,k", [(13, 64, 8), (6, 256, 4), (5, 300, 20), (9, 7, 3)])
def test_gate_gradient_over_the_logits(smoe, T, E, k):
    """dlogits may be the logits themselves (the C entry point)."""
    import ctypes
    for score in ("softmax", "sigmoid"):
        for renormalise in (False, True):
            x, dw = _normal((T, E), 12, torch.float32).cuda(), _normal((T, k), 13, torch.float32).cuda()
            rule = smoe.gate_rule(score, renormalise=renormalise)
            idx, _ = smoe.score_gate(x, k, rule)
            want = smoe.score_gate_bwd(x, idx, dw, rule)
            rc = smoe.lib.smoe_score_gate_bwd(smoe.ctx(), torch.cuda.current_stream().cuda_stream, x.data_ptr(), idx.data_ptr(), dw.data_ptr(), T, E, k, rule._c, x.data_ptr())
            assert rc == 0 and torch.equal(x, want)


# --------------------------------------------------------------------------------------------------------------- norm
# fp32 on the way: the sum of squares in a thread's up to 32 terms, 6 lane steps and up to 16 wavefronts (54 additions at most, half of which reach rstd, the sums
# being of one sign), root, division and the products: 40 units.
NORM_UNITS = 40 * EPS32
NORMS = [(1, 1), (3, 7), (2, 128), (5, 512), (4, 520), (3, 999), (2, 1024), (7, 2048), (3, 4096), (2, 4100), (2, 8192), (1, 16384), (1, 32768), (2, 5001), (2, 10001), (1, 32767), (3, 20000), (70, 40), (600, 264), (1030, 8)]


@pytest.mark.parametrize("rows,d", NORMS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("residual", [False, True])
def test_norm_and_its_gradient(smoe, rows, d, dtype, residual):
    _log(f"norm {(rows, d)} {dtype} {residual}")
    X, R = _normal((rows, d), 1, dtype), _normal((rows, d), 2, dtype, 3.0) if residual else None
    w, eps = (1 + 0.3 * _normal((d,), 3, torch.float32)).to(dtype), 1e-5
    n = smoe.add_norm_fwd(X.cuda(), w.cuda(), None if R is None else R.cuda(), eps=eps, packed=True)
    s, y, rstd = oracle.add_norm(_f64(X), None if R is None else _f64(R), _f64(w), eps)
    half = HALF[dtype]
    added = EPS32 * np.abs(s) if residual else 0.0
    if residual:
        _near(n.S, s, half * np.abs(s) + added * (1 + half), "S")
    y_tol = NORM_UNITS * np.abs(y) + 2 * EPS32 * np.abs(y)
    _near(n.Y, y, half * np.abs(y) + (1 + half) * y_tol, "Y")
    _near(n.rstd, rstd, NORM_UNITS * rstd, "rstd")
    _near_packed(smoe, n.Y8, y, y_tol)
    dY, dS = _normal((rows, d), 4, dtype), _normal((rows, d), 5, dtype) if residual else None
    dX, dw = smoe.add_norm_bwd(dY.cuda(), n.S, w.cuda(), n.rstd, dS=None if dS is None else dS.cuda())
    S, r = _f64(n.S), _f64(n.rstd)
    dx, dweight = oracle.add_norm_bwd(_f64(dY), None if dS is None else _f64(dS), S, _f64(w), r)
    u = np.abs(S * r[:, None])
    g = np.abs(_f64(dY) * _f64(w))
    terms = r[:, None] * (g + u * (g * u).mean(-1, keepdims=True)) + (0 if dS is None else np.abs(_f64(dS)))
    _near(dX, dx, half * np.abs(dx) + 80 * EPS32 * terms, "dX")
    # sums over the rows: at most rows / 512 + 1 in a thread, 512 parts in 16 shares of 32 and 16
    units = (rows / 512 + 2 + 32 + 16 + 4) * EPS32
    _near(dw, dweight, half * np.abs(dweight) + units * (np.abs(_f64(dY)) * u).sum(0), "dweight")


def _near_packed(smoe, rows, y, tol):
    """Packed rows are within half a step of y, by the power of two that y's largest asks for (either, next to a border)."""
    codes, exps = rows.values.cpu().numpy(), rows.exps.cpu().numpy()
    d = y.shape[-1]
    P = codes.shape[-1]
    assert P == -(-d // 128) * 128
    assert (codes[:, d:] == 0).all()
    full = np.zeros((y.shape[0], P))
    full[:, :d] = np.abs(y)
    slack = np.zeros_like(full)
    slack[:, :d] = tol
    top = full.reshape(-1, P // 32, 32).max(-1)
    wide = slack.reshape(-1, P // 32, 32).max(-1)
    e = exps.astype(np.float64) - 127
    assert ((top - wide) <= 448 * 2.0 ** e).all()
    assert ((top + wide >= 224 * 2.0 ** e) | (exps == 1)).all()
    got = oracle.unpack8(codes, exps, d)
    half = np.maximum(np.abs(y) * 2.0 ** -4, np.repeat(2.0 ** e, 32, -1)[:, :d] * 2.0 ** -10)
    over = np.abs(got - y) - (half * 1.01 + 2 * tol)
    assert (over <= 0).all(), over.max()


def test_norm_in_place_of_its_inputs(smoe):
    for rows, d, dtype in ((5, 9000, torch.float32), (5, 264, torch.bfloat16), (3, 4096, torch.float32), (4, 77, torch.bfloat16), (2, 20000, torch.bfloat16)):
        X, R, w = _normal((rows, d), 1, dtype).cuda(), _normal((rows, d), 2, dtype).cuda(), _normal((d,), 3, dtype).cuda()
        dY, dS = _normal((rows, d), 4, dtype).cuda(), _normal((rows, d), 5, dtype).cuda()
        want = smoe.add_norm_fwd(X, w, R)
        dX, dw = smoe.add_norm_bwd(dY, want.S, w, want.rstd, dS=dS)
        x, r = X.clone(), R.clone()
        got = smoe.add_norm_fwd(x, w, r, out=smoe.Norm(r, x, None, torch.empty_like(want.rstd)))
        assert got.S is r and got.Y is x and torch.equal(r, want.S) and torch.equal(x, want.Y)
        for where in ("dY", "S", "dS"):
            t = dict(dY=dY.clone(), S=want.S.clone(), dS=dS.clone())
            a, b = smoe.add_norm_bwd(t["dY"], t["S"], w, want.rstd, dS=t["dS"], out=(t[where], torch.empty_like(w)))
            assert torch.equal(a, dX) and torch.equal(b, dw), where


def test_norm_of_zero_huge_and_bad_rows(smoe):
    d = 300
    x = _normal((6, d), 1, torch.float32)
    x[0] = 0
    x[1] *= 1e30                                   # squares past fp32
    x[2] *= 3e37
    x[3, 5] = float("nan")
    x[4, 7] = float("inf")
    w = torch.ones(d)
    for dtype in (torch.float32, torch.bfloat16):
        n = smoe.add_norm_fwd(x.to(dtype).cuda(), w.to(dtype).cuda(), eps=1e-6, packed=True)
        y = _f64(n.Y)
        s, want, _ = oracle.add_norm(_f64(x.to(dtype))[[0, 1, 2, 5]], None, np.ones(d), 1e-6)
        assert np.abs(y[[0, 1, 2, 5]] - want).max() <= (NORM_UNITS + HALF[dtype]) * np.abs(want).max()
        assert np.isnan(y[3]).all() and np.isnan(y[4, 7]) and (np.delete(y[4], 7) == 0).all()
        back = _f64(smoe.rows8_unpack(n.Y8))
        assert np.isnan(back[3]).all() and (back[0] == 0).all() and np.isfinite(back[[1, 2, 5]]).all()


def test_norm_of_no_rows(smoe):
    w = _normal((64,), 1).cuda()
    none = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    n = smoe.add_norm_fwd(none, w, none, packed=True)
    assert n.Y.shape == (0, 64) and n.Y8.rows == 0
    dX, dw = smoe.add_norm_bwd(none, none, w, n.rstd)
    assert dX.shape == (0, 64) and (dw == 0).all()


# ------------------------------------------------------------------------------------------------------ rows in 8 bits
def _specials(d, seed):
    x = torch.randn(12, d, generator=_gen(seed), dtype=torch.float32) * torch.exp(4 * torch.randn(12, d, generator=_gen(seed + 1)))
    x[0], x[1, 0] = 0, float("inf")
    x[2, d // 2] = float("nan")
    x[3] *= 2.0 ** -140
    x[4] = -0.0
    x[5] = torch.sign(x[5]) * 1.96 * 2.0 ** 127
    x[6] = x[6].abs().clamp(max=1) * 3.0e38
    x[7, 0] = 448.0
    x[8, 0], x[8, 1:] = 448.0, 0.0009765625 * torch.arange(d - 1)      # steps and ties of the smallest values
    x[9] = float("nan")
    x[10] = float("-inf")
    return x


@pytest.mark.parametrize("d", [1, 5, 32, 64, 100, 128, 999, 2048])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_pack_and_unpack_bit_for_bit(smoe, d, dtype):
    _log(f"rows8 {d} {dtype}")
    x = (_specials(d, d) if d >= 5 else _normal((12, d), d, torch.float32)).to(dtype)
    rows = smoe.rows8_pack(x.cuda())
    codes, exps = oracle.pack8(_f64(x))
    got = rows.values.cpu().numpy()
    bad = np.isnan(oracle.e4m3_values()[codes])
    assert np.array_equal(rows.exps.cpu().numpy(), exps)
    assert np.array_equal(got[~bad], codes[~bad]) and ((got[bad] & 0x7F) == 0x7F).all()
    values = oracle.unpack8(codes, exps, d)
    back = smoe.rows8_unpack(rows, torch.float32).cpu().numpy()
    assert np.array_equal(back, values.astype(np.float32), equal_nan=True)
    assert np.array_equal(smoe.rows8_unpack(rows).float().cpu().numpy(), torch.from_numpy(values).to(torch.bfloat16).float().numpy(), equal_nan=True)


def _weights(shape, seed, dtype=torch.bfloat16):
    return _normal(shape, seed, dtype, shape[1] ** -0.5)


def _stored(smoe, W, halves=1):
    """The values that packed weights stand for, [E, d_in, d_out], by the oracle."""
    W = _f64(W)
    out = np.empty_like(W)
    for e in range(W.shape[0]):
        out[e] = oracle.unpack8(*oracle.pack8(W[e].T), W.shape[1]).T
    return out


@pytest.mark.parametrize("E,d_in,d_out,halves", [(1, 32, 16, 1), (2, 128, 64, 1), (3, 100, 40, 1), (2, 200, 72, 2), (1, 257, 30, 2), (2, 128, 128, 2), (1, 1, 1, 1)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_weights_as_laid_out(smoe, E, d_in, d_out, halves, dtype):
    W = _weights((E, d_in, d_out), 11, dtype)
    w = smoe.weights8(W.cuda(), halves=halves)
    half = d_out // halves
    groups, steps = halves * 2 * -(-half // 32), -(-d_in // 128)
    codes = w.values.cpu().numpy().reshape(E, groups, steps, 8, 16, 16)          # [.., sixteenth of the step, column, element]
    exps = w.exps.cpu().numpy().reshape(E, groups, steps, 16, 4)
    codes = codes.transpose(0, 1, 4, 2, 3, 5).reshape(E, groups * 16, steps * 128)
    exps = exps.transpose(0, 1, 3, 2, 4).reshape(E, groups * 16, steps * 4)
    per = groups * 16 // halves
    for e in range(E):
        for h in range(halves):
            want = np.zeros((per, d_in))
            want[:half] = _f64(W)[e].T[h * half:(h + 1) * half]
            c, x = oracle.pack8(want)
            assert np.array_equal(codes[e, h * per:(h + 1) * per], c) and np.array_equal(exps[e, h * per:(h + 1) * per], x)


# ----------------------------------------------------------------------------------------------------------- products
def _slack(x, W):
    """Bound of a product's error before it is rounded, by column: an instruction's is under 2^-11 of its largest term (64 terms or more), and the fp32 sums'."""
    out = np.zeros(W.shape[1])
    for k in range(0, W.shape[0], 64):
        out += 2.0 ** -11 * np.abs(x[k:k + 64]).max() * np.abs(W[k:k + 64]).max(0)
    return out + (W.shape[0] / 64 + 4) * EPS32 * (np.abs(x) @ np.abs(W))


def _routed(smoe, T, E, k, seed, skew=0.0, only=None):
    logits = torch.randn(T, E, generator=_gen(seed))
    if skew:
        logits = logits - skew * torch.log(torch.arange(1, E + 1, dtype=torch.float32))
    if only is not None:
        logits[:, [e for e in range(E) if e not in only]] = -float("inf")
    idx, gates = oracle.score_gate(_f64(logits), k)
    ei = torch.from_numpy(idx).cuda()
    return idx, gates.astype(np.float32), smoe.route(ei, E)


LINEARS = [  # T, d_in, d_out, E, k
    (1, 32, 8, 1, 1), (5, 128, 64, 4, 2), (33, 100, 72, 3, 2), (64, 256, 128, 8, 4), (3, 999, 24, 2, 1), (70, 384, 200, 2, 1), (17, 130, 1000, 5, 3),
]


@pytest.mark.parametrize("T,d_in,d_out,E,k", LINEARS)
@pytest.mark.parametrize("form", ["slots", "sum", "grouped out", "grouped in"])
def test_linear_in_8_bits(smoe, T, d_in, d_out, E, k, form):
    _log(f"plinear8 {(T, d_in, d_out, E, k)} {form}")
    idx, gates, r = _routed(smoe, T, E, k, 21)
    X, W = _normal((T, d_in), 22) * torch.exp(_normal((d_in,), 23)), _weights((E, d_in, d_out), 24)
    x = oracle.unpack8(*oracle.pack8(_f64(X)), d_in)
    w = _stored(smoe, W)
    want = oracle.plinear8(x, w, idx)
    tol = np.stack([_slack(x[t], w[idx[t, j]]) for t in range(T) for j in range(k)])
    order = r.sorted_scattered_idxs.cpu().numpy()
    rows, packed = smoe.rows8_pack(X.cuda()), smoe.weights8(W.cuda())
    half = HALF[torch.bfloat16]
    if form == "slots":
        Y, Yhat = smoe.plinear8_fwd(rows, packed, r, k)
        assert Y is Yhat
    elif form == "grouped out":
        Y, _ = smoe.plinear8_fwd(rows, packed, r, k, grouped_out=True)
        want, tol = want[order], tol[order]
    elif form == "grouped in":
        rows = smoe.rows8_pack(X[order // k].cuda())
        Y, _ = smoe.plinear8_fwd(rows, packed, r, 1, grouped_in=True)
    else:
        Y, Yhat = smoe.plinear8_fwd(rows, packed, r, k, torch.from_numpy(gates).cuda())
        _near(Yhat, want, half * np.abs(want) + (1 + half) * tol, "Yhat")
        g = gates.astype(np.float64)
        slots = (half * np.abs(want) + (1 + half) * tol).reshape(T, k, -1)
        want, tol = oracle.plinear8(x, w, idx, g), (slots * g[..., None]).sum(1) + (k + 1) * EPS32 * (np.abs(want).reshape(T, k, -1) * g[..., None]).sum(1)
    _near(Y, want, half * np.abs(want) + (1 + half) * tol, form)


# enough columns that wavefronts stand side by side (256, 1280), and the contractions at which they share it all the same (1024, 2048), but for more rows
@pytest.mark.parametrize("T,d_in", [(20, 256), (20, 1280), (20, 1024), (20, 2048), (300, 1024), (7, 2050)])
def test_wide_weights_of_few_rows(smoe, T, d_in):
    E, k, d_out = 16, 2, 16392
    _log(f"plinear8 wide {(T, d_in)}")
    idx, _, r = _routed(smoe, T, E, k, 71)
    X = _normal((T, d_in), 72)
    W = torch.randn(E, d_in, d_out, generator=torch.Generator("cuda").manual_seed(73), device="cuda").mul_(0.05).bfloat16()
    smoe.set_kernel_mode(1)
    try:
        Y = smoe.plinear8_fwd(smoe.rows8_pack(X.cuda()), smoe.weights8(W), r, k)[0]
    finally:
        smoe.set_kernel_mode(0)
    columns = torch.cat([torch.arange(0, d_out, 797), torch.tensor([d_out - 1])])
    kept = _f64(W[:, :, columns.cuda()])
    w = [oracle.unpack8(*oracle.pack8(kept[e].T), d_in).T for e in range(E)]
    x = oracle.unpack8(*oracle.pack8(_f64(X)), d_in)
    slots = range(0, T * k, max(1, T * k // 40))
    want = np.stack([x[s // k] @ w[idx[s // k, s % k]] for s in slots])
    tol = np.stack([_slack(x[s // k], w[idx[s // k, s % k]]) for s in slots])
    half = HALF[torch.bfloat16]
    _near(Y[list(slots)][:, columns.cuda()], want, half * np.abs(want) + (1 + half) * tol, "wide")


MLPS = [  # T, d_model, d_expert, E, k, act
    (1, 32, 32, 1, 1, "swiglu"), (4, 256, 64, 8, 2, "swiglu"), (9, 128, 100, 4, 2, "gelu"), (40, 200, 72, 2, 2, "swiglu"), (20, 256, 160, 16, 4, "gelu"), (130, 136, 40, 3, 1, "swiglu"),
    (3, 1000, 33, 2, 2, "swiglu"), (6, 128, 257, 3, 2, "gelu"),
]


def _mlp_case(smoe, T, d_model, d_expert, E, k, act, seed=31, **routing):
    idx, gates, r = _routed(smoe, T, E, k, seed, **routing)
    code = smoe.ACT_SWIGLU if act == "swiglu" else smoe.ACT_GELU
    X = _normal((T, d_model), seed + 1) * torch.exp(0.7 * _normal((d_model,), seed + 2))
    W1, W2 = _weights((E, d_model, smoe.hidden_width(code, d_expert)), seed + 3), _weights((E, d_expert, d_model), seed + 4)
    packed = smoe.weights8(W1.cuda(), halves=2 if act == "swiglu" else 1), smoe.weights8(W2.cuda())
    return idx, gates, r, code, X, W1, W2, packed


@pytest.mark.parametrize("T,d_model,d_expert,E,k,act", MLPS)
def test_mlp_in_8_bits(smoe, T, d_model, d_expert, E, k, act):
    _log(f"mlp8 {(T, d_model, d_expert, E, k, act)}")
    idx, gates, r, code, X, W1, W2, packed = _mlp_case(smoe, T, d_model, d_expert, E, k, act)
    Y = smoe.mlp8_fwd(smoe.rows8_pack(X.cuda()), *packed, r, k, torch.from_numpy(gates).cuda(), code)
    x = oracle.unpack8(*oracle.pack8(_f64(X)), d_model)
    want, tol = oracle.mlp8(x, _stored(smoe, W1), _stored(smoe, W2), idx, gates.astype(np.float64), code, slack=_slack, rounding=ROW)
    half = HALF[torch.bfloat16]
    _near(Y, want, half * np.abs(want) + (1 + half) * tol + k * EPS32 * np.abs(want).max(), "Y")


def test_mlp_with_empty_and_crowded_experts(smoe):
    for only in ([3], [0, 7], [5, 6, 2]):
        T, k = 70, min(2, len(only))
        idx, gates, r, code, X, W1, W2, packed = _mlp_case(smoe, T, 128, 64, 8, k, "swiglu", only=only)
        assert set(idx.ravel()) <= set(only)
        Y = smoe.mlp8_fwd(smoe.rows8_pack(X.cuda()), *packed, r, k, torch.from_numpy(gates).cuda(), code)
        x = oracle.unpack8(*oracle.pack8(_f64(X)), 128)
        want, tol = oracle.mlp8(x, _stored(smoe, W1), _stored(smoe, W2), idx, gates.astype(np.float64), code, slack=_slack, rounding=ROW)
        _near(Y, want, 2.0 ** -8 * np.abs(want) + 1.01 * tol + 1e-6 * np.abs(want).max(), str(only))


def test_a_bad_row_stays_by_itself(smoe):
    """NaN in one token's row: its output is NaN, the others' are what they were."""
    T, k = 37, 2
    idx, gates, r, code, X, W1, W2, packed = _mlp_case(smoe, T, 160, 96, 4, k, "swiglu")
    g = torch.from_numpy(gates).cuda()
    clean = smoe.mlp8_fwd(smoe.rows8_pack(X.cuda()), *packed, r, k, g, code)
    bad = X.clone()
    bad[11, 150] = float("nan")
    bad[20, 0] = float("inf")
    Y = smoe.mlp8_fwd(smoe.rows8_pack(bad.cuda()), *packed, r, k, g, code)
    others = [t for t in range(T) if t not in (11, 20)]
    assert torch.isnan(Y[[11, 20]]).all() and torch.equal(Y[others], clean[others])


def test_no_tokens(smoe):
    r = smoe.route(torch.empty(0, 2, dtype=torch.int32, device="cuda"), 4)
    W1, W2 = smoe.weights8(_weights((4, 64, 64), 1).cuda(), halves=2), smoe.weights8(_weights((4, 32, 64), 2).cuda())
    none = smoe.rows8_pack(torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"))
    g = torch.empty(0, 2, dtype=torch.float32, device="cuda")
    assert smoe.mlp8_fwd(none, W1, W2, r, 2, g, smoe.ACT_SWIGLU).shape == (0, 64)
    assert smoe.plinear8_fwd(none, smoe.weights8(_weights((4, 64, 8), 1).cuda()), r, 2, g)[0].shape == (0, 8)
    idx, gates = smoe.score_gate(torch.empty(0, 4, device="cuda"), 2, smoe.gate_rule())
    assert idx.shape == (0, 2) and smoe.score_gate_bwd(torch.empty(0, 4, device="cuda"), idx, gates, smoe.gate_rule()).shape == (0, 4)


# ------------------------------------------------------------------------------------------------------ a block of them
def _block(smoe, s):
    """Norm -> router -> experts -> back into the stream, of a serving step."""
    n = smoe.add_norm_fwd(s["X"], s["weight"], s["R"], packed=True)
    logits = n.Y.float() @ s["router"]
    idx, gates = smoe.score_gate(logits, 3, s["rule"], s["bias"])
    r = smoe.route(idx, 16)
    Y = smoe.mlp8_fwd(n.Y8, s["W1"], s["W2"], r, 3, gates, smoe.ACT_SWIGLU)
    m = smoe.add_norm_fwd(Y, s["weight"], n.S)
    return n, logits, idx, gates, Y, m


def _block_state(smoe, T, seed):
    d, de, E = 256, 96, 16
    s = {"X": _normal((T, d), seed).cuda(), "R": _normal((T, d), seed + 1, std=2.0).cuda(), "weight": (1 + 0.1 * _normal((d,), 3)).cuda(),
         "router": _normal((d, E), 4, torch.float32, d ** -0.5).cuda(), "bias": _normal((E,), 5, torch.float32, 0.1).cuda(),
         "rule": smoe.gate_rule("sigmoid", 4, 2, 2, True, 2.0)}
    s["w"] = _weights((E, d, 2 * de), 6), _weights((E, de, d), 7)
    s["W1"], s["W2"] = smoe.weights8(s["w"][0].cuda(), halves=2), smoe.weights8(s["w"][1].cuda())
    return s


@pytest.mark.parametrize("T", [1, 5, 100])
def test_a_block_as_it_is_served(smoe, T):
    """Each step against the oracle, on what the step before left."""
    _log(f"block {T}")
    s = _block_state(smoe, T, 50)
    n, logits, idx, gates, Y, m = _block(smoe, s)
    want, w = oracle.score_gate(_f64(logits), 3, "sigmoid", bias=_f64(s["bias"]), groups=4, kept_groups=2, group_best=2, scale=2.0)
    assert np.array_equal(idx.cpu().numpy(), want)
    _near(gates, w, _weight_units(_f64(logits)) * w, "gates")
    x = oracle.unpack8(n.Y8.values.cpu().numpy(), n.Y8.exps.cpu().numpy(), 256)
    _, y, _ = oracle.add_norm(_f64(s["X"]), _f64(s["R"]), _f64(s["weight"]), 1e-6)
    _near_packed(smoe, n.Y8, y, (NORM_UNITS + 3 * EPS32) * np.abs(y))
    want, tol = oracle.mlp8(x, _stored(smoe, s["w"][0]), _stored(smoe, s["w"][1]), idx.cpu().numpy(), _f64(gates), 2, slack=_slack, rounding=ROW)
    _near(Y, want, 2.0 ** -8 * np.abs(want) + 1.01 * tol + 1e-6 * np.abs(want).max(), "Y")
    stream, y, _ = oracle.add_norm(_f64(Y), _f64(n.S), _f64(s["weight"]), 1e-6)
    _near(m.S, stream, 2.0 ** -8 * np.abs(stream) * 1.01 + EPS32 * np.abs(stream))
    _near(m.Y, y, 2.0 ** -8 * np.abs(y) * 1.01 + 2 * NORM_UNITS * np.abs(y))


@pytest.mark.parametrize("T", [24, 1500])
def test_a_block_replays_from_a_graph_on_another_stream(smoe, T):
    state, others = _block_state(smoe, T, 60), [_block_state(smoe, T, 60 + 10 * i) for i in range(3)]
    names = ("X", "R")

    def step():
        n, logits, idx, gates, Y, m = _block(smoe, state)
        dX, dw = smoe.add_norm_bwd(m.Y, n.S, state["weight"], n.rstd, dS=m.S)
        dl = smoe.score_gate_bwd(logits, idx, gates, state["rule"])
        return n.S, n.Y, n.Y8.values, n.Y8.exps, logits, idx, gates, Y, m.S, m.Y, dX, dw, dl

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        captured = step()
    for other in others + others[:1]:
        for n in names:
            state[n].copy_(other[n])
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in captured]
        for a, b in zip(got, step()):
            assert torch.equal(a, b)


def test_rows_past_32_bits(smoe):
    """More elements than 2^31: the last rows are those of a call of their own."""
    rows, d = 2 ** 19 + 37, 4104
    X = torch.zeros(rows, d, dtype=torch.bfloat16, device="cuda")
    last = _normal((50, d), 1).cuda()
    X[-50:] = last
    w = _normal((d,), 2).cuda()
    n, few = smoe.add_norm_fwd(X, w, X, packed=True), smoe.add_norm_fwd(last, w, last, packed=True)
    for a, b in ((n.S, few.S), (n.Y, few.Y), (n.rstd, few.rstd), (n.Y8.values, few.Y8.values), (n.Y8.exps, few.Y8.exps)):
        assert torch.equal(a[-50:], b)
    packed = smoe.rows8_pack(X)
    assert torch.equal(packed.values[-50:], smoe.rows8_pack(last).values)
    assert torch.equal(smoe.rows8_unpack(packed)[-50:], smoe.rows8_unpack(smoe.rows8_pack(last)))
    dX, dw = smoe.add_norm_bwd(X, n.S, w, n.rstd, out=(X, torch.empty_like(w)))
    want, dweight = smoe.add_norm_bwd(last, few.S, w, few.rstd)
    assert torch.equal(dX[-50:], want) and torch.equal(dX[:3], torch.zeros_like(dX[:3]))
    tol = 64 * EPS32 * (last.double().abs() * (few.S.double() * few.rstd[:, None].double()).abs()).sum(0)      # another order of the sums, and a rounding
    assert ((dw.double() - dweight.double()).abs() <= 2 * HALF[torch.bfloat16] * dweight.double().abs() + tol).all()


def test_more_rows_than_a_launch_has(smoe):
    rows = 2 ** 21 + 101
    X, w = torch.randn(rows, 8, device="cuda"), torch.ones(8, device="cuda")
    n, last = smoe.add_norm_fwd(X, w, X, packed=True), smoe.add_norm_fwd(X[-128:].contiguous(), w, X[-128:].contiguous(), packed=True)
    for a, b in ((n.S, last.S), (n.Y, last.Y), (n.rstd, last.rstd), (n.Y8.values, last.Y8.values), (n.Y8.exps, last.Y8.exps)):
        assert torch.equal(a[-128:], b)
    assert torch.equal(n.S, X + X)
    packed = smoe.rows8_pack(X)
    assert torch.equal(packed.values[-128:], smoe.rows8_pack(X[-128:].contiguous()).values)


def test_identical_calls_give_identical_bits(smoe):
    a, b = (_block(smoe, _block_state(smoe, 65, 80)) for _ in range(2))
    for x, y in ((a[0].Y, b[0].Y), (a[3], b[3]), (a[4], b[4]), (a[5].Y, b[5].Y)):
        assert torch.equal(x, y)
    X, w = _normal((3000, 264), 1).cuda(), _normal((264,), 2).cuda()
    n = smoe.add_norm_fwd(X, w)
    one, two = (smoe.add_norm_bwd(X, X, w, n.rstd) for _ in range(2))
    assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])
