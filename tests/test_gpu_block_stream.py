"""The products in 8 bits on the kernels for many rows: tiles of both shapes, ragged segments, several rounds of tiles, odd and even numbers of stages; against
the oracle on sampled rows, and on all rows against the kernels for few rows."""
import numpy as np
import pytest
import torch

import oracle
from test_gpu_block import HALF, ROW, _f64, _log, _mlp_case, _near, _normal, _routed, _slack, _stored, _weights

pytestmark = pytest.mark.gpu
FEW = 1            # smoe_set_kernel_mode: the kernels for few rows, whatever the size


@pytest.fixture(scope="module")
def smoe():
    import paper_2403_08245_amd as m
    return m


@pytest.fixture(params=[3, 4], ids=["128 x 256", "256 x 256"])
def shape(request, smoe):
    smoe.set_kernel_mode(request.param)
    yield request.param
    smoe.set_kernel_mode(0)


def _few(smoe, call, mode):
    smoe.set_kernel_mode(FEW)
    try:
        return call()
    finally:
        smoe.set_kernel_mode(mode)


LINEARS = [  # T, d_in, d_out, E, k: even, odd, many and few stages; one column tile and several; more tiles than compute units
    (150, 256, 136, 2, 2), (300, 384, 520, 3, 1), (90, 2048, 72, 1, 2), (5, 640, 8, 4, 2), (700, 500, 264, 5, 3), (5000, 256, 2056, 3, 2), (4000, 384, 1032, 40, 4), (2600, 130, 768, 200, 5), (400, 128, 264, 3, 2), (333, 40, 1000, 2, 1), (3000, 100, 1536, 30, 4),
]


@pytest.mark.parametrize("T,d_in,d_out,E,k", LINEARS)
@pytest.mark.parametrize("form", ["slots", "grouped out", "grouped in"])
def test_linear(smoe, shape, T, d_in, d_out, E, k, form):
    _log(f"plinear8 stream {shape} {(T, d_in, d_out, E, k)} {form}")
    idx, gates, r = _routed(smoe, T, E, k, 41, skew=0.7)
    X, W = _normal((T, d_in), 42) * torch.exp(_normal((d_in,), 43)), _weights((E, d_in, d_out), 44)
    order = r.sorted_scattered_idxs.cpu().numpy()
    packed = smoe.weights8(W.cuda())
    rows = smoe.rows8_pack((X[order // k] if form == "grouped in" else X).cuda())
    call = lambda: smoe.plinear8_fwd(rows, packed, r, 1 if form == "grouped in" else k, grouped_in=form == "grouped in", grouped_out=form == "grouped out")[0]
    Y = call()
    small = _few(smoe, call, shape)
    x = oracle.unpack8(*oracle.pack8(_f64(X)), d_in)
    w = _stored(smoe, W)
    sample = np.unique(np.concatenate([np.arange(0, T * k, max(1, T * k // 150)), [T * k - 1], order[[0, -1]]]))
    want = np.stack([x[s // k] @ w[idx[s // k, s % k]] for s in sample])
    tol = np.stack([_slack(x[s // k], w[idx[s // k, s % k]]) for s in sample])
    at = np.argsort(order)[sample] if form == "grouped out" else sample
    half = HALF[torch.bfloat16]
    _near(Y[torch.from_numpy(at).cuda()], want, half * np.abs(want) + (1 + half) * tol, form)
    # all rows: each of the two within its bound of the same number
    a, b = Y.float(), small.float()
    big = tol.max() * 4                               # of rows that were not sampled, with larger entries
    assert ((a - b).abs() <= 2 * half * torch.maximum(a.abs(), b.abs()) + 2 * big).all()
    assert torch.equal(Y, call())


MLPS = [  # T, d_model, d_expert, E, k, act
    (300, 256, 264, 4, 2, "swiglu"), (257, 304, 200, 2, 2, "gelu"), (520, 384, 1000, 3, 2, "swiglu"), (130, 256, 130, 1, 1, "gelu"), (1500, 512, 224, 64, 8, "swiglu"), (2000, 264, 161, 6, 3, "swiglu"),
    (900, 640, 320, 5, 2, "gelu"), (700, 120, 128, 4, 2, "swiglu"), (500, 384, 60, 6, 2, "gelu"),
]


@pytest.mark.parametrize("T,d_model,d_expert,E,k,act", MLPS)
def test_mlp(smoe, shape, T, d_model, d_expert, E, k, act):
    _log(f"mlp8 stream {shape} {(T, d_model, d_expert, E, k, act)}")
    idx, gates, r, code, X, W1, W2, packed = _mlp_case(smoe, T, d_model, d_expert, E, k, act, seed=51, skew=0.7)
    rows, g = smoe.rows8_pack(X.cuda()), torch.from_numpy(gates).cuda()
    call = lambda: smoe.mlp8_fwd(rows, *packed, r, k, g, code)
    Y = call()
    small = _few(smoe, call, shape)
    x = oracle.unpack8(*oracle.pack8(_f64(X)), d_model)
    sample = np.unique(np.concatenate([np.arange(0, T, max(1, T // 40)), [T - 1]]))
    want, tol = oracle.mlp8(x[sample], _stored(smoe, W1), _stored(smoe, W2), idx[sample], gates[sample].astype(np.float64), code, slack=_slack, rounding=ROW)
    half = HALF[torch.bfloat16]
    _near(Y[torch.from_numpy(sample).cuda()], want, half * np.abs(want) + (1 + half) * tol + k * 2.0 ** -24 * np.abs(want).max(), "Y")
    a, b = Y.float(), small.float()
    assert ((a - b).abs() <= 2 * half * torch.maximum(a.abs(), b.abs()) + 2 * 4 * tol.max()).all()
    assert torch.equal(Y, call())


def test_a_bad_row_stays_by_itself(smoe, shape):
    T, k = 400, 2
    idx, gates, r, code, X, W1, W2, packed = _mlp_case(smoe, T, 264, 96, 4, k, "swiglu", seed=61)
    g = torch.from_numpy(gates).cuda()
    clean = smoe.mlp8_fwd(smoe.rows8_pack(X.cuda()), *packed, r, k, g, code)
    bad = X.clone()
    bad[11, 250] = float("nan")
    bad[399, 0] = float("inf")
    bad[200] = 1e30                               # products past fp32 in places
    Y = smoe.mlp8_fwd(smoe.rows8_pack(bad.cuda()), *packed, r, k, g, code)
    others = [t for t in range(T) if t not in (11, 200, 399)]
    assert torch.isnan(Y[[11, 399]]).all() and torch.equal(Y[others], clean[others])


def test_few_rows_and_many_agree_where_the_rule_changes(smoe):
    """Either side of sizes where the kernels change (64 rows an expert here, as estimated)."""
    for T in (32, 64, 65, 130, 400):
        idx, gates, r, code, X, W1, W2, packed = _mlp_case(smoe, T, 256, 128, 4, 2, "swiglu", seed=71)
        rows, g = smoe.rows8_pack(X.cuda()), torch.from_numpy(gates).cuda()
        Y = smoe.mlp8_fwd(rows, *packed, r, 2, g, code)
        x = oracle.unpack8(*oracle.pack8(_f64(X)), 256)
        want, tol = oracle.mlp8(x, _stored(smoe, W1), _stored(smoe, W2), idx, gates.astype(np.float64), code, slack=_slack, rounding=ROW)
        _near(Y, want, 2.0 ** -8 * np.abs(want) + 1.01 * tol + 1e-6 * np.abs(want).max(), str(T))


@pytest.mark.parametrize("act", ["swiglu", "gelu"])
def test_rows_of_all_sizes(smoe, shape, act):
    """Rows from 2^-60 to 2^30: hidden rows and rows of the weighted sum far from 1, in one tile."""
    T, k = 300, 2
    idx, gates, r, code, X, W1, W2, packed = _mlp_case(smoe, T, 256, 320, 3, k, act, seed=81)
    X = (X.float() * 2.0 ** torch.linspace(-60, 30, T).round()[:, None]).to(torch.bfloat16)
    Y = smoe.mlp8_fwd(smoe.rows8_pack(X.cuda()), *packed, r, k, torch.from_numpy(gates).cuda(), code)
    x = oracle.unpack8(*oracle.pack8(_f64(X)), 256)
    with np.errstate(over="ignore"):
        want, tol = oracle.mlp8(x, _stored(smoe, W1), _stored(smoe, W2), idx, gates.astype(np.float64), code, slack=_slack, rounding=ROW)
    half = HALF[torch.bfloat16]
    _near(Y, want, half * np.abs(want) + (1 + half) * tol + k * 2.0 ** -24 * np.abs(want).max(1, keepdims=True) * 2, "Y")


def test_weights_past_the_caches(smoe):
    """Weights over half of the last-level cache (128 MB) are read past it by tiles that are their expert's only one: experts with one tile, with several and with none."""
    E, d, N, k = 66, 1024, 2048, 1
    logits = torch.zeros(3000, E)
    pick = torch.cat([torch.zeros(400), torch.ones(128), torch.full((129,), 2), torch.randint(3, 60, (2343,), generator=torch.Generator().manual_seed(1)).float()]).long()
    logits[torch.arange(3000), pick] = 5.0
    idx, _ = oracle.score_gate(_f64(logits), k)
    r = smoe.route(torch.from_numpy(idx).cuda(), E)
    X, W = _normal((3000, d), 2), _weights((E, d, N), 3)
    packed = smoe.weights8(W.cuda())
    assert packed.values.numel() > 128 << 20
    rows = smoe.rows8_pack(X.cuda())
    smoe.set_kernel_mode(3)
    try:
        Y = smoe.plinear8_fwd(rows, packed, r, k)[0]
    finally:
        smoe.set_kernel_mode(0)
    x = oracle.unpack8(*oracle.pack8(_f64(X)), d)
    for t in (0, 5, 399, 400, 527, 528, 656, 657, 1500, 2999):
        w = oracle.unpack8(*oracle.pack8(_f64(W[idx[t, 0]]).T), d).T
        want = x[t] @ w
        _near(Y[t], want, 2.0 ** -8 * np.abs(want) + 1.01 * _slack(x[t], w), str(t))
    few = _few(smoe, lambda: smoe.plinear8_fwd(rows, packed, r, k)[0], 0).float()
    assert ((Y.float() - few).abs() <= 2.0 ** -6 * few.abs() + 0.05).all()
