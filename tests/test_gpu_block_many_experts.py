"""The products in 8 bits with as many experts as the kernels for many rows number (256), and with more, which the kernels for few rows take at every size."""
import numpy as np
import pytest
import torch

import oracle
from test_gpu_block import HALF, ROW, _f64, _log, _mlp_case, _near, _normal, _routed, _slack, _stored, _weights

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def smoe():
    import paper_2403_08245_amd as m
    yield m
    m.set_kernel_mode(0)


@pytest.mark.parametrize("mode", [0, 1, 3, 4])
@pytest.mark.parametrize("T,E,k", [(40, 256, 4), (40, 257, 4), (900, 257, 3), (3000, 300, 8), (5, 1000, 8)])
def test_linear(smoe, mode, T, E, k):
    d_in, d_out = 160, 72
    _log(f"plinear8 of many experts {mode} {(T, E, k)}")
    idx, gates, r = _routed(smoe, T, E, k, 141, skew=0.5)
    X, W = _normal((T, d_in), 142), _weights((E, d_in, d_out), 143)
    smoe.set_kernel_mode(mode)
    Y, Yhat = smoe.plinear8_fwd(smoe.rows8_pack(X.cuda()), smoe.weights8(W.cuda()), r, k, torch.from_numpy(gates).cuda())
    x, w = oracle.unpack8(*oracle.pack8(_f64(X)), d_in), _stored(smoe, W)
    sample = np.unique(np.concatenate([np.arange(0, T * k, max(1, T * k // 300)), [T * k - 1]]))
    want = np.stack([x[s // k] @ w[idx[s // k, s % k]] for s in sample])
    tol = np.stack([_slack(x[s // k], w[idx[s // k, s % k]]) for s in sample])
    half = HALF[torch.bfloat16]
    _near(Yhat[torch.from_numpy(sample).cuda()], want, half * np.abs(want) + (1 + half) * tol, "Yhat")
    t = np.arange(0, T, max(1, T // 50))
    rows = np.stack([np.stack([x[i] @ w[idx[i, j]] for j in range(k)]) for i in t])
    off = np.stack([np.stack([_slack(x[i], w[idx[i, j]]) for j in range(k)]) for i in t])
    g = gates[t].astype(np.float64)[..., None]
    want = (rows * g).sum(1)
    tol = ((half * np.abs(rows) + (1 + half) * off) * g).sum(1) + (k + 1) * 2.0 ** -24 * (np.abs(rows) * g).sum(1)
    _near(Y[torch.from_numpy(t).cuda()], want, half * np.abs(want) + (1 + half) * tol, "Y")


@pytest.mark.parametrize("mode", [0, 3, 4])
@pytest.mark.parametrize("T,E,k,act", [(30, 256, 2, "swiglu"), (30, 257, 2, "swiglu"), (1500, 300, 6, "swiglu"), (700, 260, 2, "gelu")])
def test_mlp(smoe, mode, T, E, k, act):
    d_model, d_expert = 136, 100
    _log(f"mlp8 of many experts {mode} {(T, E, k, act)}")
    idx, gates, r, code, X, W1, W2, packed = _mlp_case(smoe, T, d_model, d_expert, E, k, act, seed=151, skew=0.5)
    smoe.set_kernel_mode(mode)
    Y = smoe.mlp8_fwd(smoe.rows8_pack(X.cuda()), *packed, r, k, torch.from_numpy(gates).cuda(), code)
    t = np.arange(0, T, max(1, T // 60))
    x = oracle.unpack8(*oracle.pack8(_f64(X)), d_model)
    want, tol = oracle.mlp8(x[t], _stored(smoe, W1), _stored(smoe, W2), idx[t], gates[t].astype(np.float64), code, slack=_slack, rounding=ROW)
    half = HALF[torch.bfloat16]
    got = Y[torch.from_numpy(t).cuda()]
    _near(got, want, half * np.abs(want) + (1 + half) * tol + k * 2.0 ** -24 * np.abs(want).max(), "Y")
    assert np.sqrt(np.mean((_f64(got) - want) ** 2) / np.mean(want ** 2)) <= 4e-3      # test_gpu_block_precision.py derives it
