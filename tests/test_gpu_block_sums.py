"""The weighted sums of smoe_plinear8_fwd: rows in bf16, the very ones that the call without gates leaves, summed with what rounding took from them.

Root mean square against 64 bits: values of one sign and logarithm spread evenly are off by 2^-7 / sqrt(12) sqrt(0.375 / ln 2) = 1.66e-3 after one rounding to bf16 and by 2.35e-3
after two; of rows that are known to a quarter of their last place, so to half of that quarter, the second is a quarter as large: 1.71e-3, held to 1.9e-3.  Sums of more than eight
rows, or of widths that are not whole 64s, are of the rounded ones."""
import numpy as np
import pytest
import torch

import oracle
from test_gpu_block import _f64, _log, _normal, _routed, _stored, _weights

pytestmark = pytest.mark.gpu
MODES = pytest.mark.parametrize("mode", [1, 3, 4], ids=["few rows", "128 x 256", "256 x 256"])


@pytest.fixture(scope="module")
def smoe():
    import paper_2403_08245_amd as m
    yield m
    m.set_kernel_mode(0)


LINEARS = [  # T, d_in, d_out, E, k
    (1, 32, 8, 1, 1), (5, 128, 64, 4, 2), (300, 256, 136, 2, 2), (90, 2048, 72, 3, 3), (50, 640, 8, 16, 16), (700, 500, 264, 5, 5), (500, 256, 2056, 3, 1), (400, 384, 1032, 40, 8), (60, 130, 768, 40, 20),
    (30, 100, 200, 48, 40), (4000, 256, 96, 4, 2), (300, 256, 64, 2, 2), (700, 500, 320, 5, 5), (400, 384, 1024, 40, 8), (90, 2048, 192, 3, 3), (260, 100, 832, 9, 7), (900, 260, 448, 3, 1), (3000, 256, 640, 8, 4),
]


@MODES
@pytest.mark.parametrize("T,d_in,d_out,E,k", LINEARS)
def test_sums(smoe, mode, T, d_in, d_out, E, k):
    _log(f"sums {mode} {(T, d_in, d_out, E, k)}")
    idx, gates, r = _routed(smoe, T, E, k, 161, skew=0.5)
    X, W = _normal((T, d_in), 162) * torch.exp(_normal((d_in,), 163)), _weights((E, d_in, d_out), 164)
    rows, packed, g = smoe.rows8_pack(X.cuda()), smoe.weights8(W.cuda()), torch.from_numpy(gates).cuda()
    smoe.set_kernel_mode(mode)
    Y, Yhat = smoe.plinear8_fwd(rows, packed, r, k, g)
    assert torch.equal(Yhat, smoe.plinear8_fwd(rows, packed, r, k)[0])
    again = smoe.plinear8_fwd(rows, packed, r, k, g)
    assert torch.equal(Y, again[0]) and torch.equal(Yhat, again[1])
    t = np.arange(0, T, max(1, T // 200))
    x, w = oracle.unpack8(*oracle.pack8(_f64(X)), d_in), _stored(smoe, W)
    want = oracle.plinear8(x[t], w, idx[t], gates[t])
    got = _f64(Y[torch.from_numpy(t).cuda()])
    held = 1.9e-3 if k <= 8 and d_out % 64 == 0 else 2.6e-3
    if got.size >= 500:                                     # of fewer values the root mean square is no number to rely on
        off = np.sqrt(np.mean((got - want) ** 2) / np.mean(want ** 2))
        _log(f"  {off:.2e}")
        assert off <= held
    # every row: the sum of the rows that were left, two roundings away at most
    rough = (Yhat.double().view(T, k, d_out) * g.double()[..., None])
    tol = 2.0 ** -7 * rough.abs().sum(1) + 1e-30
    assert ((Y.double() - rough.sum(1)).abs() <= tol).all()


@MODES
def test_gates_over_other_groups_than_the_routing(smoe, mode):
    """gates_k need not be the fan-out: expert-sorted rows, one slot each, summed in groups of three."""
    T, k, E, d_in, d_out = 90, 3, 4, 256, 136
    idx, gates, r = _routed(smoe, T, E, k, 171)
    X, W = _normal((T, d_in), 172), _weights((E, d_in, d_out), 173)
    order = r.sorted_scattered_idxs.long()
    packed, g = smoe.weights8(W.cuda()), torch.from_numpy(gates).cuda()
    smoe.set_kernel_mode(mode)
    Y, Yhat = smoe.plinear8_fwd(smoe.rows8_pack(X.cuda()), packed, r, k, g)
    grouped = smoe.rows8_pack(X.cuda()[order // k].contiguous())
    Z, Zhat = smoe.plinear8_fwd(grouped, packed, r, 1, g, grouped_in=True)
    assert torch.equal(Y, Z) and torch.equal(Yhat, Zhat)


@MODES
def test_rows_of_all_sizes_and_bad_ones(smoe, mode):
    """Rows from 2^-100 to 2^100, of both signs, next to rows of NaN, of infinities past fp32 and of zeros: Yhat as without gates, each sum by itself."""
    T, k, E, d_in, d_out = 280, 2, 3, 128, 200
    idx, gates, r = _routed(smoe, T, E, k, 181)
    X = (_normal((T, d_in), 182).float() * 2.0 ** torch.linspace(-100, 100, T).round()[:, None]).to(torch.bfloat16)
    X[5, 9], X[150], X[200] = float("nan"), 0, 3e38
    W = _weights((E, d_in, d_out), 183)
    rows, packed, g = smoe.rows8_pack(X.cuda()), smoe.weights8(W.cuda()), torch.from_numpy(gates).cuda()
    smoe.set_kernel_mode(mode)
    Y, Yhat = smoe.plinear8_fwd(rows, packed, r, k, g)
    plain = smoe.plinear8_fwd(rows, packed, r, k)[0]
    assert torch.equal(Yhat.isnan(), plain.isnan()) and torch.equal(Yhat.nan_to_num(0.0), plain.nan_to_num(0.0))
    assert torch.isnan(Y[5]).all() and (Y[150] == 0).all() and torch.isfinite(Y[[4, 6, 149, 151]]).all()
    t = [i for i in range(T) if i not in (5, 150, 200)]
    rough = Yhat.double().view(T, k, d_out) * g.double()[..., None]
    assert ((Y.double() - rough.sum(1)).abs() <= 2.0 ** -7 * rough.abs().sum(1) + 1e-38)[t].all()


def test_sums_replay_from_a_graph(smoe):
    T, k, E, d_in, d_out = 700, 4, 8, 384, 264
    _, gates, r = _routed(smoe, T, E, k, 191)
    packed, g = smoe.weights8(_weights((E, d_in, d_out), 192).cuda()), torch.from_numpy(gates).cuda()
    rows = smoe.rows8_pack(_normal((T, d_in), 193).cuda())
    call = lambda: smoe.plinear8_fwd(rows, packed, r, k, g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        Y, Yhat = call()
    for seed in (194, 195, 194):
        smoe.rows8_pack(_normal((T, d_in), seed).cuda(), out=rows)
        graph.replay()
        torch.cuda.synchronize()
        a, b = call()
        assert torch.equal(Y, a) and torch.equal(Yhat, b)
