"""How near the experts' products in 8 bits come to the definition in 64 bits: the hidden rows' codes one by one, and whole outputs in the root mean square, which bounds
of single entries that add up every error's worst case cannot show.

A second product with the identity shows the hidden rows themselves: what a code stands for has four bits, which bf16 keeps.
What a code may be off: a value h is rounded to steps of 2^-4 to 2^-3 of it, so an error of d |h| takes it over a border with a probability of about d / 0.09.  h is made of one
normal factor (GELU) or two (SwiGLU) whose products have errors of d times their deviation; over the factor's distribution, down to where it is as small as d / 0.09 itself,
that is 0.8 (d / 0.09) ln(0.09 / d) for each.
  Few rows: bf16 products (exact) in fp32 sums, 512 / 32 of them one behind the other, and the activation's roundings: d = 3e-7, 7e-5 of the codes for two factors.  Held to 2e-4.
  Many rows: the 8-bit instruction's sums, d = 1.4e-5: 2.2e-3.  Held to 6.6e-3.
Root mean square of a whole output: its own rounding, at most 2^-8 / sqrt(3) = 2.26e-3, and the rows' of the weighted sum, 2^-11 / sqrt(3) = 2.8e-4; a share p of codes off by
a step, 2^-3 at most, adds sqrt(p) / 8: 0.8e-3 for 4e-5 of the codes, 3.1e-3 for 6e-4.  In all 2.4e-3 and 3.9e-3, held to 2.75e-3 and 4e-3."""
import numpy as np
import pytest
import torch

import oracle
from test_gpu_block import _f64, _log, _mlp_case, _normal, _routed, _stored, _weights

pytestmark = pytest.mark.gpu
FEW, HALF_TILES, BIG_TILES = 1, 3, 4        # smoe_set_kernel_mode
WHOLE = {FEW: 2.75e-3, HALF_TILES: 4e-3, BIG_TILES: 4e-3}
CODES = {FEW: 2e-4, HALF_TILES: 6.6e-3, BIG_TILES: 6.6e-3}
MODES = pytest.mark.parametrize("mode", [FEW, HALF_TILES, BIG_TILES], ids=["few rows", "128 x 256", "256 x 256"])
# One code a step off moves a token's output by 2^-3 |h| of that hidden value's row of W2 at most, so by less than 2^-3 of the output's size; with what else is off:
ONE = 0.15


@pytest.fixture(scope="module")
def smoe():
    import paper_2403_08245_amd as m
    yield m
    m.set_kernel_mode(0)


def _rms(a):
    return float(np.sqrt(np.mean(np.square(a))))


def _pieces(y):
    """Norms of a row's pieces of 128 columns, [rows, pieces]."""
    n = -(-y.shape[1] // 128)
    full = np.zeros((y.shape[0], n * 128))
    full[:, :y.shape[1]] = y
    return np.sqrt(np.square(full.reshape(-1, n, 128)).sum(-1))


def _close_by_rows(got, want, what):
    """Every piece of 128 columns of every row, to what a code or two a step off and the roundings leave of it."""
    off, size = _pieces(got - want), _pieces(want)
    assert (off <= ONE * size).all(), f"{what}: {int((off > ONE * size).sum())} of {off.size} pieces, worst {np.max(off / np.maximum(size, 1e-300)):.3f}"


@MODES
@pytest.mark.parametrize("act", ["swiglu", "gelu"])
@pytest.mark.parametrize("T,E,k", [(64, 16, 2), (150, 16, 2)])
def test_codes_of_the_hidden_rows(smoe, mode, act, T, E, k):
    d = 512
    _log(f"codes {mode} {act} {T}")
    idx, _, r = _routed(smoe, T, E, k, 91)
    code = smoe.ACT_SWIGLU if act == "swiglu" else smoe.ACT_GELU
    X = _normal((T, d), 92) * torch.exp(0.7 * _normal((d,), 93))
    W1 = _weights((E, d, smoe.hidden_width(code, d)), 94)
    eye = torch.eye(d).expand(E, d, d).contiguous().to(torch.bfloat16)
    gates = torch.zeros(T, k)
    gates[:, k - 1] = 1.0                                   # the last slot's hidden row and nothing else
    smoe.set_kernel_mode(mode)
    Y = smoe.mlp8_fwd(smoe.rows8_pack(X.cuda()), smoe.weights8(W1.cuda(), halves=2 if act == "swiglu" else 1), smoe.weights8(eye.cuda()), r, k, gates.cuda(), code)
    x, w1 = oracle.unpack8(*oracle.pack8(_f64(X)), d), _stored(smoe, W1)
    want, _ = oracle.mlp8(x, w1, _f64(eye), idx, gates.double().numpy(), code)
    other = _f64(Y) != want
    assert other.mean() <= CODES[mode], f"{int(other.sum())} of {other.size} codes"
    # those that differ are the next code, at the most with their block's steps doubled
    assert (np.abs(_f64(Y) - want)[other] <= 2.0 ** -2 * np.abs(want)[other] + np.abs(want).max() * 2.0 ** -16).all()


LAYERS = [  # T, d_model, d_expert, E, k, act
    (64, 512, 224, 64, 8, "swiglu"), (300, 256, 264, 4, 2, "swiglu"), (257, 304, 200, 2, 2, "gelu"), (200, 384, 1000, 3, 2, "swiglu"), (40, 2048, 512, 8, 4, "swiglu"),
]


@MODES
@pytest.mark.parametrize("T,d_model,d_expert,E,k,act", LAYERS)
def test_layer_in_the_root_mean_square(smoe, mode, T, d_model, d_expert, E, k, act):
    _log(f"rms {mode} {(T, d_model, d_expert, E, k, act)}")
    idx, gates, r, code, X, W1, W2, packed = _mlp_case(smoe, T, d_model, d_expert, E, k, act, seed=101)
    smoe.set_kernel_mode(mode)
    Y = _f64(smoe.mlp8_fwd(smoe.rows8_pack(X.cuda()), *packed, r, k, torch.from_numpy(gates).cuda(), code))
    x = oracle.unpack8(*oracle.pack8(_f64(X)), d_model)
    want, _ = oracle.mlp8(x, _stored(smoe, W1), _stored(smoe, W2), idx, gates.astype(np.float64), code)
    _close_by_rows(Y, want, "Y")
    off = _rms(Y - want) / _rms(want)
    _log(f"  {off:.2e}")
    assert off <= WHOLE[mode]


@pytest.mark.parametrize("mode", [HALF_TILES, BIG_TILES])
@pytest.mark.parametrize("T,d_model,d_expert,E,k,act", [(1500, 512, 224, 64, 8, "swiglu"), (2000, 264, 161, 6, 3, "swiglu"), (900, 640, 320, 5, 2, "gelu"), (700, 120, 128, 4, 2, "swiglu"),
                                                          (520, 384, 1000, 3, 2, "swiglu"), (3000, 256, 640, 2, 1, "gelu")])
def test_every_row_of_both_kernels(smoe, mode, T, d_model, d_expert, E, k, act):
    """No row is left out, another token's, or a power of two off: each piece of 128 columns of each row against the kernels for few rows."""
    _log(f"rows {mode} {(T, d_model, d_expert, E, k, act)}")
    idx, gates, r, code, X, W1, W2, packed = _mlp_case(smoe, T, d_model, d_expert, E, k, act, seed=111, skew=0.7)
    rows, g = smoe.rows8_pack(X.cuda()), torch.from_numpy(gates).cuda()
    Y = {}
    for m in (FEW, mode):
        smoe.set_kernel_mode(m)
        Y[m] = _f64(smoe.mlp8_fwd(rows, *packed, r, k, g, code))
    _close_by_rows(Y[mode], Y[FEW], "Y")
    assert _rms(Y[mode] - Y[FEW]) / _rms(Y[FEW]) <= WHOLE[mode] + WHOLE[FEW]


def test_many_routed_rows_on_the_kernels_for_few(smoe):
    """More routed rows than the layer sums from fp32 (8192): no rounding to bf16 between the second product and the sum.  Values of one sign and logarithm spread evenly are off by
    2^-7 / sqrt(12) sqrt(0.375 / ln 2) = 1.66e-3 after one rounding to bf16, 2.35e-3 after two; fp16 rows add 2.1e-4, hidden codes 0.8e-3."""
    T, d_model, d_expert, E, k = 4200, 264, 96, 6, 2
    _log("rms of many rows on the kernels for few")
    idx, gates, r, code, X, W1, W2, packed = _mlp_case(smoe, T, d_model, d_expert, E, k, "swiglu", seed=121)
    smoe.set_kernel_mode(FEW)
    Y = smoe.mlp8_fwd(smoe.rows8_pack(X.cuda()), *packed, r, k, torch.from_numpy(gates).cuda(), code)
    sample = np.arange(0, T, 13)
    x = oracle.unpack8(*oracle.pack8(_f64(X[sample])), d_model)
    want, _ = oracle.mlp8(x, _stored(smoe, W1), _stored(smoe, W2), idx[sample], gates[sample].astype(np.float64), code)
    got = _f64(Y[torch.from_numpy(sample).cuda()])
    _close_by_rows(got, want, "Y")
    assert _rms(got - want) / _rms(want) <= 1.9e-3


@pytest.mark.parametrize("d_model", [256, 72])
def test_many_rows_of_all_sizes_on_the_kernels_for_few(smoe, d_model):
    """Rows from 2^-60 to 2^30, as many as are summed from fp16 with a power of two for 64 columns; a row of NaN, and one of products past fp32."""
    T, E, k = 4200, 3, 2
    idx, gates, r, code, X, W1, W2, packed = _mlp_case(smoe, T, d_model, 160, E, k, "swiglu", seed=131)
    X = (X.float() * 2.0 ** torch.linspace(-60, 30, T).round()[:, None]).to(torch.bfloat16)
    X[77, 3] = float("nan")
    X[1234] = 1e30
    smoe.set_kernel_mode(FEW)
    Y = smoe.mlp8_fwd(smoe.rows8_pack(X.cuda()), *packed, r, k, torch.from_numpy(gates).cuda(), code)
    sample = np.array([t for t in range(0, T, 21) if t not in (77, 1234)])
    x = oracle.unpack8(*oracle.pack8(_f64(X[sample])), d_model)
    with np.errstate(over="ignore"):
        want, _ = oracle.mlp8(x, _stored(smoe, W1), _stored(smoe, W2), idx[sample], gates[sample].astype(np.float64), code)
    got = _f64(Y[torch.from_numpy(sample).cuda()])
    off, size = _pieces(got - want), _pieces(want)
    assert (off <= ONE * size + 1e-37).all()                # under 1e-37 fp32 has fewer bits
    assert torch.isnan(Y[77]).all() and torch.isfinite(Y[[76, 78, 1233, 1235]]).all()


def test_small_rows_on_the_kernels_for_few(smoe):
    """Rows down to 2^-112, whose codes stand for numbers next to the least that bf16 and fp32 hold in full."""
    T, d, E, k = 60, 256, 3, 1
    idx, gates, r, code, X, W1, W2, packed = _mlp_case(smoe, T, d, 160, E, k, "gelu", seed=201)
    X = (X.float() * 2.0 ** torch.linspace(-112, -40, T).round()[:, None]).to(torch.bfloat16)
    smoe.set_kernel_mode(FEW)
    Y = _f64(smoe.mlp8_fwd(smoe.rows8_pack(X.cuda()), *packed, r, k, torch.from_numpy(gates).cuda(), code))
    x = oracle.unpack8(*oracle.pack8(_f64(X)), d)
    want, _ = oracle.mlp8(x, _stored(smoe, W1), _stored(smoe, W2), idx, gates.astype(np.float64), code)
    off, size = _pieces(Y - want), _pieces(want)
    assert (off <= ONE * size + 1e-37).all()
    assert _rms(Y[20:] / np.abs(want[20:]).max(1, keepdims=True) - want[20:] / np.abs(want[20:]).max(1, keepdims=True)) <= 1e-3      # rounding alone: 1.66e-3 of a value, a third of the largest
