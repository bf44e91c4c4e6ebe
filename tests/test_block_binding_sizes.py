"""Sizes and numbers that 32 bits do not hold never reach the library cut down to other ones (CPU, with stand-ins for device tensors)."""
import pytest

from test_block_refusals import a_rows, a_weights, bytes_, floats, launches, m, smoe  # noqa: F401 (fixtures)
from test_cache_binding import Tensor, ints

WRAPS = (2 ** 32, -2 ** 32)


@pytest.mark.parametrize("by", WRAPS)
@pytest.mark.parametrize("name,value", [("groups", 4), ("kept_groups", 2), ("group_best", 2)])
def test_gate_rule(smoe, name, value, by):
    rule = dict(groups=4, kept_groups=2, group_best=2)
    smoe.gate_rule("sigmoid", **rule)
    with pytest.raises(ValueError):
        smoe.gate_rule("sigmoid", **{**rule, name: value + by})


@pytest.mark.parametrize("scale", [1e39, -1e39, float("inf"), float("nan")])
def test_gate_scale(smoe, scale):
    with pytest.raises(ValueError):
        smoe.gate_rule("softmax", scale=scale)


@pytest.mark.parametrize("by", WRAPS)
def test_products(smoe, by):
    r = smoe.Routing(ints(8), ints(8), ints(5), 8, 4)
    none = smoe.Routing(ints(0), ints(0), ints(5), 0, 4)
    X, W1, W2, g = a_rows(smoe, 4, 96), a_weights(smoe, 4, 96, 128, 2), a_weights(smoe, 4, 64, 96), floats(4, 2)
    G1 = a_weights(smoe, 4, 96, 64)
    for bad in (lambda: smoe.plinear8_fwd(a_rows(smoe, 4, 64), W2, r, 2 + by), lambda: smoe.plinear8_fwd(a_rows(smoe, 4, 64), W2, r, 2 + by, g),
                lambda: smoe.plinear8_fwd(a_rows(smoe, 8, 64), W2, r, 1 + by, grouped_in=True), lambda: smoe.mlp8_fwd(X, W1, W2, r, 2 + by, g, smoe.ACT_SWIGLU),
                lambda: smoe.mlp8_fwd(a_rows(smoe, 0, 96), W1, W2, none, 2 + by, floats(0, 2), smoe.ACT_SWIGLU), lambda: smoe.mlp8_fwd(X, G1, W2, r, 2, g, smoe.ACT_GELU + by)):
        with pytest.raises(ValueError):
            bad()
    assert not launches(smoe)


@pytest.mark.parametrize("by", WRAPS)
def test_weights(smoe, by):
    nb = 2 * 2 * 2048
    for E, d_in, d_out, halves in ((2 + by, 128, 32, 1), (2, 128 + by, 32, 1), (2, 128, 32 + by, 1), (2, 128, 32, 1 + by)):
        with pytest.raises(ValueError):
            smoe.Weights8(bytes_(nb), bytes_(nb // 32), E, d_in, d_out, halves)
    with pytest.raises(ValueError):
        smoe.weights8(Tensor(2, 128, 32), halves=1 + by)
    assert not launches(smoe)


