"""The gate by scores at logits whose scores 64 bits do not hold apart, and at masks of large finite values, against the fp64 oracle."""
import numpy as np
import pytest
import torch

import oracle
from test_gpu_block import _f64, _log, _near, _normal, _weight_units

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def smoe():
    import paper_2403_08245_amd as m
    return m


def _compare(smoe, x, b, k, score, groups, kept, best, renormalise):
    rule = dict(score=score, renormalise=renormalise, scale=1.5)
    idx, w = oracle.score_gate(_f64(x), k, bias=None if b is None else _f64(b), groups=groups, kept_groups=kept, group_best=best, **rule)
    got, gates = smoe.score_gate(x.cuda(), k, smoe.gate_rule(score, groups, kept, best, renormalise, 1.5), None if b is None else b.cuda())
    assert np.array_equal(got.cpu().numpy(), idx)
    _near(gates, w, _weight_units(np.clip(_f64(x), -100, 100)) * np.abs(w) + 1e-37, "gates")       # differences past 100 leave nothing of a weight
    return idx


FORMS = pytest.mark.parametrize("E,k,groups,kept,best", [(8, 2, 1, 1, 1), (64, 6, 1, 1, 1), (64, 6, 8, 3, 1), (64, 6, 8, 8, 2), (64, 6, 8, 3, 2), (256, 8, 8, 8, 2), (256, 8, 8, 4, 1), (60, 20, 5, 5, 2), (700, 9, 1, 1, 1)])


@FORMS
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("bias", [False, True])
def test_scores_that_are_equal_in_64_bits(smoe, E, k, groups, kept, best, score, bias):
    """Without a bias the exact scores' order, which is the logits'; with one, of zeros here, 64-bit scores and the lower expert."""
    _log(f"gate saturated {score} {bias} {(E, k, groups, kept, best)}")
    b = torch.zeros(E) if bias else None
    u = torch.rand(4, E, generator=torch.Generator().manual_seed(1))
    rows = [25 + 35 * u[0], 38 + 60 * u[1], 1e-20 * (u[2] - 0.5), 20 + 2.0 ** -16 * (u[3] * 64).round()]
    if score == "softmax":
        rows.append(-2000 * u[0])                           # scores that are 0 in 64 bits
    idx = _compare(smoe, torch.stack(rows).float(), b, k, score, groups, kept, best, True)
    if score == "sigmoid" and bias and kept == groups:
        assert idx[1].tolist() == list(range(k))            # all 1
    if not bias and kept == groups:
        assert idx[1, 0] == int(rows[1].argmax())


@FORMS
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("mask", [-1e9, torch.finfo(torch.float32).min])
def test_large_finite_masks_and_logits_of_bf16_values(smoe, E, k, groups, kept, best, score, bias, mask):
    """Experts masked by a large finite number, which are not the masked ones of the definition: they have a score, however small.  Logits of few bits tie often."""
    _log(f"gate finite masks {score} {bias} {(E, k, groups, kept, best)}")
    x = _normal((40, E), 11).float()
    x[10:20, 1::3] = mask
    x[20:30, : E - 1] = mask
    x[30:33] = mask
    b = _normal((E,), 12, torch.float32, 0.1) if bias else None
    for renormalise in (False, True):
        _compare(smoe, x, b, k, score, groups, kept, best, renormalise)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E", [3, 8, 16, 60, 64])
def test_every_expert_chosen(smoe, E, score):
    x = _normal((50, E), 13, torch.float32)
    for b in (None, _normal((E,), 14, torch.float32, 0.1)):
        _compare(smoe, x, b, E, score, 1, 1, 1, True)
