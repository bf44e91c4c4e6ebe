"""Edges of the paged cache and the attention over it: queries that attend nothing, lengths at the ends of int32."""
import sys

import numpy as np
import pytest
import torch

from test_gpu_cache import _case, _normal

pytestmark = pytest.mark.gpu


def _log(*a):
    print(*a, flush=True, file=sys.stderr)


@pytest.fixture(scope="module")
def smoe():
    import paper_2403_08245_amd as m
    return m


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("lens,N,G", [([40, 33, 64], 1, 2), ([900, 33, 2000], 1, 2), ([40, 33, 64], 3, 2), ([900, 33, 2000], 3, 2), ([900, 33, 2000], 2, 12)])
def test_a_query_that_attends_nothing_gives_zeros_whatever_the_values_hold(smoe, lens, N, G, value):
    """All of the scores that the first and the last sequence's queries see are -infinity, in one piece or several: O = 0 and LSE = -infinity, also where the
    values at those positions are infinite or NaN.  The sequence between them is what it is without them."""
    _log(f"attends nothing lens={lens} N={N} G={G} {value}")
    cache, table, K, V = _case(smoe, lens, 16, 2, 128, False, 301)
    Q = torch.ones(3, N, G, 2, 128).bfloat16()
    n = torch.tensor(lens, dtype=torch.int32).cuda()
    want = smoe.cached_attention_fwd(Q.cuda(), cache, table.cuda(), n)
    for b in (0, 2):
        used = table[b, :-(-lens[b] // 16)].long().cuda()
        cache.K[used] = float("-inf")
        cache.V[used] = value
    O, L = smoe.cached_attention_fwd(Q.cuda(), cache, table.cuda(), n)
    for b in (0, 2):
        assert bool((O[b] == 0).all()) and bool((L[b] == -np.inf).all())
    assert torch.equal(O[1], want[0][1]) and torch.equal(L[1], want[1][1])
