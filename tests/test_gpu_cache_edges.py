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


@pytest.mark.parametrize("rotary", [False, True])
def test_lengths_at_the_ends_of_int32_have_no_places(smoe, rotary):
    """lens[b] - N under -2^31 does not come out as a position at the other end: nothing is written, and reads are zeros.  (65540 new positions in a
    table of 32767 pages of 65536, all of them the one page there is: 2^31 - 65540 would be one of its positions.)"""
    N, page, width = 65540, 65536, 32767
    _log(f"lengths at the ends of int32 rotary={rotary}")
    cache = smoe.kv_cache(1, page, 1, 64)
    for t in (cache.K, cache.V):
        t.fill_(3.0)
    table = torch.zeros(1, width, dtype=torch.int32).cuda()
    K = torch.ones(N, 1, 64, dtype=torch.bfloat16).cuda()
    more = dict(rotary=smoe.rotary_table(64)) if rotary else {}
    for told in (-2 ** 31, -2 ** 31 + 3, -2 ** 31 + N - 1, -1, 0):
        lens = torch.tensor([told], dtype=torch.int64).to(torch.int32).cuda()
        smoe.cache_append(cache, K, K, table, lens=lens, **more)
        assert bool((cache.K == 3.0).all()) and bool((cache.V == 3.0).all()), told
        k, v = smoe.cache_read(cache, table, lens=lens, N=N)
        assert not k.any() and not v.any(), told
