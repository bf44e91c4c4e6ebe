"""Edges of the paged cache and the attention over it: queries that attend nothing, lengths at the ends of int32."""
import sys

import numpy as np
import pytest
import torch

import oracle
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


@pytest.mark.parametrize("turned", [False, True])
def test_the_largest_values_stay_finite_in_8_bits(smoe, turned):
    """bf16 holds finite values up to (2 - 2^-7) 2^127.  Of a row whose scale is 2^120, those from 248 2^120 on are nearer to 2^128 than to 240 2^120,
    but no type here holds 2^128: they are stored as the latter.  Everything else as ever.  (Turned by position 0, which changes nothing.)"""
    _log(f"largest values in 8 bits turned={turned}")
    top, page, d = torch.finfo(torch.bfloat16).max, 16, 64
    big = 2.0 ** 127
    heads = [top, -top, 1.9375 * big, -1.9375 * big, 1.9296875 * big, 1.875 * big, -1.8828125 * big, 1.75 * big]
    x = _normal((8, 1, d), 321)
    x[:, 0, ::7] *= 2.0 ** 120
    for i, v in enumerate(heads):
        x[i, 0, i] = v
        x[i, 0, 20] = -v / 3
    cache = smoe.kv_cache(1, page, 1, d, True)
    table, lens = torch.zeros(1, 1, dtype=torch.int32).cuda(), torch.tensor([8], dtype=torch.int32).cuda()
    at = dict(seqs=torch.zeros(8, dtype=torch.int32).cuda(), positions=torch.zeros(8, dtype=torch.int32).cuda()) if turned else dict(lens=lens)
    if turned:                            # position 0 for each of them: one sequence each
        table = torch.arange(8, dtype=torch.int32)[:, None].cuda()
        cache = smoe.kv_cache(8, page, 1, d, True)
        at["seqs"] = torch.arange(8, dtype=torch.int32).cuda()
    smoe.cache_append(cache, x.cuda(), x.cuda(), table, rotary=smoe.rotary_table(d) if turned else None, **at)
    read = smoe.cache_read(cache, table, **(at if turned else dict(at, N=8)))
    value = oracle.e4m3_values()
    want = np.stack([value[c] * 2.0 ** e for c, e in map(oracle.e4m3_encode, x.double().numpy().reshape(8, d))])
    want = np.clip(want, -240 * 2.0 ** 120, 240 * 2.0 ** 120)
    for t in read:
        assert bool(t.isfinite().all()) and np.array_equal(t.double().cpu().numpy().reshape(8, d), want)


def test_every_stored_value_is_read_as_it_is(smoe):
    """All 256 codes at scales over the whole range: exact in bf16, but for e < -124, where the smallest steps (2^-9 2^e) lie under bf16's least (2^-133)
    and the value is rounded to the nearest once."""
    _log("every stored value")
    bytes_ = [1, 2, 3, 4, 60, 127, 200, 246]
    codes = torch.arange(256, dtype=torch.uint8).view(4, 64)
    cache = smoe.kv_cache(len(bytes_), 16, 1, 64, True)
    for i, e in enumerate(bytes_):
        for t, exps in ((cache.K, cache.K_exp), (cache.V, cache.V_exp)):
            t[i, 0, :4] = codes.cuda()
            exps[i, 0, :4] = e
    table = torch.arange(len(bytes_), dtype=torch.int32)[:, None].cuda()
    lens = torch.full((len(bytes_),), 4, dtype=torch.int32).cuda()
    for t in smoe.cache_read(cache, table, lens=lens, N=4):
        got = t.double().cpu().numpy().reshape(len(bytes_), 256)
        for row, e in zip(got, bytes_):
            want = oracle.e4m3_values() * 2.0 ** (e - 127)
            step = np.exp2(np.maximum(np.floor(np.log2(np.maximum(np.abs(want), 2.0 ** -126))) - 7, -133))
            nearest = np.where(np.isnan(want), want, np.rint(want / step) * step)
            assert np.array_equal(row, nearest, equal_nan=True), e
            assert e < 3 or np.array_equal(nearest, want, equal_nan=True)
