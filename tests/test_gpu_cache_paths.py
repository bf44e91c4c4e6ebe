"""The forms of the cache's and positions' kernels that sizes select: many sequences, cut ones, several rounds of rows, reads past the caches, two
numbers a weight.  Each test states, in the rule's own terms, that its sizes reach the form it is for."""
import math
import sys

import numpy as np
import pytest
import torch

import oracle
from test_gpu_cache import HALF_STEP, _case, _check_attention, _f64, _gen, _normal, _table

pytestmark = pytest.mark.gpu

LAST_LEVEL_CACHE = 256 << 20


def _log(*a):
    print(*a, flush=True, file=sys.stderr)


@pytest.fixture(scope="module")
def smoe():
    import paper_2403_08245_amd as m
    return m


class Cut:
    """How the attention cuts a batch: steps of 32 keys, a piece as long as makes about `target` of them over the batch, 8 steps at least; sequences of
    up to 16 steps whole; 256 pieces at most."""

    def __init__(self, lens, cap, N, G, h, d=128):
        R = N * G
        two = R > 16
        tiles = -(-R // (32 if two else 16))
        self.rows, self.units = min(R, 32 if two else 16), tiles * h
        self.target = 512 if two or N > 1 else 768
        steps = [max(-(-min(max(n, 0), cap) // 32), 1) for n in lens]
        per = max(int(sum(steps) * self.units * 1.01 / self.target) + 1, 8)
        self.pieces = [1 if cap <= 512 or s <= 16 else min(-(-s // per), 256) for s in steps]
        self.long = [-(-s // n) for s, n in zip(steps, self.pieces)]            # steps of a piece
        self.empty = [n - -(-s // l) for s, n, l in zip(steps, self.pieces, self.long)]
        self.cut_units = sum(n > 1 for n in self.pieces) * self.units
        self.a_lane = -(-len(lens) // 64)                                       # sequences of a lane
        most = min(len(lens) * self.units, self.target)                         # units that the join's launch provides for
        self.join_rows = 1
        while 2 * self.join_rows <= 1024 // d and self.join_rows < self.rows and most * -(-self.rows // (2 * self.join_rows)) >= 512:
            self.join_rows *= 2


# ---------------------------------------------------------------------------------------------------- the cut of many sequences
def _ragged(B, long):
    lens = [(i * 37) % 23 for i in range(B)]
    for b, n in long.items():
        lens[b] = n
    return lens


@pytest.mark.parametrize("B,long,N,G,h,d,a_lane", [
    (70, {69: 700, 1: 513}, 1, 2, 2, 64, 2), (300, {5: 700, 64: 513, 150: 1300, 151: 512, 299: 2049}, 1, 2, 2, 64, 5), (300, {0: 900, 298: 530}, 2, 3, 1, 128, 5),
    (300, {299: 1111}, 3, 7, 1, 64, 5), (4200, {0: 600, 63: 513, 64: 700, 65: 1200, 131: 800, 4199: 1024}, 1, 1, 1, 64, 66), (4200, {65: 3000}, 2, 2, 1, 64, 66)])
@pytest.mark.parametrize("quantised", [False, True])
def test_cut_among_many_sequences(smoe, B, long, N, G, h, d, a_lane, quantised):
    """More sequences than a wavefront has lanes, than the lengths a lane keeps (256 in all), and than a lane's neighbours search at once (4096), with a few
    long ones in several pieces among them."""
    lens = _ragged(B, long)
    cut = Cut(lens, 10 ** 9, N, G, h)
    _log(f"cut among {B} N={N} G={G} h={h} d={d} e4m3={quantised}: pieces {[cut.pieces[b] for b in long]}")
    assert cut.a_lane == a_lane and cut.cut_units >= 1 and all((cut.pieces[b] > 1) == (lens[b] > 512) for b in range(B))
    cache, table, K, V = _case(smoe, lens, 16, h, d, quantised, 401)
    assert table.shape[1] * 16 > 512
    Q = _normal((B, N, G, h, d), 404)
    O, L = smoe.cached_attention_fwd(Q.cuda(), cache, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    _check_attention(O, L, Q, K, V, lens)


@pytest.mark.parametrize("B,h,G,d,join_rows", [(64, 4, 4, 128, 2), (150, 4, 4, 128, 4), (150, 4, 3, 64, 4), (80, 8, 16, 128, 8)])
def test_join_of_several_rows_a_block(smoe, B, h, G, d, join_rows):
    lens = [(i * 97) % 600 + 1 for i in range(B)]
    lens[0], lens[B // 2], lens[B - 1] = 2100, 1300, 900
    cut = Cut(lens, 10 ** 9, 1, G, h, d)
    _log(f"join of several rows {B} {h} {G} {d}: {cut.join_rows} rows, {cut.cut_units} units cut")
    assert cut.join_rows == join_rows and cut.cut_units >= 2 * h
    cache, table, K, V = _case(smoe, lens, 32, h, d, False, 411)
    Q = _normal((B, 1, G, h, d), 414)
    O, L = smoe.cached_attention_fwd(Q.cuda(), cache, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    _check_attention(O, L, Q, K, V, lens)


@pytest.mark.parametrize("N,G", [(1, 1), (1, 12), (2, 12)])
def test_as_many_pieces_as_there_may_be(smoe, N, G):
    """One sequence of 65600 keys: 257 pieces of 8 steps would be, 256 of 9 are, the last of them empty."""
    lens = [65600]
    cut = Cut(lens, 10 ** 9, N, G, 1)
    _log(f"most pieces N={N} G={G}: {cut.pieces} of {cut.long}, {cut.empty} empty")
    assert cut.pieces == [256] and cut.empty[0] > 0
    cache, table, K, V = _case(smoe, lens, 64, 1, 64, False, 421)
    Q = _normal((1, N, G, 1, 64), 424)
    O, L = smoe.cached_attention_fwd(Q.cuda(), cache, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    _check_attention(O, L, Q, K, V, lens)


@pytest.mark.parametrize("N,G", [(1, 4), (3, 2), (3, 8)])
@pytest.mark.parametrize("quantised", [False, True])
def test_attention_past_the_caches(smoe, N, G, quantised):
    """A table that reaches more than 64 MB of cache is read past the caches, a narrower one through them: the same bits, and right ones."""
    page, h, d, lens = 256, 8, 128, [3000, 17, 512]
    _log(f"attention past the caches N={N} G={G} e4m3={quantised}")
    size = page * h * d * (2 if quantised else 4)
    extra = LAST_LEVEL_CACHE // 4 // size
    K, V = _normal((sum(lens), h, d), 431), _normal((sum(lens), h, d), 432)
    table, pages = _table(lens, page, 433, spare=extra)
    assert 3 * table.shape[1] * size < LAST_LEVEL_CACHE // 4 < min(pages, 3 * (table.shape[1] + extra)) * size
    cache = smoe.kv_cache(pages, page, h, d, quantised)
    seqs = torch.tensor([b for b, n in enumerate(lens) for _ in range(n)], dtype=torch.int32).cuda()
    pos = torch.tensor([p for n in lens for p in range(n)], dtype=torch.int32).cuda()
    smoe.cache_append(cache, K.cuda(), V.cuda(), table.cuda(), seqs=seqs, positions=pos)
    k, v = smoe.cache_read(cache, table.cuda(), seqs=seqs, positions=pos)
    split = lambda t: np.split(_f64(t), np.cumsum(lens)[:-1])
    Q, n = _normal((3, N, G, h, d), 434), torch.tensor(lens, dtype=torch.int32).cuda()
    O, L = smoe.cached_attention_fwd(Q.cuda(), cache, table.cuda(), n)
    wide = torch.cat([table, torch.full((3, extra), -1, dtype=torch.int32)], 1).cuda()
    past = smoe.cached_attention_fwd(Q.cuda(), cache, wide, n)
    assert torch.equal(O, past[0]) and torch.equal(L, past[1])
    _check_attention(*past, Q, split(k), split(v), lens)


# ------------------------------------------------------------------------------------------------ what two numbers a weight are for
@pytest.mark.parametrize("lens,N,G,h,d", [([1], 1, 1, 1, 128), ([40, 511, 17], 1, 4, 2, 128), ([3000, 40], 1, 4, 1, 64), ([40, 300], 3, 2, 1, 128), ([3000, 40], 3, 2, 2, 64),
                                          ([300, 50], 2, 12, 1, 128), ([3000, 50], 2, 12, 1, 128)])
@pytest.mark.parametrize("quantised", [False, True])
def test_weights_that_add_up_to_one(smoe, lens, N, G, h, d, quantised):
    """Columns of one value: O is that value, whatever the weights are, as long as those that multiply it are those that are summed.  As two bf16
    numbers a weight is within 2^-16; the sums' roundings are 75 a step of 32 keys and wavefront at most (32 products of each of two instructions, the
    eight weights and their sum's) of 2^-24, and no wavefront here has more than 25 steps: together under 2^-12, a good deal less than the 2^-9 (half a
    step under a power of two) at which a bf16 value becomes its neighbour.  One number a weight, cut to 8 bits, is off by 2^-8 in the mean."""
    _log(f"weights add up lens={lens} N={N} G={G} h={h} d={d} e4m3={quantised}")
    assert all(-(-l // 4) <= 25 for l in Cut(lens, 10 ** 9, N, G, h).long)
    cache, table, K, V = _case(smoe, lens, 16, h, d, quantised, 441)
    seqs = torch.tensor([b for b, n in enumerate(lens) for _ in range(n)], dtype=torch.int32)
    pos = torch.tensor([p for n in lens for p in range(n)], dtype=torch.int32)
    value = torch.tensor([1.0, -1.0, 2.0, 0.5, 1.5, -1.75, 448.0, 1.25]).repeat(d // 8).bfloat16()       # e4m3 holds them at the scale of 448
    flat = torch.from_numpy(np.concatenate(K)).bfloat16().cuda()
    smoe.cache_append(cache, flat, value.expand(len(seqs), h, d).contiguous().cuda(), table.cuda(), seqs=seqs.cuda(), positions=pos.cuda())
    O, _ = smoe.cached_attention_fwd(_normal((len(lens), N, G, h, d), 444).cuda(), cache, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    for b, n in enumerate(lens):
        for i in range(N):
            want = value if n - N + i >= 0 else torch.zeros_like(value)
            assert torch.equal(O[b, i].cpu(), want.expand(G, h, d)), (b, i)


def _attend64(Q, K, V):
    """Q [N, G, h, d], K and V [len, h, d] on the device, in 64 bits: O, the same of |V|, and what fp32 can cost a score (d + 2 roundings of 2^-24
    of the sum of |q k| / sqrt(d))."""
    N, G, h, d = Q.shape
    q, k, v = Q.double().permute(2, 0, 1, 3).reshape(h, N * G, d), K.double().permute(1, 2, 0).contiguous(), V.double().permute(1, 0, 2).contiguous()
    s = torch.matmul(q, k) / math.sqrt(d)
    n = K.shape[0]
    hidden = torch.arange(n, device=s.device)[None] > (n - N + torch.arange(N, device=s.device)).repeat_interleave(G)[:, None]
    p = torch.softmax(s.masked_fill(hidden, -math.inf), -1)
    e = torch.matmul(q.abs(), k.abs()).amax(-1) * ((d + 2) * 2.0 ** -24 / math.sqrt(d))
    back = lambda t: t.view(h, N, G, -1).permute(1, 2, 0, 3)
    return back(torch.matmul(p, v)), back(torch.matmul(p, v.abs())), back(e[..., None])


@pytest.mark.parametrize("lens,N,G,h,d", [([40, 511, 77], 1, 4, 2, 128), ([3000, 40], 1, 4, 1, 64), ([40, 300], 3, 2, 1, 128), ([3000, 50], 2, 12, 1, 128)])
@pytest.mark.parametrize("quantised", [False, True])
def test_attention_carries_sixteen_bits_of_the_weights(smoe, lens, N, G, h, d, quantised):
    """|O - O*| <= 2^-8 |O*|, the output's own rounding, and (2^-16 + 2^-17 + 2 e + 2^-12) sum p |v| before it: two bf16 numbers a weight, exponentials
    of arguments under 2^5 and a quotient (good to 2^-18 and 2^-22), scores off by e, and the sums as in the test above.  Weights of one bf16 number would add 2^-8 sum p |v|."""
    _log(f"sixteen bits lens={lens} N={N} G={G} h={h} d={d} e4m3={quantised}")
    cache, table, K, V = _case(smoe, lens, 16, h, d, quantised, 451)
    Q = _normal((len(lens), N, G, h, d), 454).cuda()
    O, _ = smoe.cached_attention_fwd(Q, cache, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    for b in range(len(lens)):
        want, weight, e = _attend64(Q[b], torch.from_numpy(K[b]).cuda(), torch.from_numpy(V[b]).cuda())
        before = (2.0 ** -16 + 2.0 ** -17 + 2 * e + 2.0 ** -12) * weight
        err = (O[b].double() - want).abs()
        assert bool((err <= HALF_STEP * (want.abs() + before) + before).all()), float((err / (HALF_STEP * want.abs() + before)).max())


# ------------------------------------------------------------------------------------------------------- several rounds of rows
def _rounds(rows, heads, d):
    """Rounds of a token's rows that one wavefront takes."""
    rounds = -(-heads // (64 // (d // 8)))
    return min(max(rows * rounds // 8192, 1), 8, rounds)


@pytest.mark.parametrize("B,T,hq,hk,d,rot,dtype,rounds", [
    (2, 4096, 16, 4, 128, 128, torch.bfloat16, 5), (3, 2731, 16, 3, 128, 128, torch.bfloat16, 5), (2, 3001, 9, 2, 128, 40, torch.float32, 2), (1, 30011, 36, 2, 64, 64, torch.bfloat16, 5),
    (1, 9001, 19, 1, 72, 44, torch.bfloat16, 3), (1, 9001, 16, 15, 256, 130, torch.float32, 8)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_of_many_rows(smoe, B, T, hq, hk, d, rot, dtype, rounds, layout):
    """Wavefronts that take several rounds of a token's rows, two of them in flight, the last ones partly filled: against the formula in 64 bits (all
    rows, on the device), in place as out of place, and there and back."""
    assert _rounds(B * T, hq + hk, d) == rounds and rounds > 1
    _log(f"rotary of many rows {(B, T, hq, hk, d, rot)} {dtype} {layout}")
    gen = torch.Generator("cuda").manual_seed(461)
    new = lambda h: torch.randn(B, T, h, d, generator=gen, device="cuda").to(dtype)
    Q, K = new(hq), new(hk)
    positions = torch.randint(0, 200000, (B, T), generator=gen, device="cuda", dtype=torch.int32)
    table = smoe.rotary_table(rot, layout=layout)
    freqs = torch.from_numpy(oracle.rotary_frequencies(rot)[0]).cuda()
    w = (positions.double()[..., None, None] * freqs)
    n = rot // 2
    for entry, sign in ((smoe.rotary_fwd, 1.0), (smoe.rotary_bwd, -1.0)):
        got = entry(Q, K, table, positions)
        for x, y in zip((Q, K), got):
            pairs = (x[..., 0:rot:2], x[..., 1:rot:2]) if layout == "interleaved" else (x[..., :n], x[..., n:rot])
            out = (y[..., 0:rot:2], y[..., 1:rot:2]) if layout == "interleaved" else (y[..., :n], y[..., n:rot])
            a, b = (t.double() for t in pairs)
            fp32 = 6.4e-7 * (a.abs() + b.abs())               # as the tests of small sizes derive it
            for z, want in zip(out, (a * w.cos() - sign * b * w.sin(), sign * a * w.sin() + b * w.cos())):
                tol = fp32 if dtype == torch.float32 else fp32 * (1 + HALF_STEP) + HALF_STEP * want.abs()
                assert bool(((z.double() - want).abs() <= tol).all())
            assert torch.equal(y[..., rot:], x[..., rot:])
        q, k = Q.clone(), K.clone()
        entry(q, k, table, positions, out=(q, k))
        assert torch.equal(q, got[0]) and torch.equal(k, got[1])


@pytest.mark.parametrize("quantised", [False, True])
def test_append_of_many_turned_rows(smoe, quantised):
    """Prompts turned as they are written, several rounds a wavefront: the stored rows and the queries are those of the same calls in small parts."""
    B, h, G, d, page = 5, 4, 3, 128, 64
    lens = [3001, 17, 4096, 1500, 900]
    M = sum(lens)
    assert _rounds(M, G * h + 2 * h, d) == 5
    _log(f"append of many turned rows e4m3={quantised}")
    table, pages = _table(lens, page, 471)
    K, V, Q = (_normal(s, 472 + i).cuda() for i, s in enumerate(((M, h, d), (M, h, d), (M, G, h, d))))
    seqs = torch.tensor([b for b, n in enumerate(lens) for _ in range(n)], dtype=torch.int32).cuda()
    pos = torch.tensor([p for n in lens for p in range(n)], dtype=torch.int32).cuda()
    rotary = smoe.rotary_table(d)
    caches = [smoe.kv_cache(pages, page, h, d, quantised) for _ in range(2)]
    q = smoe.cache_append(caches[0], K, V, table.cuda(), seqs=seqs, positions=pos, rotary=rotary, Q=Q)
    for i in range(0, M, 1000):
        part = slice(i, i + 1000)
        assert _rounds(len(K[part]), G * h + 2 * h, d) == 1
        few = smoe.cache_append(caches[1], K[part], V[part], table.cuda(), seqs=seqs[part], positions=pos[part], rotary=rotary, Q=Q[part])
        assert torch.equal(few, q[part])
    for a, b in zip(*([t for t in (c.K, c.V, c.K_exp, c.V_exp) if t is not None] for c in caches)):
        rows = [t.view(torch.uint8).transpose(1, 2)[table.cuda()[seqs.long(), (pos // page).long()].long(), (pos % page).long()] for t in (a, b)]
        assert torch.equal(*rows)


@pytest.mark.parametrize("h,d,tokens,quantised", [(8, 128, 34001, False), (8, 128, 67003, True), (16, 64, 34001, False), (16, 64, 67003, True), (8, 128, 17001, False)])
def test_round_trip_past_the_caches(smoe, h, d, tokens, quantised):
    """More than half the last-level cache written, more than a quarter of it read: the same rows, bit for bit, at places in no order."""
    written, rows = tokens * h * d * (2 if quantised else 4), tokens * h * d * 4
    assert rows > LAST_LEVEL_CACHE // 4 and (written > LAST_LEVEL_CACHE // 2 or tokens == 17001)
    _log(f"round trip h={h} d={d} tokens={tokens} e4m3={quantised}")
    page = 64
    lens = [tokens - 5000, 4990, 10]
    table, pages = _table(lens, page, 481)
    gen = torch.Generator("cuda").manual_seed(482)
    K, V = (torch.randn(tokens, h, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    mix = torch.randperm(tokens, generator=_gen(483)).cuda()
    seqs = torch.tensor([b for b, n in enumerate(lens) for _ in range(n)], dtype=torch.int32).cuda()[mix]
    pos = torch.tensor([p for n in lens for p in range(n)], dtype=torch.int32).cuda()[mix]
    cache = smoe.kv_cache(pages, page, h, d, quantised)
    smoe.cache_append(cache, K, V, table.cuda(), seqs=seqs, positions=pos)
    k, v = smoe.cache_read(cache, table.cuda(), seqs=seqs, positions=pos)
    if not quantised:
        assert torch.equal(k, K) and torch.equal(v, V)
        return
    few = smoe.kv_cache(pages, page, h, d, True)
    for i in range(0, tokens, 8000):                # through the caches
        part = slice(i, i + 8000)
        smoe.cache_append(few, K[part], V[part], table.cuda(), seqs=seqs[part], positions=pos[part])
        back = smoe.cache_read(few, table.cuda(), seqs=seqs[part], positions=pos[part])
        assert torch.equal(k[part], back[0]) and torch.equal(v[part], back[1])
    for x, y in ((K, k), (V, v)):                   # and within half a step of the rows: 2^-4, or 2^-10 at a scale of at most max / 224
        x, y = x.double(), y.double()
        assert bool(((y - x).abs() <= 2.0 ** -4 * x.abs() + 2.0 ** -10 / 224 * x.abs().amax(-1, keepdim=True)).all())
