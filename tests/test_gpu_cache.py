"""Rotary positions, the paged key-value cache, attention over it and the layer's decoding pass, against the fp64 oracle."""
import sys

import numpy as np
import pytest
import torch

import oracle
import smoe_inputs as si
from helpers import TOL

pytestmark = pytest.mark.gpu

HALF_STEP = 2.0 ** -8        # a rounding to bf16 is off by at most this, relative to the value


def _log(*a):
    print(*a, flush=True, file=sys.stderr)


@pytest.fixture(scope="module")
def smoe():
    import paper_2403_08245_amd as m
    return m


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _normal(shape, seed, dtype=torch.bfloat16, std=1.0):
    return (torch.randn(*shape, generator=_gen(seed), dtype=torch.float32) * std).to(dtype)


def _f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


# ------------------------------------------------------------------------------------------------------------- rotary
# What fp32 costs a turned element, times (|a| + |b|) m: the angle is cut to 2^-32 turns (1.5e-9 radians) and rounded to 24 bits of a half
# turn (2^-25 * pi = 9.4e-8), sine and cosine are good to 4 units of 2^-24 (2.4e-7), and the amplitude, its product and the two
# products and sum round five times (3e-7).
TURN = 6.4e-7


def _turn_tolerance(x, want, rot, interleaved, amplitude, dtype):
    a = np.abs(_f64(x))
    pairs = a.copy()
    n = rot // 2
    if interleaved:
        s = a[..., 0:rot:2] + a[..., 1:rot:2]
        pairs[..., 0:rot:2], pairs[..., 1:rot:2] = s, s
    else:
        s = a[..., :n] + a[..., n:rot]
        pairs[..., :n], pairs[..., n:rot] = s, s
    pairs[..., rot:] = 0
    fp32 = TURN * amplitude * pairs
    return fp32 if dtype == torch.float32 else fp32 * (1 + HALF_STEP) + HALF_STEP * np.abs(want) * (pairs > 0)


ROTARY = [  # B, T, G, h, d, rot
    (1, 1, 1, 1, 8, 2), (2, 5, 4, 4, 128, 128), (3, 33, 3, 2, 64, 32), (1, 7, 1, 3, 72, 20), (1, 3, 5, 1, 96, 96), (2, 2, 2, 1, 256, 130), (1, 2, 1, 1, 512, 512),
    (1, 9, 8, 5, 128, 16), (1, 4, 16, 8, 16, 6),
]


@pytest.mark.parametrize("B,T,G,h,d,rot", ROTARY)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_and_its_gradient(smoe, B, T, G, h, d, rot, dtype, layout):
    _log(f"rotary {(B, T, G, h, d, rot)} {dtype} {layout}")
    scaling, factor = (("none", 1.0), ("blend", 8.0), ("linear", 3.7))[(T + d) % 3]
    table = smoe.rotary_table(rot, layout=layout, scaling=scaling, factor=factor, trained_length=2048.0)
    freqs, amp = oracle.rotary_frequencies(rot, scaling=scaling, factor=factor, trained_length=2048.0)
    Q, K = _normal((B, T, G, h, d), 1, dtype), _normal((B, T, h, d), 2, dtype)
    given = torch.randint(0, 200000, (B, T), generator=_gen(3), dtype=torch.int32)
    given[0, 0] = -3
    for positions in (None, given):
        at = torch.arange(T, dtype=torch.int32).repeat(B) if positions is None else positions.reshape(-1)
        pos = None if positions is None else positions.cuda()
        for entry, back in ((smoe.rotary_fwd, False), (smoe.rotary_bwd, True)):
            got = entry(Q.cuda(), K.cuda(), table, pos)
            for x, y in zip((Q, K), got):
                want = oracle.rotate_rows(_f64(x).reshape(B * T, -1, d), at.numpy(), freqs, amp, layout == "interleaved", back).reshape(x.shape)
                err, tol = np.abs(_f64(y) - want), _turn_tolerance(x, want, rot, layout == "interleaved", amp, dtype)
                assert y.shape == x.shape and (err <= tol).all(), (back, float(np.max(err - tol)))
                assert torch.equal(y.cpu()[..., rot:], x[..., rot:])


def test_rotary_extreme_positions(smoe):
    """Every position int32 holds has its exact angle: the oracle's own angle, in 64 bits, is off by up to 2^31 * 2^-52 radians there."""
    at = torch.tensor([[0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 12345, 1000003]], dtype=torch.int32)
    x = _normal((1, 7, 2, 64), 5, torch.float32)
    table = smoe.rotary_table(64)
    freqs, amp = oracle.rotary_frequencies(64)
    want = oracle.rotate_rows(_f64(x)[0], at.numpy(), freqs, amp)[None]
    y, none = smoe.rotary_fwd(x.cuda(), None, table, at.cuda())
    assert none is None and (np.abs(_f64(y) - want) <= _turn_tolerance(x, want, 64, False, 1.0, torch.float32) + 1e-6 * np.abs(_f64(x)).max()).all()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,rot", [(128, 128), (72, 20), (512, 260)])
def test_rotary_in_place_is_the_same(smoe, layout, d, rot):
    table = smoe.rotary_table(rot, layout=layout)
    Q, K = _normal((2, 9, 7, d), 7).cuda(), _normal((2, 9, 3, d), 8).cuda()
    want = smoe.rotary_fwd(Q, K, table)
    q, k = Q.clone(), K.clone()
    got = smoe.rotary_fwd(q, k, table, out=(q, k))
    assert got[0] is q and torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_rotary_copies_what_it_does_not_turn_bit_by_bit(smoe):
    """Infinities and NaN behind the turned part stay what they are, and do not reach it."""
    x = _normal((1, 3, 2, 32), 9)
    x[..., 16:] = float("inf")
    x[..., 20] = float("nan")
    for layout in ("half", "interleaved"):
        y, _ = smoe.rotary_fwd(x.cuda(), None, smoe.rotary_table(16, layout=layout))
        assert torch.equal(y.cpu()[..., 16:].view(torch.int16), x[..., 16:].view(torch.int16)) and bool(y[..., :16].isfinite().all())


def test_rotary_of_no_rows_and_refusals(smoe):
    table = smoe.rotary_table(64)
    q, _ = smoe.rotary_fwd(torch.empty(0, 5, 2, 64, dtype=torch.bfloat16, device="cuda"), None, table)
    assert q.shape == (0, 5, 2, 64)
    x = _normal((2, 3, 2, 64), 1).cuda()
    for bad in (lambda: smoe.rotary_fwd(x.transpose(0, 1), None, table), lambda: smoe.rotary_fwd(x, x[:1], table), lambda: smoe.rotary_fwd(x.cpu(), None, table),
                lambda: smoe.rotary_fwd(x, None, table, torch.zeros(5, dtype=torch.int32, device="cuda")), lambda: smoe.rotary_fwd(x, None, table, out=(x, x))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: smoe.rotary_fwd(x.half(), None, table), lambda: smoe.rotary_fwd(x, x.float(), table), lambda: smoe.rotary_fwd(x, None, table, torch.zeros(2, 3, device="cuda"))):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(smoe.SmoeError):
        smoe.rotary_fwd(x, x.clone(), table, out=(x, x))          # Q's result over K's
    with pytest.raises(smoe.SmoeError):
        smoe.rotary_fwd(torch.zeros(1, 1, 1, 60, dtype=torch.bfloat16, device="cuda"), None, smoe.rotary_table(4))


# ----------------------------------------------------------------------------------------------------- writing and reading
def _table(lens, page, seed, spare=2, width=None, behind=None):
    """A page table with the pages in no order, and how many pages there are; what lies behind a sequence's pages is `behind`."""
    need = [-(-max(int(n), 0) // page) for n in lens]
    total = sum(need) + spare
    order = torch.randperm(total, generator=_gen(seed)).to(torch.int32)
    w = max(max(need), 1) if width is None else width
    table = torch.full((len(lens), w), 0 if behind is None else behind, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, total


def _stored(cache):
    """The values a cache holds, in fp64."""
    if cache.K_exp is None:
        return _f64(cache.K), _f64(cache.V)
    value = oracle.e4m3_values()
    return tuple(value[x.cpu().numpy()] * 2.0 ** (e.cpu().numpy().astype(np.float64)[..., None] - 127) for x, e in ((cache.K, cache.K_exp), (cache.V, cache.V_exp)))


def _difficult_rows(M, h, d, seed):
    """Rows of every kind a quantiser meets."""
    x = _normal((M, h, d), seed)
    kinds = [lambda r: r.zero_(), lambda r: r.mul_(2.0 ** -120), lambda r: r.mul_(1e30), lambda r: r.clamp_(-1, 1).__setitem__(3, 448.0), lambda r: r.__setitem__(0, 450.0),
             lambda r: r.__setitem__(d - 1, float("inf")), lambda r: r.__setitem__(5, float("nan")), lambda r: r.fill_(float("-inf")), lambda r: r.__setitem__(7, 0.001),
             lambda r: r.copy_(torch.arange(d) - d // 2), lambda r: r.fill_(2.0 ** -133), lambda r: r.copy_(torch.linspace(15.5, 20.5, d))]
    for i, kind in enumerate(kinds):
        if i < M * h:
            kind(x.view(M * h, d)[i])
    return x


@pytest.mark.parametrize("page,h,d", [(16, 1, 128), (64, 3, 64), (256, 2, 128), (16, 5, 64)])
@pytest.mark.parametrize("quantised", [False, True])
def test_append_and_read_listed_places(smoe, page, h, d, quantised):
    """Exact in both formats: bf16 rows as they are, e4m3 codes and exponents as the table says, other places untouched, padding left
    out and read as zeros, values back exactly."""
    _log(f"append/read page={page} h={h} d={d} e4m3={quantised}")
    lens = [page + 3, 1, 2 * page, 0, 5]
    table, pages = _table(lens, page, 11, behind=10 ** 6)
    seqs = torch.tensor([b for b, n in enumerate(lens) for _ in range(n)], dtype=torch.int32)
    pos = torch.tensor([p for n in lens for p in range(n)], dtype=torch.int32)
    mix = torch.randperm(len(seqs), generator=_gen(12))
    seqs, pos = seqs[mix], pos[mix]
    bad = torch.tensor([[-1, 0], [5, 0], [0, -1], [0, 2 ** 31 - 1], [3, 0], [1, page], [2, 2 * page]], dtype=torch.int32)       # none of these has a place
    seqs, pos = torch.cat([bad[:3, 0], seqs, bad[3:, 0]]), torch.cat([bad[:3, 1], pos, bad[3:, 1]])
    good = slice(3, 3 + sum(lens))
    M = len(seqs)
    K, V = _difficult_rows(M, h, d, 13), _normal((M, h, d), 14)
    cache = smoe.kv_cache(pages, page, h, d, quantised)
    before = [t.clone() for t in (cache.K, cache.V)]
    where = dict(seqs=seqs.cuda(), positions=pos.cuda())
    assert smoe.cache_append(cache, K.cuda(), V.cuda(), table.cuda(), **where) is None
    written = torch.zeros(pages, page, dtype=torch.bool)
    ids = table[seqs[good].long(), (pos[good] // page).long()].long()
    slot = (pos[good] % page).long()
    written[ids, slot] = True
    assert int(written.sum()) == sum(lens)
    for stored, exps, old, x in ((cache.K, cache.K_exp, before[0], K), (cache.V, cache.V_exp, before[1], V)):
        got = stored.cpu()
        untouched = ~written[:, None, :].expand(pages, h, page)
        assert torch.equal(got.view(torch.uint8).view(pages, h, page, -1)[untouched], old.cpu().view(torch.uint8).view(pages, h, page, -1)[untouched])
        rows = got[ids, :, slot]
        if not quantised:
            assert torch.equal(rows.view(torch.int16), x[good].view(torch.int16))
            continue
        want = [oracle.e4m3_encode(r) for r in _f64(x[good]).reshape(-1, d)]
        codes = torch.from_numpy(np.stack([w[0] for w in want])).view(-1, h, d)
        nan = (codes & 127) == 127
        assert torch.equal(rows[~nan], codes[~nan]) and bool(((rows & 127) == 127)[nan].all())
        assert exps.cpu()[ids, :, slot].reshape(-1).tolist() == [w[1] + 127 for w in want]
    k, v = smoe.cache_read(cache, table.cuda(), **where)
    for got, held in zip((k, v), _stored(cache)):
        got = _f64(got)
        assert np.array_equal(got[good], held[ids.numpy(), :, slot.numpy()], equal_nan=True)
        assert not got[:3].any() and not got[good.stop:].any()


@pytest.mark.parametrize("quantised", [False, True])
@pytest.mark.parametrize("N,rot,layout", [(1, 128, "half"), (3, 64, "half"), (2, 20, "half"), (2, 128, "interleaved"), (1, 0, "half")])
def test_append_last_places_and_turn(smoe, quantised, N, rot, layout):
    """The last N positions of every sequence, keys and queries turned: a stored key is off by the turn's fp32 error and one rounding."""
    _log(f"append last N={N} rot={rot} {layout} e4m3={quantised}")
    page, h, d, G = 16, 2, 128, 3
    lens = torch.tensor([N, 40, 1, 0, 17, 64], dtype=torch.int32)
    B = len(lens)
    table, pages = _table(lens, page, 21)
    K, V, Q = _normal((B * N, h, d), 22), _normal((B * N, h, d), 23), _normal((B * N, G, h, d), 24)
    at = (lens[:, None] - N + torch.arange(N)).reshape(-1)
    cache = smoe.kv_cache(pages, page, h, d, quantised)
    rotate = {}
    wantK, wantQ = _f64(K), None
    if rot:
        rotate = dict(rotary=smoe.rotary_table(rot, layout=layout), Q=Q.cuda())
        freqs, _ = oracle.rotary_frequencies(rot)
        wantK = oracle.rotate_rows(wantK, at.numpy(), freqs, interleaved=layout == "interleaved")
        wantQ = oracle.rotate_rows(_f64(Q).reshape(B * N, -1, d), at.numpy(), freqs, interleaved=layout == "interleaved").reshape(Q.shape)
    q = smoe.cache_append(cache, K.cuda(), V.cuda(), table.cuda(), lens=lens.cuda(), **rotate)
    if rot:
        assert (np.abs(_f64(q) - wantQ) <= _turn_tolerance(Q, wantQ, rot, layout == "interleaved", 1.0, torch.bfloat16)).all()
        again = rotate["Q"].clone()
        assert smoe.cache_append(cache, K.cuda(), V.cuda(), table.cuda(), lens=lens.cuda(), rotary=rotate["rotary"], Q=again, out=again) is again and torch.equal(again, q)
    else:
        assert q is None
    k, v = (_f64(t) for t in smoe.cache_read(cache, table.cuda(), lens=lens.cuda(), N=N))
    real = (at >= 0).numpy()
    assert not k[~real].any() and not v[~real].any()
    if not quantised:
        assert np.array_equal(v[real], _f64(V)[real])
        tol = _turn_tolerance(K, wantK, rot, layout == "interleaved", 1.0, torch.bfloat16) if rot else 0 * wantK
        assert (np.abs(k - wantK)[real] <= tol[real]).all()
    else:
        assert np.array_equal(v[real], np.stack([oracle.e4m3_values()[c] * 2.0 ** e for c, e in map(oracle.e4m3_encode, _f64(V)[real].reshape(-1, d))]).reshape(-1, h, d))
        # half a step of e4m3, 2^-4 relative, or half of its smallest step at the row's scale (amax / 448 * 2, at most, times 2^-10)
        tol = 2.0 ** -4 * np.abs(wantK) + np.abs(wantK).max(-1, keepdims=True) / 224 * 2.0 ** -10 + TURN * 2 * np.abs(_f64(K)).max()
        assert (np.abs(k - wantK)[real] <= tol[real]).all()


@pytest.mark.parametrize("quantised", [False, True])
def test_append_turns_keys_alone(smoe, quantised):
    """Without queries the stored keys are the same bits as with them, and as those of listed places."""
    page, h, d = 16, 3, 64
    lens = torch.tensor([20, 7, 33], dtype=torch.int32)
    table, pages = _table(lens, page, 171)
    table, K, V, Q = table.cuda(), _normal((6, h, d), 172).cuda(), _normal((6, h, d), 173).cuda(), _normal((6, 5, d), 174).cuda()
    rotary = smoe.rotary_table(32, scaling="linear", factor=2.0)
    seqs = torch.tensor([0, 0, 1, 1, 2, 2], dtype=torch.int32)
    positions = (lens[seqs.long()] - 2 + torch.tensor([0, 1] * 3)).to(torch.int32)
    out = []
    for more in (dict(lens=lens.cuda(), Q=Q), dict(lens=lens.cuda()), dict(seqs=seqs.cuda(), positions=positions.cuda())):
        cache = smoe.kv_cache(pages, page, h, d, quantised)
        smoe.cache_append(cache, K, V, table, rotary=rotary, **more)
        out.append([t for t in (cache.K, cache.V, cache.K_exp, cache.V_exp) if t is not None])
    for a, b, c in zip(*out):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)) and torch.equal(a.view(torch.uint8), c.view(torch.uint8))


def test_append_leaves_out_bad_pages_and_reads_zeros(smoe):
    lens, page = torch.tensor([30, 20], dtype=torch.int32), 16
    table, pages = _table(lens, page, 31)
    table[0, 1], table[1, 0] = pages, -7
    K = _normal((2 * 20, 1, 64), 32)
    cache = smoe.kv_cache(pages, page, 1, 64)
    smoe.cache_append(cache, K.cuda(), K.cuda(), table.cuda(), lens=lens.cuda())
    k, v = smoe.cache_read(cache, table.cuda(), lens=lens.cuda(), N=20)
    k = k.cpu().view(2, 20, 64)
    K = K.view(2, 20, 64)
    assert torch.equal(k[0, :6], K[0, :6]) and not k[0, 6:].any()          # positions 10 .. 15 of sequence 0
    assert torch.equal(k[1, 16:], K[1, 16:]) and not k[1, :16].any()       # positions 16 .. 19 of sequence 1
    assert torch.equal(k.view(-1, 1, 64).cuda(), v)


def test_cache_offsets_past_32_bits(smoe):
    """A cache of 2^32 elements and more a tensor: the last pages are written, read and attended."""
    page, h, d = 256, 8, 128
    pages = 2 ** 32 // (page * h * d) + 5
    K, V = (torch.zeros(pages, h, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache = smoe.KVCache(K, V)
    lens = torch.tensor([page + 9], dtype=torch.int32).cuda()
    table = torch.tensor([[pages - 1, pages - 3]], dtype=torch.int32).cuda()
    k, v, q = _normal((page + 9, h, d), 41), _normal((page + 9, h, d), 42), _normal((1, 1, 2, h, d), 43)
    smoe.cache_append(cache, k.cuda(), v.cuda(), table, lens=lens)
    assert torch.equal(K[pages - 1].cpu(), k[:page].transpose(0, 1)) and torch.equal(K[pages - 3, :, :9].cpu(), k[page:].transpose(0, 1))
    back = smoe.cache_read(cache, table, lens=lens, N=page + 9)
    assert torch.equal(back[0].cpu(), k) and torch.equal(back[1].cpu(), v)
    O, L = smoe.cached_attention_fwd(q.cuda(), cache, table, lens)
    _check_attention(O, L, q, [_f64(k)], [_f64(v)], [page + 9])
    assert int((K.view(pages, -1).abs().amax(1) > 0).sum()) == 2


# ------------------------------------------------------------------------------------------------------------- attention
def _check_attention(O, L, Q, K, V, lens, visible=None):
    """Against the oracle.  A score is a sum of d products in fp32, off by (d + 2) 2^-24 sum |q k| / sqrt(d) =: e at most; the weights are
    rounded to bf16 and O once more, and the exponential and the sum of the weights are good to 2^-18 (the hardware's exp2 and log2, a few units of
    2^-23, of arguments that are rounded to 24 bits of at most 2^7: 2^-17 in the worst; scores here stay under 2^6).
    So |O - O*| <= 2^-8 |O*| + (2^-8 + 2 e + 2^-17) sum p |v|, |L - L*| <= e + 2^-17 + 2^-22 |L*|."""
    Oref, Lref = oracle.cached_attention(_f64(Q), K, V, lens, visible)
    absV = [np.abs(np.nan_to_num(v, posinf=0, neginf=0)) for v in V]
    weight, _ = oracle.cached_attention(_f64(Q), K, absV, lens, visible)
    B, N, G, h, d = Q.shape
    e = np.zeros(Q.shape[:-1])
    for b in range(B):
        n = max(0, min(int(lens[b]), K[b].shape[0]))
        if n:
            kk = np.nan_to_num(np.abs(K[b][:n]), posinf=0, neginf=0).max(0)           # [h, d]
            e[b] = (np.abs(_f64(Q[b])) * kk).sum(-1)
    e *= (d + 2) * 2.0 ** -24 / np.sqrt(d)
    O, L = _f64(O), _f64(L)
    tol = HALF_STEP * np.abs(Oref) + (HALF_STEP + 2 * e[..., None] + 2.0 ** -17) * weight + 1e-30
    err = np.abs(O - Oref)
    assert np.isfinite(O).all() and (err <= tol).all(), float(np.max(err / tol))
    empty = np.isneginf(Lref)
    assert np.array_equal(empty, np.isneginf(L))
    L, Lref, e = L[~empty], Lref[~empty], e[~empty]
    assert (np.abs(L - Lref) <= e + 2.0 ** -17 + 2.0 ** -22 * np.abs(Lref)).all()


def _case(smoe, lens, page, h, d, quantised, seed, width=None, behind=10 ** 6, std=1.0, width_extra=0):
    """A cache filled up to each sequence's length and holding NaN elsewhere: (cache, table, K, V as stored, per sequence)."""
    table, pages = _table(lens, page, seed, width=width, behind=behind)
    if width_extra:
        table = torch.cat([table, torch.full((len(lens), width_extra), behind, dtype=torch.int32)], 1)
    cache = smoe.kv_cache(pages, page, h, d, quantised)
    for t in (cache.K, cache.V):
        t.fill_(0x7F if quantised else float("nan"))
    for t in (cache.K_exp, cache.V_exp):
        if t is not None:
            t.fill_(255)
    seqs = torch.tensor([b for b, n in enumerate(lens) for _ in range(n)], dtype=torch.int32)
    pos = torch.tensor([p for n in lens for p in range(n)], dtype=torch.int32)
    K, V = _normal((len(seqs), h, d), seed + 1, std=std), _normal((len(seqs), h, d), seed + 2)
    if len(seqs):
        smoe.cache_append(cache, K.cuda(), V.cuda(), table.cuda(), seqs=seqs.cuda(), positions=pos.cuda())
        k, v = smoe.cache_read(cache, table.cuda(), seqs=seqs.cuda(), positions=pos.cuda())
    else:
        k, v = K, V
    split = lambda t: [x for x in np.split(_f64(t), np.cumsum(lens)[:-1])]
    return cache, table, split(k), split(v)


ATTEND = [  # lens, N, G, h, d, page
    ([1], 1, 1, 1, 128, 16), ([0], 1, 2, 1, 64, 16), ([15, 16, 17, 0, 1, 31, 32, 33], 1, 4, 2, 128, 16), ([63, 64, 65, 127, 128, 129], 1, 8, 1, 64, 32),
    ([5, 1, 0, 40, 2, 3], 3, 2, 3, 128, 16), ([1000, 3, 511, 513], 2, 5, 2, 128, 64), ([300, 299], 4, 8, 1, 64, 256), ([7, 260], 5, 16, 1, 128, 16),
    ([2049], 1, 16, 1, 128, 128), ([100, 90, 80], 7, 3, 1, 64, 16), ([33] * 70, 1, 1, 1, 128, 16), ([600, 20], 17, 2, 2, 128, 32),
]


@pytest.mark.parametrize("lens,N,G,h,d,page", ATTEND)
@pytest.mark.parametrize("quantised", [False, True])
def test_cached_attention(smoe, lens, N, G, h, d, page, quantised):
    """Lengths around every tile's and page's end, none at all, fewer than the new tokens; NaN in every place that is not written, and page
    numbers that do not exist behind the last page."""
    _log(f"cached attention lens={lens[:8]} N={N} G={G} h={h} d={d} page={page} e4m3={quantised}")
    cache, table, K, V = _case(smoe, lens, page, h, d, quantised, 51)
    Q = _normal((len(lens), N, G, h, d), 54)
    n = torch.tensor(lens, dtype=torch.int32).cuda()
    O, L = smoe.cached_attention_fwd(Q.cuda(), cache, table.cuda(), n)
    _check_attention(O, L, Q, K, V, lens)
    again = smoe.cached_attention_fwd(Q.cuda(), cache, table.cuda(), n)
    assert torch.equal(O, again[0]) and torch.equal(L, again[1])
    q = Q.cuda()
    over = smoe.cached_attention_fwd(q, cache, table.cuda(), n, out=(q, torch.empty_like(L)))
    assert torch.equal(over[0], O) and torch.equal(over[1], L)


@pytest.mark.parametrize("quantised", [False, True])
def test_cached_attention_long_and_ragged(smoe, quantised):
    """One long sequence among short ones: most of the keys belong to few (sequence, head) pairs."""
    lens = [9001, 3, 70, 0, 1200, 1] + [5] * 20
    _log(f"cached attention long e4m3={quantised}")
    cache, table, K, V = _case(smoe, lens, 16, 2, 128, quantised, 61, width_extra=40)
    Q = _normal((len(lens), 1, 4, 2, 128), 64)
    O, L = smoe.cached_attention_fwd(Q.cuda(), cache, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    _check_attention(O, L, Q, K, V, lens)


def test_cached_attention_long_pieces(smoe):
    """So many positions in all that a single wavefront walks more than 64 groups of 16 of them: 70 sequences that share 70001 positions' pages.
    Tolerance as in _check_attention."""
    n, B, G, d, page = 70001, 70, 2, 64, 16
    _log("cached attention long pieces")
    K, V = _normal((n, 1, d), 201).cuda(), _normal((n, 1, d), 202).cuda()
    pages = -(-n // page)
    table = torch.randperm(pages, generator=_gen(203)).to(torch.int32)[None].cuda()
    cache = smoe.kv_cache(pages, page, 1, d)
    smoe.cache_append(cache, K, V, table, seqs=torch.zeros(n, dtype=torch.int32).cuda(), positions=torch.arange(n, dtype=torch.int32).cuda())
    lens = torch.tensor([n - 13 * b for b in range(B)], dtype=torch.int32)
    Q = _normal((B, 1, G, 1, d), 204)
    O, L = smoe.cached_attention_fwd(Q.cuda(), cache, table.expand(B, -1).contiguous(), lens.cuda())
    k, v = K[:, 0].double(), V[:, 0].double()
    s = torch.matmul(Q.cuda().double().view(B * G, d), k.t().contiguous()) * d ** -0.5
    s.masked_fill_(torch.arange(n, device="cuda") >= lens.cuda().repeat_interleave(G)[:, None], -torch.inf)
    lse = torch.logsumexp(s, 1)
    w = torch.exp(s - lse[:, None])
    want, weight = torch.matmul(w, v), torch.matmul(w, v.abs())
    e = (d + 2) * 2.0 ** -24 * float((Q.cuda().double().view(B * G, d).abs() * k.abs().amax(0)).sum(1).max()) / d ** 0.5
    err = (O.double().view(B * G, d) - want).abs()
    assert bool((err <= HALF_STEP * want.abs() + (HALF_STEP + 2 * e + 2.0 ** -17) * weight).all())
    assert float((L.double().view(-1) - lse).abs().max()) <= e + 2.0 ** -17 + 2.0 ** -22 * float(lse.abs().max())


def test_cached_attention_large_batch(smoe):
    """More sequences than a wavefront has lanes or a block threads."""
    lens = [(i * 37) % 23 for i in range(1500)]
    _log("cached attention large batch")
    cache, table, K, V = _case(smoe, lens, 16, 1, 64, False, 71)
    Q = _normal((len(lens), 1, 2, 1, 64), 74)
    O, L = smoe.cached_attention_fwd(Q.cuda(), cache, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    _check_attention(O, L, Q, K, V, lens)


def test_cached_attention_lengths_and_pages_out_of_range(smoe):
    """Lengths past the table count as the table's, negative ones as none; positions on pages that do not exist are not seen."""
    lens = [48, 48, 48, 48]
    _log("cached attention bad lengths and pages")
    cache, table, K, V = _case(smoe, lens, 16, 1, 128, False, 81)
    Q = _normal((4, 1, 3, 1, 128), 84)
    told = torch.tensor([10 ** 6, -5, 48, 2 ** 31 - 1], dtype=torch.int32)
    table[2, 1] = cache.pages
    table[3] = -1
    visible = [[True] * 48, [], [t < 16 or t >= 32 for t in range(48)], [False] * 48]
    O, L = smoe.cached_attention_fwd(Q.cuda(), cache, table.cuda(), told.cuda())
    _check_attention(O, L, Q, K, V, [48, 0, 48, 48], visible)
    told = torch.tensor([-2 ** 31] * 4, dtype=torch.int32)
    O, L = smoe.cached_attention_fwd(Q.cuda(), cache, table.cuda(), told.cuda())
    assert not O.any() and bool((L == -np.inf).all())


@pytest.mark.parametrize("what", ["nan", "inf", "lowest"])
def test_cached_attention_hidden_positions_do_not_reach_a_query(smoe, what):
    """The newest tokens' rows hold NaN, infinities or the lowest values: the earlier queries of the same call do not see them."""
    _log(f"cached attention hidden {what}")
    lens, N = [37, 64, 4], 4
    cache, table, K, V = _case(smoe, lens, 16, 1, 128, False, 91)
    value = {"nan": float("nan"), "inf": float("inf"), "lowest": torch.finfo(torch.bfloat16).min}[what]
    for b, n in enumerate(lens):
        p = n - 1
        cache.K[table[b, p // 16], :, p % 16] = value
        cache.V[table[b, p // 16], :, p % 16] = value
    Q = _normal((3, N, 2, 1, 128), 94)
    O, L = smoe.cached_attention_fwd(Q.cuda(), cache, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    cut = [n - 1 for n in lens]
    _check_attention(O[:, :3].contiguous(), L[:, :3].contiguous(), Q[:, :3], K, V, cut)
    if what == "nan":
        assert bool(O[:, 3].isnan().all()) and bool(L[:, 3].isnan().all())       # who sees it has it


def test_cached_attention_scores_of_minus_infinity_and_extremes(smoe):
    """Keys whose scores are -infinity have no weight; a query that sees no others attends nothing.  A key whose score exceeds the
    others by more than the exponent's range holds takes all the weight, wherever it stands."""
    _log("cached attention extreme scores")
    lens = [40, 40, 200]
    cache, table, K, V = _case(smoe, lens, 16, 1, 64, False, 101)
    Q = torch.ones(3, 1, 2, 1, 64).bfloat16()
    put = lambda b, p, x: cache.K[table[b, p // 16], :, p % 16].fill_(x)
    for p in range(40):
        put(0, p, float("-inf"))
        if p != 7:
            put(1, p, float("-inf"))
    for p in range(200):
        put(2, p, -torch.finfo(torch.bfloat16).max / 64)
    put(2, 131, 40.0)
    O, L = smoe.cached_attention_fwd(Q.cuda(), cache, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    assert not O[0].any() and bool((L[0] == -np.inf).all())
    for b, p in ((1, 7), (2, 131)):
        want = torch.from_numpy(V[b][p, 0]).to(torch.bfloat16)
        assert torch.equal(O[b, 0, :, 0].cpu(), want.expand(2, 64))
    assert np.allclose(_f64(L[2]), 40.0 * 64 / 8)


@pytest.mark.parametrize("lens,N,G", [([40, 1, 700], 1, 2), ([40, 9, 700], 3, 2), ([40, 9, 700], 2, 12)])
def test_cached_attention_infinite_values_that_are_seen(smoe, lens, N, G):
    """An infinite value that a query sees makes that column infinite, of its sign, and no other column anything: every weight here is far
    from underflow (scores of normal rows differ by less than 2^6), so infinity times it is infinity, not NaN."""
    _log(f"cached attention infinite values {lens} N={N} G={G}")
    cache, table, K, V = _case(smoe, lens, 16, 1, 128, False, 191)
    for b in range(3):
        for p in range(0, lens[b] - N + 1, 5):           # positions that every query sees
            for column, x in ((3, float("inf")), (64, float("-inf"))):
                cache.V[table[b, p // 16], :, p % 16, column] = x
    Q = _normal((3, N, G, 1, 128), 194)
    O, L = smoe.cached_attention_fwd(Q.cuda(), cache, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    assert bool((O[..., 3] == float("inf")).all()) and bool((O[..., 64] == float("-inf")).all())
    O[..., 3], O[..., 64] = 0.0, 0.0                      # and the other columns are what they are without these two
    for v in V:
        v[..., 3], v[..., 64] = 0.0, 0.0
    _check_attention(O, L, Q, K, V, lens)


def test_cached_attention_refusals(smoe):
    cache = smoe.kv_cache(3, 16, 2, 64)
    table, lens = torch.zeros(2, 1, dtype=torch.int32).cuda(), torch.ones(2, dtype=torch.int32).cuda()
    Q = _normal((2, 1, 2, 2, 64), 1).cuda()
    for bad in (lambda: smoe.cached_attention_fwd(Q[:1], cache, table, lens), lambda: smoe.cached_attention_fwd(Q[..., :32].contiguous(), cache, table, lens),
                lambda: smoe.cached_attention_fwd(Q.transpose(2, 3), cache, table, lens), lambda: smoe.cached_attention_fwd(Q, cache, table, lens[:1]),
                lambda: smoe.cached_attention_fwd(Q, cache, table[0], lens), lambda: smoe.cached_attention_fwd(Q, cache, table.cpu(), lens),
                lambda: smoe.KVCache(cache.K, cache.V[:, :1].contiguous()), lambda: smoe.KVCache(cache.K.transpose(1, 2), cache.V.transpose(1, 2)),
                lambda: smoe.cache_append(cache, Q[:, 0, 0], Q[:, 0, 0], table, lens=lens, Q=Q), lambda: smoe.cache_append(cache, Q, Q, table),
                lambda: smoe.cache_append(cache, Q[:1, 0, 0], Q[:1, 0, 0], table, lens=lens), lambda: smoe.cache_read(cache, table, seqs=lens)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: smoe.cached_attention_fwd(Q.float(), cache, table, lens), lambda: smoe.cached_attention_fwd(Q, cache, table.long(), lens),
                lambda: smoe.cached_attention_fwd(Q, cache, table, lens.float()), lambda: smoe.KVCache(cache.K.float(), cache.V.float())):
        with pytest.raises(TypeError):
            bad()
    for page, d in ((24, 64), (8, 64), (16, 96)):
        with pytest.raises(smoe.SmoeError):
            smoe.cached_attention_fwd(_normal((2, 1, 2, 2, d), 1).cuda(), smoe.kv_cache(3, page, 2, d), table, lens)


# --------------------------------------------------------------------------------------------------------- as they are used
def _layer(d_model, E, h, seed, d=128):
    std = d_model ** -0.5
    return dict(W_K=_normal((d_model, h * d), seed, std=std).cuda(), W_V=_normal((d_model, h * d), seed + 1, std=std).cuda(),
                W_Q=_normal((E, d_model, h * d), seed + 2, std=std).cuda(), W_O=_normal((E, h * d, d_model), seed + 3, std=(h * d) ** -0.5).cuda())


@pytest.mark.parametrize("B,P,new,N,k,h,quantised", [(2, 21, 6, 1, 2, 2, False), (1, 40, 6, 3, 4, 1, False), (3, 0, 8, 2, 1, 2, False), (2, 50, 4, 1, 3, 1, True)])
def test_decoding_continues_the_layer(smoe, B, P, new, N, k, h, quantised):
    """A prompt through smoe_momha_fwd, its keys and values appended, then tokens by N at a time through momha_decode: the same outputs as
    the layer over the whole sequence."""
    _log(f"decode after prompt B={B} P={P} new={new} N={N} k={k} h={h} e4m3={quantised}")
    d_model, E, d, page, T = 256, 8, 128, 16, P + new
    w = _layer(d_model, E, h, 111)
    weights = (w["W_K"], w["W_V"], w["W_Q"], w["W_O"])
    X, logits = _normal((B, T, d_model), 115).cuda(), _normal((B, T, E), 116, torch.float32).cuda()
    route = lambda z: (lambda ei, g: (smoe.route(ei, E), g))(*smoe.topk_gate(z.reshape(-1, E).contiguous(), k))
    r, g = route(logits)
    whole, buf = smoe.momha_fwd(X.view(B * T, d_model), *weights, r, k, g, B, T, h, d)
    whole = _f64(whole).reshape(B, T, d_model)
    table, pages = _table([T] * B, page, 117)
    table, cache = table.cuda(), smoe.kv_cache(pages, page, h, d, quantised)
    lens = torch.full((B,), P, dtype=torch.int32).cuda()
    if P:
        cut = lambda t: t.view(B, T, h, d)[:, :P].reshape(B * P, h, d).contiguous()
        smoe.cache_append(cache, cut(buf.K), cut(buf.V), table, lens=lens)
    for t in range(P, T, N):
        lens += N
        x, z = X[:, t:t + N].reshape(B * N, d_model).contiguous(), logits[:, t:t + N]
        r, g = route(z)
        O = smoe.momha_decode(x, *weights, r, k, g, cache, table, lens)
        err = np.abs(_f64(O).reshape(B, N, -1) - whole[:, t:t + N]).max() / np.abs(whole).max()
        # both sides are within TOL of exact; e4m3 rows are off by up to 2^-4 (half a step) each, keys and values both
        assert err <= (2 * TOL[torch.bfloat16] if not quantised else 2.0 ** -3), (t, err)


@pytest.mark.parametrize("lens,N,d_model,E,k,h,d,rot,quantised", [
    ([40, 3, 17], 1, 256, 8, 2, 2, 128, 128, False), ([1], 1, 64, 4, 4, 1, 64, 0, False), ([9, 30], 2, 104, 4, 2, 1, 64, 20, False), ([25] * 70, 1, 128, 8, 2, 1, 64, 64, False),
    ([20] * 45, 3, 96, 4, 1, 2, 64, 0, False), ([50, 0, 1, 64, 33], 2, 2080, 4, 3, 3, 64, 64, True), ([30] * 20, 1, 160, 16, 8, 2, 128, 128, True),
    ([9] * 260, 2, 64, 4, 1, 1, 64, 64, False), ([21, 2, 40], 1, 96, 8, 3, 2, 64, 20, False), ([40, 7], 3, 64, 32, 8, 1, 128, 52, True)])
def test_decoding_layer_sizes(smoe, lens, N, d_model, E, k, h, d, rot, quantised):
    """The layer's decoding pass against the oracle's pieces: rows in one and several tiles, widths that fill a block of columns or not, contractions
    off the steps of 32, more rows than the small dense kernel takes, fewer positions than new tokens.  Tolerance: that of the layer's other
    tests, of the largest entry; for a cache in 8 bits another 2^-4, half a step of its values, and as much for the keys'."""
    _log(f"decode layer B={len(lens)} N={N} d_model={d_model} E={E} k={k} h={h} d={d} rot={rot} e4m3={quantised}")
    B, page = len(lens), 16
    M = B * N
    w = _layer(d_model, E, h, 211, d)
    before = [max(0, n - N) for n in lens]
    cache, table, K, V = _case(smoe, before, page, h, d, quantised, 215, width=-(-max(lens) // page) + 1, behind=0)
    need = [-(-n // page) for n in lens]
    pages = cache.pages
    # pages of their own for all positions, the old ones moved there
    fresh = smoe.kv_cache(sum(need) + 1, page, h, d, quantised)
    at, new_table = 0, torch.zeros_like(table)
    for b, n in enumerate(need):
        new_table[b, :n] = torch.arange(at, at + n)
        at += n
    seqs = torch.tensor([b for b, n in enumerate(before) for _ in range(n)], dtype=torch.int32)
    pos = torch.tensor([p for n in before for p in range(n)], dtype=torch.int32)
    if len(seqs):
        old = smoe.cache_read(cache, table.cuda(), seqs=seqs.cuda(), positions=pos.cuda())
        smoe.cache_append(fresh, *old, new_table.cuda(), seqs=seqs.cuda(), positions=pos.cuda())
    X, logits = _normal((M, d_model), 216), _normal((M, E), 217, torch.float32)
    ei, g = smoe.topk_gate(logits.cuda(), k)
    rotary = smoe.rotary_table(rot) if rot else None
    told = torch.tensor(lens, dtype=torch.int32)
    O = smoe.momha_decode(X.cuda(), w["W_K"], w["W_V"], w["W_Q"], w["W_O"], smoe.route(ei, E), k, g, fresh, new_table.cuda(), told.cuda(), rotary=rotary)
    oei, og = oracle.topk_gate(logits.numpy(), k)
    assert np.array_equal(ei.cpu().numpy(), oei)
    x, W = _f64(X), {n: _f64(t) for n, t in w.items()}
    newK, newV = (x @ W[n] for n in ("W_K", "W_V"))
    newQ = np.stack([[x[m] @ W["W_Q"][e] for e in oei[m]] for m in range(M)]).reshape(M, k * h, d)
    at = (told.long()[:, None] - N + torch.arange(N)).reshape(-1).numpy()
    newK = newK.reshape(M, h, d)
    if rot:
        freqs, _ = oracle.rotary_frequencies(rot)
        newK, newQ = oracle.rotate_rows(newK, at, freqs), oracle.rotate_rows(newQ, at, freqs)
    full = lambda old, new: [np.concatenate([old[b], new[b * N:(b + 1) * N][max(0, N - lens[b]):]]) for b in range(B)]
    att, _ = oracle.cached_attention(newQ.reshape(B, N, k, h, d), full(K, newK), full(V, newV.reshape(M, h, d)), lens)
    att = att.reshape(M, k, h * d)
    want = np.stack([sum(og[m, j] * (att[m, j] @ W["W_O"][e]) for j, e in enumerate(oei[m])) for m in range(M)])
    err = np.abs(_f64(O) - want).max() / np.abs(want).max()
    _log(f"  error {err:.2e}")
    assert err <= TOL[torch.bfloat16] + (2 * 2.0 ** -4 if quantised else 0)
    # the new rows are in the cache, the keys turned
    k_row, v_row = (_f64(t) for t in smoe.cache_read(fresh, new_table.cuda(), lens=told.cuda(), N=N))
    real = at >= 0
    for got, ref in ((k_row, newK), (v_row, newV.reshape(M, h, d))):
        # A projection may be rounded to bf16 before it is turned: a' = a cos w - b sin w is then off by 2^-8 (|a| + |b|), and
        # |a| + |b| <= sqrt(2) |(a, b)| = sqrt(2) |(a', b')| <= 2 max |a'| over the row.  What is stored is rounded once more, by half a step of
        # its type (2^-4 in e4m3, or half its smallest step, 2^-10 at a scale of at most max / 224).  Sums in fp32: 2^-15 of the largest.
        scale = np.abs(ref).max(-1, keepdims=True)
        tol = (2.0 ** -4 if quantised else HALF_STEP) * np.abs(ref) * (1 + HALF_STEP) + (2 * HALF_STEP + 2.0 ** -15) * scale + (2.0 ** -10 / 224 * scale if quantised else 0)
        assert (np.abs(got - ref)[real] <= tol[real]).all() and not got[~real].any()


def test_prefill_and_decoding_with_positions(smoe):
    """Rotary prefill (turn, causal attention, append), then tokens one by one (turn and append in one launch, attention over the cache),
    against the oracle's causal attention over turned rows of the whole sequence."""
    B, P, new, G, h, d, page = 2, 70, 5, 3, 2, 128, 32
    _log("prefill and decoding with positions")
    T = P + new
    Q, K, V = _normal((B, T, G, h, d), 121), _normal((B, T, h, d), 122), _normal((B, T, h, d), 123)
    table_r = smoe.rotary_table(d, scaling="blend", factor=4.0)
    freqs, amp = oracle.rotary_frequencies(d, scaling="blend", factor=4.0)
    at = np.tile(np.arange(T), B)
    turned = [oracle.rotate_rows(_f64(x).reshape(B * T, -1, d), at, freqs, amp).reshape(x.shape) for x in (Q, K)]
    want, _ = oracle.attention_fwd(*turned, _f64(V))
    table, pages = _table([T] * B, page, 124)
    cache, table = smoe.kv_cache(pages, page, h, d), table.cuda()
    part = lambda t, a, b: t[:, a:b].contiguous().cuda()
    q, k = smoe.rotary_fwd(part(Q, 0, P), part(K, 0, P), table_r)
    O, _ = smoe.attention_fwd(q, k, part(V, 0, P))
    err = lambda got, ref: np.abs(_f64(got) - ref).max() / np.abs(want).max()
    assert err(O, want[:, :P]) <= TOL[torch.bfloat16]
    lens = torch.full((B,), P, dtype=torch.int32).cuda()
    smoe.cache_append(cache, k.view(B * P, h, d), part(V, 0, P).view(B * P, h, d), table, lens=lens)
    for t in range(P, T):
        lens += 1
        q = smoe.cache_append(cache, part(K, t, t + 1)[:, 0], part(V, t, t + 1)[:, 0], table, lens=lens, rotary=table_r, Q=part(Q, t, t + 1))
        O, _ = smoe.cached_attention_fwd(q, cache, table, lens)
        assert err(O[:, 0], want[:, t]) <= TOL[torch.bfloat16], t


def test_decoding_step_replays_from_graphs(smoe):
    """A decoding step with positions captured once and replayed while lengths, table and inputs change in place, two captured graphs using
    one workspace in turn, with eager work between the replays: the same bits as the eager step."""
    _log("decode graph")
    B, N, k, h, d, d_model, E, page = 5, 1, 2, 2, 128, 256, 8, 16
    w = _layer(d_model, E, h, 131)
    weights = (w["W_K"], w["W_V"], w["W_Q"], w["W_O"])
    rotary = smoe.rotary_table(d)
    width = 12
    caches = [smoe.kv_cache(B * width, page, h, d) for _ in range(2)]
    for c in caches:
        c.K.normal_(generator=torch.Generator("cuda").manual_seed(1))
        c.V.normal_(generator=torch.Generator("cuda").manual_seed(2))
    table = torch.randperm(B * width, generator=_gen(132)).to(torch.int32).view(B, width).cuda()
    lens = torch.tensor([100, 7, 1, 64, 150], dtype=torch.int32).cuda()
    x, z = _normal((B, d_model), 133).cuda(), _normal((B, E), 134, torch.float32).cuda()
    ws = torch.empty(smoe.lib.smoe_momha_decode_workspace_bytes(B, N, k, d_model, h, d), dtype=torch.uint8, device="cuda")

    def step(cache):
        ei, g = smoe.topk_gate(z, k)
        return smoe.momha_decode(x, *weights, smoe.route(ei, E), k, g, cache, table, lens, rotary=rotary, ws=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs, outs = [], []
    with torch.cuda.stream(side):
        for c in caches:                    # warm-up outside the capture; it writes to the caches, so to both
            step(c)
    torch.cuda.synchronize()
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i], stream=side):
            outs.append(step(caches[i]))
    for seed in range(4):
        lens.copy_(torch.tensor([[101, 8, 2, 65, 151], [1, 192, 33, 0, 32], [17, 16, 15, 190, 3], [102, 9, 3, 66, 152]][seed], dtype=torch.int32))
        x.copy_(_normal((B, d_model), 140 + seed))
        z.copy_(_normal((B, E), 150 + seed, torch.float32))
        for i in range(2):
            graphs[i].replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        kept = [(c.K.clone(), c.V.clone()) for c in caches]
        for i in range(2):
            assert torch.equal(got[i], step(caches[i]))
            assert torch.equal(caches[i].K, kept[i][0]) and torch.equal(caches[i].V, kept[i][1])
        assert torch.equal(got[0], got[1])


def test_calls_on_another_stream(smoe):
    """Work goes to the current stream, in its order."""
    _log("another stream")
    lens = torch.tensor([200, 3], dtype=torch.int32).cuda()
    cache, table, K, V = _case(smoe, [200, 3], 16, 1, 128, False, 161)
    Q = _normal((2, 1, 4, 1, 128), 164)
    q = Q.cuda()
    want = smoe.cached_attention_fwd(q, cache, table.cuda(), lens)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    table = table.cuda()
    with torch.cuda.stream(side):
        late = torch.zeros_like(q)
        big = torch.zeros(1 << 26, device="cuda")
        for _ in range(20):
            big.add_(1.0)
        late.copy_(q)                       # behind the additions on this stream
        got = smoe.cached_attention_fwd(late, cache, table, lens)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
