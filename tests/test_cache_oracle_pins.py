"""Pins of the cache oracle, and the host arithmetic of the library that goes with it (CPU)."""
import ctypes
import math

import numpy as np
import pytest
import torch

import oracle


def test_rotation_hand_values_and_layouts():
    """A quarter turn of one pair, at a position that the frequency makes a quarter: (1, 2) -> (-2, 1)."""
    x = np.array([[[1.0, 2.0, 5.0]]])
    f = np.array([math.pi / 2])
    assert np.allclose(oracle.rotate_rows(x, [1], f), [[[-2.0, 1.0, 5.0]]])
    assert np.allclose(oracle.rotate_rows(x, [1], f, back=True), [[[2.0, -1.0, 5.0]]])
    y = np.arange(6.0).reshape(1, 1, 6)
    f = np.array([0.3, 0.7])
    half, inter = oracle.rotate_rows(y, [2], f), oracle.rotate_rows(y[:, :, [0, 2, 1, 3, 4, 5]], [2], f, interleaved=True)
    assert np.allclose(half[0, 0, [0, 2, 1, 3, 4, 5]], inter[0, 0])


def test_rotation_depends_on_the_distance_only_and_keeps_lengths():
    rng = np.random.default_rng(0)
    f, m = oracle.rotary_frequencies(8)
    q, k = rng.standard_normal((1, 1, 8)), rng.standard_normal((1, 1, 8))
    dots = [float(np.sum(oracle.rotate_rows(q, [p + 5], f) * oracle.rotate_rows(k, [p], f))) for p in (0, 17, 4000)]
    assert np.allclose(dots, dots[0]) and m == 1.0
    assert np.allclose(np.linalg.norm(oracle.rotate_rows(q, [123], f)), np.linalg.norm(q))


def test_rotation_gradient_against_differences():
    rng = np.random.default_rng(1)
    x, up = rng.standard_normal((2, 1, 10)), rng.standard_normal((2, 1, 10))
    f, m = oracle.rotary_frequencies(6, scaling="blend", factor=4.0, trained_length=64.0)
    for inter in (False, True):
        fwd = lambda y: float(np.sum(up * oracle.rotate_rows(y, [3, 40], f, m, inter)))
        grad = oracle.rotate_rows(up, [3, 40], f, m, inter, back=True)
        for i in np.ndindex(x.shape):
            step = np.zeros_like(x)
            step[i] = 1e-6
            assert abs((fwd(x + step) - fwd(x - step)) / 2e-6 - grad[i]) < 1e-7


def test_e4m3_table_matches_the_types_own_conversion():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    got = oracle.e4m3_values()
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~np.isnan(got)], want[~np.isnan(want)])


def test_e4m3_rows():
    codes, e = oracle.e4m3_encode([448.0, -1.0, 0.0, 17.0, 19.0])            # 17 and 19 lie between 16, 18 and 20: the even codes
    assert e == 0 and oracle.e4m3_values()[codes].tolist() == [448.0, -1.0, 0.0, 16.0, 20.0]
    codes, e = oracle.e4m3_encode([450.0, 1.0])                             # 450 / 2 = 225: between 224 and 240
    assert e == 1 and oracle.e4m3_values()[codes].tolist() == [224.0, 0.5]
    codes, e = oracle.e4m3_encode([math.inf, math.nan, 3.0])
    assert e == -7 and np.isnan(oracle.e4m3_values()[codes][:2]).all() and oracle.e4m3_values()[codes][2] == 384.0
    assert oracle.e4m3_encode([0.0, -0.0]) [1] == -126
    x = torch.randn(64, generator=torch.Generator().manual_seed(3)).double().numpy()
    codes, e = oracle.e4m3_encode(x)
    assert np.array_equal(codes, torch.tensor(x * 2.0 ** -e, dtype=torch.float32).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_cached_attention_is_the_causal_attention_of_the_last_rows():
    rng = np.random.default_rng(2)
    Q, K, V = rng.standard_normal((2, 9, 3, 2, 4)), rng.standard_normal((2, 9, 2, 4)), rng.standard_normal((2, 9, 2, 4))
    O, L = oracle.attention_fwd(Q, K, V)
    for lens, N in (([9, 6], 3), ([9, 2], 4)):
        q = np.stack([np.concatenate([np.zeros((max(0, N - n), 3, 2, 4)), Q[b, max(0, n - N):n]]) for b, n in enumerate(lens)])
        got, lse = oracle.cached_attention(q, K, V, lens)
        for b, n in enumerate(lens):
            m = min(n, N)
            assert np.allclose(got[b, N - m:], O[b, n - m:n]) and np.allclose(lse[b, N - m:], L[b, n - m:n])
            assert not got[b, :N - m].any() and np.isneginf(lse[b, :N - m]).all()


@pytest.mark.parametrize("rot,base,scaling,factor", [(2, 10000.0, "none", 1.0), (128, 10000.0, "none", 1.0), (64, 500000.0, "linear", 4.0), (2, 10000.0, "base", 8.0),
                                                     (128, 10000.0, "base", 8.0), (20, 10000.0, "blend", 3.7), (128, 1000000.0, "blend", 32.0)])
def test_library_frequencies(rot, base, scaling, factor):
    """Fractions of a turn times 2^64.  f and f / 2 pi are a few roundings of 2^-53 off (powers, products), so a few 2^-50 of them."""
    import paper_2403_08245_amd as m
    turns, amp = np.zeros(rot // 2, dtype=np.uint64), ctypes.c_float()
    rc = m.lib.smoe_rotary_frequencies(rot, base, m.ROTARY_SCALINGS[scaling], factor, 8192.0, turns.ctypes.data, ctypes.byref(amp))
    assert rc == 0
    f, a = oracle.rotary_frequencies(rot, base, scaling, factor, 8192.0)
    want = f / (2 * math.pi)
    assert (np.abs(turns.astype(np.float64) * 2.0 ** -64 - want) <= 2.0 ** -49 * want + 2.0 ** -63).all()
    assert amp.value == np.float32(a)


def test_library_frequencies_refusals():
    import paper_2403_08245_amd as m
    turns, amp = np.zeros(64, dtype=np.uint64), ctypes.c_float()
    call = lambda rot=8, base=1e4, scaling=0, factor=1.0, length=4096.0, t=turns.ctypes.data, a=ctypes.byref(amp): \
        m.lib.smoe_rotary_frequencies(rot, base, scaling, factor, length, t, a)
    assert call() == 0
    for bad in (dict(rot=0), dict(rot=7), dict(rot=-2), dict(base=1.0), dict(base=math.nan), dict(base=math.inf), dict(scaling=4), dict(scaling=-1), dict(factor=0.5),
                dict(factor=math.nan), dict(factor=math.inf), dict(scaling=3, length=0.0), dict(scaling=3, length=math.nan), dict(t=None), dict(a=None)):
        assert call(**bad) == -1, bad
    with pytest.raises(ValueError):
        m.rotary_table(8, layout="thirds", device="cpu")
    with pytest.raises(m.SmoeError):
        m.rotary_table(7, device="cpu")


# ------------------------------------------------------------------------------------------------ refusals of the entry points
class Args:
    """Keyword arguments of an entry point in order, with values that are accepted; a call replaces some of them."""

    def __init__(self, entry, **values):
        self.entry, self.values = entry, values

    def __call__(self, **other):
        assert set(other) <= set(self.values)
        return self.entry(*(self.values | other).values())


@pytest.fixture(scope="module")
def calls():
    """Entry points with a stand-in context and host addresses: every call here has to be refused before a launch.  (That the arguments
    are otherwise accepted shows in the calls with no rows, which succeed without one.)"""
    import paper_2403_08245_amd as m
    lib = m.lib
    keep = (ctypes.c_char * 65536)()
    mem = (ctypes.addressof(keep) + 255) & ~255
    ctx, a, b, c, d = mem, mem + 4096, mem + 8192, mem + 16384, mem + 24576
    cache = m.smoe_cache(a, b, None, None, 4, 16, 2, 64, 0)
    e4m3 = m.smoe_cache(a, b, c, d, 4, 16, 2, 64, 1)
    at = m.smoe_places(mem, 2, 3, None, None, mem)
    listed = m.smoe_places(mem, 2, 3, mem, mem, None)
    rot = m.smoe_rotary(mem, 64, 0, 1.0)
    routing = m.smoe_routing(mem, mem, mem, 4, 4)
    ref = ctypes.byref
    return dict(
        m=m, lib=lib, mem=mem, keep=keep, cache=cache, e4m3=e4m3, at=at, listed=listed, rot=rot, routing=routing,
        turn=Args(lib.smoe_rotary_fwd, ctx=ctx, stream=None, dtype=1, Q=a, hq=2, K=b, hk=1, rows=3, d=64, T=3, positions=None, rotary=ref(rot), Qr=c, Kr=d),
        back=Args(lib.smoe_rotary_bwd, ctx=ctx, stream=None, dtype=1, Q=a, hq=2, K=b, hk=1, rows=3, d=64, T=3, positions=None, rotary=ref(rot), Qr=c, Kr=d),
        append=Args(lib.smoe_cache_append, ctx=ctx, stream=None, dtype=1, cache=ref(cache), places=ref(at), K=a, V=b, rows=2, rotary=ref(rot), Q=c, hq=4, Qr=d),
        read=Args(lib.smoe_cache_read, ctx=ctx, stream=None, dtype=1, cache=ref(cache), places=ref(at), rows=2, K=a, V=b),
        attend=Args(lib.smoe_cached_attention_fwd, ctx=ctx, stream=None, dtype=1, Q=c, N=1, G=2, cache=ref(cache), places=ref(at), O=d, LSE=a, ws=mem, ws_bytes=1 << 40),
        decode=Args(lib.smoe_momha_decode, ctx=ctx, stream=None, dtype=1, X=a, N=1, d_model=64, W_K=a, W_V=a, W_Q=a, W_O=a, r=ref(routing), k=2, gates=a,
                    cache=ref(cache), places=ref(at), rotary=ref(rot), O=d, ws=mem, ws_bytes=1 << 40))


def _cache_with(c, base="cache", **fields):
    x = type(c[base]).from_buffer_copy(c[base])
    for k, v in fields.items():
        setattr(x, k, v)
    return ctypes.byref(x)


def test_refusals_of_rotary(calls):
    for f in (calls["turn"], calls["back"]):
        q = f.values["Q"]
        assert f(rows=0) == 0
        for bad in (dict(ctx=None), dict(dtype=7), dict(Q=None), dict(Qr=None), dict(hq=0), dict(hk=-1), dict(K=None), dict(Kr=None), dict(hk=0), dict(rows=-1), dict(T=0),
                    dict(d=0), dict(rotary=None), dict(Qr=q + 16), dict(Kr=q), dict(Qr=f.values["K"]), dict(Kr=f.values["Qr"])):
            assert f(**bad) == -1, bad
        for bad in (dict(d=68), dict(d=520), dict(Q=q + 2), dict(Qr=f.values["Qr"] + 8), dict(hq=70000)):
            assert f(**bad) == -2, bad
        for fields in (dict(turns=None), dict(rot=0), dict(rot=7), dict(rot=66), dict(interleaved=2), dict(amplitude=math.nan), dict(turns=calls["mem"] + 4)):
            assert f(rotary=_cache_with(calls, "rot", **fields)) == -1, fields
        assert f(rows=2 ** 31 - 1, hq=65535, d=512, hk=0, K=None, Kr=None, Qr=1 << 60) == -2     # more than one launch can hold


def test_refusals_of_the_cache(calls):
    for name in ("append", "read", "attend", "decode"):
        f = calls[name]
        for bad in (dict(ctx=None), dict(cache=None), dict(places=None)):
            assert f(**bad) == -1, (name, bad)
        assert f(dtype=0) == -2
        for fields in (dict(K=None), dict(V=None), dict(pages=0), dict(page=0), dict(h=0), dict(d_head=0), dict(format=2), dict(format=1), dict(K_exp=calls["mem"])):
            assert f(cache=_cache_with(calls, **fields)) == -1, (name, fields)
        for fields in (dict(V_exp=None), dict(K_exp=None), dict(format=0)):
            assert f(cache=_cache_with(calls, "e4m3", **fields)) == -1, (name, fields)
        for fields in (dict(page=8), dict(page=48), dict(page=131072), dict(d_head=32), dict(d_head=96), dict(d_head=256), dict(h=70000), dict(K=calls["mem"] + 8)):
            assert f(cache=_cache_with(calls, **fields)) == -2, (name, fields)
        for fields in (dict(block_table=None), dict(sequences=0), dict(width=0), dict(lens=None), dict(seqs=calls["mem"])):
            assert f(places=_cache_with(calls, "at", **fields)) == -1, (name, fields)
        assert f(places=_cache_with(calls, "at", width=2 ** 27)) == -2, name                      # positions past 31 bits
    for name in ("append", "read"):
        f = calls[name]
        assert f(rows=0) == 0 and f(rows=0, places=ctypes.byref(calls["listed"])) == 0
        for bad in (dict(rows=-1), dict(rows=3), dict(K=None), dict(V=None)):
            assert f(**bad) == -1, bad
        assert f(K=f.values["K"] + 2) == -2
        for fields in (dict(seqs=None), dict(positions=None)):
            assert f(places=_cache_with(calls, "listed", **fields)) == -1, fields
    f = calls["append"]
    q = f.values["Q"]
    for bad in (dict(Q=None), dict(Qr=None), dict(rotary=None), dict(hq=0), dict(Qr=q + 16), dict(Qr=f.values["K"]), dict(Qr=f.values["V"])):
        assert f(**bad) == -1, bad
    assert f(Q=q + 8) == -2 and f(hq=70000) == -2


def test_refusals_of_attention_and_layer(calls):
    f, q = calls["attend"], calls["attend"].values["Q"]
    for bad in (dict(Q=None), dict(O=None), dict(LSE=None), dict(N=0), dict(G=0), dict(O=q + 16), dict(places=ctypes.byref(calls["listed"]))):
        assert f(**bad) == -1, bad
    for bad in (dict(Q=q + 2), dict(O=f.values["O"] + 8), dict(N=2 ** 16, G=2 ** 16)):
        assert f(**bad) == -2, bad
    query = calls["lib"].smoe_cached_attention_workspace_bytes
    at = _cache_with(calls, "at", width=100)                      # 1600 positions: a sequence may be shared by blocks
    need = query(ctypes.byref(calls["cache"]), at, 1, 2)
    assert need > 0 and need % 256 == 0
    for bad in (dict(ws=None), dict(ws=calls["mem"] + 16), dict(ws_bytes=need - 1)):
        assert f(places=at, **bad) == -3, bad
    assert query(ctypes.byref(calls["cache"]), ctypes.byref(calls["at"]), 1, 2) == 0      # 48 positions: nothing to share
    for sizes in ((None, at, 1, 2), (ctypes.byref(calls["cache"]), None, 1, 2), (ctypes.byref(calls["cache"]), at, 0, 2), (ctypes.byref(calls["cache"]), at, 1, 0),
                  (_cache_with(calls, d_head=96), at, 1, 2), (ctypes.byref(calls["cache"]), at, 2 ** 16, 2 ** 16)):
        assert query(*sizes) == 0
    f = calls["decode"]
    for bad in (dict(X=None), dict(W_K=None), dict(W_V=None), dict(W_Q=None), dict(W_O=None), dict(r=None), dict(gates=None), dict(O=None), dict(N=0), dict(N=2), dict(k=0),
                dict(k=3), dict(d_model=0), dict(places=ctypes.byref(calls["listed"]))):
        assert f(**bad) == -1, bad
    for bad in (dict(d_model=68), dict(X=f.values["X"] + 2), dict(O=f.values["O"] + 2), dict(W_O=f.values["W_O"] + 8)):
        assert f(**bad) == -2, bad
    need = calls["lib"].smoe_momha_decode_workspace_bytes(2, 1, 2, 64, 2, 64)
    for bad in (dict(ws=None), dict(ws=calls["mem"] + 16), dict(ws_bytes=need - 1)):
        assert f(**bad) == -3, bad
    assert calls["lib"].smoe_momha_decode_workspace_bytes(2, 1, 2, 0, 2, 64) == 0


def test_header_and_export_list_agree(calls):
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "smoe_cache.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    assert sorted(set(re.findall(r"\b(smoe_[a-z0-9_]+)\s*\(", text))) == sorted(calls["m"].CACHE_EXPORTS)
    for name in calls["m"].CACHE_EXPORTS:
        assert hasattr(calls["lib"], name)


def test_refusals_of_outputs_that_overlap(calls):
    """One launch writes them all, or reads one while it writes another."""
    f = calls["read"]
    for bad in (dict(V=f.values["K"]), dict(V=f.values["K"] + 256), dict(K=f.values["V"] + 496)):       # two rows of two heads of 64: 512 bytes each
        assert f(**bad) == -1, bad
    f = calls["attend"]
    q, o = f.values["Q"], f.values["O"]
    for bad in (dict(LSE=q), dict(LSE=o), dict(LSE=o + 1020)):                                           # Q and O: 2 x 2 x 2 x 64 bf16 = 1024 bytes
        assert f(**bad) == -1, bad
    at = _cache_with(calls, "at", width=100)
    for bad in (dict(ws=q), dict(ws=o), dict(ws=f.values["LSE"])):
        assert f(places=at, **bad) == -1, bad
