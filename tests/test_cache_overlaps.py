"""Outputs and workspaces that lie over the cache's pages, or over what the same launch reads, are refused before anything is enqueued (CPU: the
addresses stand for device memory and are never followed)."""
import ctypes

import pytest

STEP = 1 << 20


@pytest.fixture(scope="module")
def world():
    """Entry points with every array at a place of its own, which a call moves; a call that is not refused fails here for want of a device."""
    import paper_2403_08245_amd as m
    keep = (ctypes.c_char * 65536)()
    ctx = ctypes.addressof(keep)
    at = {n: (i + 1) * STEP for i, n in enumerate("K V KE VE table lens turns X W Q O LSE ws rows vals gates routing".split())}
    ref = ctypes.byref
    bf16 = m.smoe_cache(at["K"], at["V"], None, None, 4, 16, 2, 64, 0)
    e4m3 = m.smoe_cache(at["K"], at["V"], at["KE"], at["VE"], 4, 16, 2, 64, 1)
    where = m.smoe_places(at["table"], 2, 100, None, None, at["lens"])            # 1600 positions: the attention wants its workspace
    rot = m.smoe_rotary(at["turns"], 64, 0, 1.0)
    routing = m.smoe_routing(at["routing"], at["routing"], at["routing"], 4, 4)
    lib, big = m.lib, 1 << 40

    def call(name, cache, **moved):
        a, c = at | moved, ref(cache)
        if name == "append":
            return lib.smoe_cache_append(ctx, None, 1, c, ref(where), a["rows"], a["vals"], 2, ref(rot), a["Q"], 4, a["O"])
        if name == "read":
            return lib.smoe_cache_read(ctx, None, 1, c, ref(where), 2, a["rows"], a["vals"])
        if name == "attend":
            return lib.smoe_cached_attention_fwd(ctx, None, 1, a["Q"], 1, 2, c, ref(where), a["O"], a["LSE"], a["ws"], big)
        return lib.smoe_momha_decode(ctx, None, 1, a["X"], 1, 64, a["W"], a["W"], a["W"], a["W"], ref(routing), 2, a["gates"], c, ref(where), ref(rot), a["O"], a["ws"], big)
    return call, at, {"bf16": bf16, "e4m3": e4m3}, keep


PAGES = {"K": 4 * 2 * 16 * 64, "V": 4 * 2 * 16 * 64, "KE": 4 * 2 * 16, "VE": 4 * 2 * 16}     # elements


@pytest.mark.parametrize("format", ["bf16", "e4m3"])
@pytest.mark.parametrize("name,outputs", [("append", ["O"]), ("read", ["rows", "vals"]), ("attend", ["O", "LSE", "ws"]), ("decode", ["O", "ws"])])
def test_outputs_over_the_pages(world, name, outputs, format):
    call, at, caches, _ = world
    for array, n in PAGES.items():
        if format == "bf16" and array in ("KE", "VE"):
            continue
        size = n * (2 if format == "bf16" else 1)
        for out in outputs:
            for place in (at[array], at[array] + (size - 1) // 256 * 256):          # its start; its last whole line
                moved = {out: place}
                if out == "ws":                                                     # large: the other arrays go out of its way
                    moved |= {x: y + (1 << 36) for x, y in at.items() if x not in PAGES and x != "ws"}
                assert call(name, caches[format], **moved) == -1, (array, moved)


def test_a_layers_workspace_and_output(world):
    call, at, caches, _ = world
    for moved in (dict(ws=at["X"]), dict(X=at["ws"] + 4096), dict(gates=at["ws"] + 4096), dict(O=at["ws"] + 4096), dict(O=at["gates"])):
        away = {x: y + (1 << 36) for x, y in at.items() if x in ("gates", "routing", "rows", "vals") and x not in moved} if "O" not in moved or moved["O"] != at["gates"] else {}
        assert call("decode", caches["bf16"], **(away | moved)) == -1, moved


def test_calls_whose_arrays_lie_apart_are_not_refused(world):
    """They reach the launch, which this machine cannot make: another error, or none where there is a device."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("the addresses are not of this device")
    call, at, caches, _ = world
    far = {x: y + (1 << 36) for x, y in at.items() if x in ("gates", "routing", "rows", "vals")}
    for name in ("append", "read", "attend", "decode"):
        assert call(name, caches["bf16"], **far) == -4, name
    assert call("decode", caches["bf16"], **(far | dict(O=at["X"]))) == -4           # X is read before O is written


def test_more_query_rows_than_a_launch_holds(world):
    """Up to 2^31 - 1 of them: refused, and no workspace asked for, where the count of their tiles would pass 32 bits, too."""
    import paper_2403_08245_amd as m
    _, at, caches, keep = world
    ref, ctx = ctypes.byref, ctypes.addressof(keep)
    one = m.smoe_cache(at["K"], at["V"], None, None, 4, 16, 1, 64, 0)
    where = m.smoe_places(at["table"], 1, 100, None, None, at["lens"])
    for N, G in ((2 ** 31 - 1, 1), (1, 2 ** 31 - 1), (2 ** 31 - 31, 1), (2 ** 30, 1), (32768, 65535)):
        assert m.lib.smoe_cached_attention_workspace_bytes(ref(one), ref(where), N, G) == 0, (N, G)
        assert m.lib.smoe_cached_attention_fwd(ctx, None, 1, 1 << 50, N, G, ref(one), ref(where), 1 << 51, 1 << 52, 1 << 53, 1 << 40) == -2, (N, G)
        assert m.lib.smoe_momha_decode_workspace_bytes(1, N, G, 64, 1, 64) == 0, (N, G)
    assert m.lib.smoe_cached_attention_workspace_bytes(ref(one), ref(where), 2 ** 20, 1) > 0


@pytest.mark.parametrize("format", ["bf16", "e4m3"])
def test_writing_to_a_cache_whose_arrays_share_memory(world, format):
    """Keys would be written over values.  (Attention and reads of such a cache are fine: one array for both, say.)"""
    import paper_2403_08245_amd as m
    call, at, caches, _ = world
    far = {x: y + (1 << 36) for x, y in at.items() if x in ("gates", "routing", "rows", "vals")}
    size = 4 * 2 * 16 * 64 * (2 if format == "bf16" else 1)
    pairs = [("V", "K", 0), ("V", "K", size - 16), ("K", "V", size - 16)]
    if format == "e4m3":
        pairs += [("V_exp", "K_exp", 0), ("K_exp", "V", 32), ("V_exp", "K", size - 16), ("K", "V_exp", 112)]
    for moved, onto, by in pairs:
        c = m.smoe_cache.from_buffer_copy(caches[format])
        setattr(c, moved, getattr(c, onto) + by)
        for name in ("append", "decode"):
            assert call(name, c, **far) == -1, (moved, onto, name)
