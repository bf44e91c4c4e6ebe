"""The binding's checks in front of the cache's and positions' entry points, with stand-ins for device tensors (CPU): what a call refuses never
reaches the library."""
import math

import pytest
import torch


class Tensor:
    """What the binding asks of a device tensor, without memory."""
    is_cuda = True

    def __init__(self, *shape, dtype=torch.bfloat16, device=0, contiguous=True):
        self.shape, self.dtype, self.index, self.contiguous = torch.Size(shape), dtype, device, contiguous

    device = property(lambda self: torch.device("cuda", self.index))
    get_device = lambda self: self.index
    is_contiguous = lambda self: self.contiguous
    numel = lambda self: math.prod(self.shape)
    dim = lambda self: len(self.shape)
    data_ptr = lambda self: 4096


def ints(*shape, **kw):
    return Tensor(*shape, dtype=torch.int32, **kw)


class Library:
    """Records the calls that would have been made."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append(name)
            return 512 if name.endswith("_workspace_bytes") else 0
        return call


@pytest.fixture
def smoe(monkeypatch):
    import paper_2403_08245_amd as m
    monkeypatch.setattr(m, "lib", Library())
    monkeypatch.setattr(m, "_new", lambda *shape, dtype, device: Tensor(*shape, dtype=dtype))
    monkeypatch.setattr(m, "_device", lambda first: 0)
    monkeypatch.setattr(m, "_where", lambda dev: (None, None))
    return m


def a_cache(m, h=2, d=64, quantised=False):
    t = torch.uint8 if quantised else torch.bfloat16
    exps = [Tensor(4, h, 16, dtype=torch.uint8) for _ in "KV"] if quantised else []
    return m.KVCache(Tensor(4, h, 16, d, dtype=t), Tensor(4, h, 16, d, dtype=t), *exps)


def a_table(m, device=0):
    return m.RotaryTable(Tensor(32, dtype=torch.int64, device=device), 64, False, 1.0)


@pytest.mark.parametrize("quantised", [False, True])
def test_what_a_cache_and_a_table_are_made_of_does_not_change(smoe, quantised):
    """The library's view of them holds the addresses they were made with: tensors put in later would leave it writing to the old ones."""
    cache, table = a_cache(smoe, quantised=quantised), a_table(smoe)
    for thing, names in ((cache, ("K", "V", "K_exp", "V_exp", "pages", "h", "page", "d_head", "device")), (table, ("turns", "rot", "interleaved", "amplitude"))):
        for name in names:
            before = getattr(thing, name)
            with pytest.raises(AttributeError):
                setattr(thing, name, Tensor(8, 2, 16, 64))
            with pytest.raises(AttributeError):
                delattr(thing, name)
            assert getattr(thing, name) is before


def test_append_to_a_table_of_no_sequences_is_refused(smoe):
    cache, rows = a_cache(smoe), Tensor(0, 2, 64)
    with pytest.raises(ValueError):
        smoe.cache_append(cache, rows, rows, ints(0, 3), lens=ints(0))
    with pytest.raises(ValueError):
        smoe.cache_append(cache, Tensor(4, 2, 64), Tensor(4, 2, 64), ints(0, 3), lens=ints(0))
    assert not smoe.lib.calls
    smoe.cache_append(cache, rows, rows, ints(2, 3), lens=ints(2))              # no rows of two sequences are fine
    assert smoe.lib.calls == ["smoe_cache_append"]


def a_layer(m, B=3, N=2, k=2, E=4, d_model=256, h=2, d=64, **other):
    """Arguments of momha_decode, some of them replaced."""
    args = dict(X=Tensor(B * N, d_model), W_K=Tensor(d_model, h * d), W_V=Tensor(d_model, h * d), W_Q=Tensor(E, d_model, h * d), W_O=Tensor(E, h * d, d_model),
                r=m.Routing(ints(B * N * k), ints(B * N * k), ints(E + 1), B * N * k, E), k=k, gates=Tensor(B * N, k, dtype=torch.float32), cache=a_cache(m, h, d),
                block_table=ints(B, 3), lens=ints(B), rotary=a_table(m))
    return m.momha_decode(**(args | other))


def test_decoding_takes_key_and_value_weights_as_they_are_laid_out(smoe):
    """A transposed matrix has as many elements, and would be read as another."""
    for bad in (dict(W_K=Tensor(128, 256)), dict(W_V=Tensor(128, 256)), dict(W_K=Tensor(256, 64)), dict(W_V=Tensor(255, 128))):
        with pytest.raises(ValueError):
            a_layer(smoe, **bad)
    assert not smoe.lib.calls
    a_layer(smoe)
    a_layer(smoe, W_K=Tensor(256, 2, 64), W_V=Tensor(256, 2, 64))               # the heads apart
    assert smoe.lib.calls.count("smoe_momha_decode") == 2


def test_rows_are_taken_as_they_are_laid_out(smoe):
    """Rows that end in [h, d_head] or [h * d_head]; the same number of elements in another order would be read as other rows."""
    cache, table, lens = a_cache(smoe), ints(3, 3), ints(3)
    good = [Tensor(6, 2, 64), Tensor(3, 2, 2, 64), Tensor(6, 128), Tensor(3, 2, 128)]
    bad = [Tensor(6, 64, 2), Tensor(2, 6, 64), Tensor(2, 3, 128, 1), Tensor(128, 6), Tensor(768), Tensor(12, 64)]
    for x in good:
        smoe.cache_append(cache, x, x, table, lens=lens)
        smoe.cache_append(cache, x, good[0], table, lens=lens)
        smoe.cache_read(cache, table, lens=lens, N=2, out=(x, x))
    made = len(smoe.lib.calls)
    assert made == 12
    for x in bad:
        for call in (lambda: smoe.cache_append(cache, x, good[0], table, lens=lens), lambda: smoe.cache_append(cache, good[0], x, table, lens=lens),
                     lambda: smoe.cache_read(cache, table, lens=lens, N=2, out=(x, good[0])), lambda: smoe.cache_read(cache, table, lens=lens, N=2, out=(good[0], x))):
            with pytest.raises(ValueError):
                call()
    assert len(smoe.lib.calls) == made


def test_decoding_takes_routing_of_the_current_device(smoe):
    """Its index arrays are read by the kernels as everything else is."""
    for i in range(3):
        arrays = [ints(12), ints(12), ints(5)]
        for wrong, error in ((ints(*arrays[i].shape, device=1), ValueError), (ints(*arrays[i].shape, contiguous=False), ValueError),
                             (Tensor(*arrays[i].shape, dtype=torch.int64), TypeError)):
            with pytest.raises(error):
                a_layer(smoe, r=smoe.Routing(*arrays[:i], wrong, *arrays[i + 1:], 12, 4))
    assert not smoe.lib.calls


def test_sizes_past_32_bits_are_refused(smoe):
    """The library counts rows and table entries in 32 bits: one that wrapped would turn, or look up, the wrong ones."""
    table, cache = a_table(smoe), a_cache(smoe)
    for shape in ((2, 2 ** 30, 1, 64), (2 ** 32 + 1, 1, 1, 64), (1, 2 ** 32 + 5, 1, 64), (1, 1, 2 ** 32 + 1, 64), (1, 1, 1, 2 ** 32 + 64)):
        for entry in (smoe.rotary_fwd, smoe.rotary_bwd):
            with pytest.raises(ValueError):
                entry(Tensor(*shape), None, table)
    with pytest.raises(ValueError):
        smoe.rotary_fwd(Tensor(1, 1, 1, 64), Tensor(1, 1, 2 ** 32 + 1, 64), table)
    one = Tensor(1, 2, 64)
    for block_table, lens in ((ints(1, 2 ** 32 + 1), ints(1)), (ints(2 ** 32 + 1, 1), ints(2 ** 32 + 1))):
        for call in (lambda: smoe.cache_append(cache, one, one, block_table, seqs=ints(1), positions=ints(1)), lambda: smoe.cache_read(cache, block_table, lens=lens),
                     lambda: smoe.cached_attention_fwd(Tensor(block_table.shape[0], 1, 1, 2, 64), cache, block_table, lens)):
            with pytest.raises(ValueError):
                call()
    assert not smoe.lib.calls
    smoe.rotary_fwd(Tensor(1, 2 ** 31 - 1, 1, 64), None, table)
    assert smoe.lib.calls == ["smoe_rotary_fwd"]
