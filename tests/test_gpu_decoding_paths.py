"""The decoding pass of the attention layer where sequences are cut, where weights pass the caches, and where its projections meet the cache in bf16,
against 64 bits; what it keeps in fp32, by the error of its output; and a captured step whose cut changes between replays."""
import math
import sys

import pytest
import torch

import oracle
from helpers import TOL
from test_gpu_cache import _gen, _normal, _table

pytestmark = pytest.mark.gpu


def _log(*a):
    print(*a, flush=True, file=sys.stderr)


@pytest.fixture(scope="module")
def smoe():
    import paper_2403_08245_amd as m
    return m


class Step:
    """A layer, a cache filled up to each sequence's last N positions, and the inputs of one pass."""

    def __init__(self, m, lens, N, d_model, E, k, h, d, rot, quantised, seed=501, page=16, spare_columns=0):
        self.m, self.lens, self.N, self.E, self.k, self.h, self.d, self.page = m, lens, N, E, k, h, d, page
        gen = torch.Generator("cuda").manual_seed(seed)
        new = lambda *s, std=1.0: (torch.randn(*s, generator=gen, device="cuda") * std).bfloat16()
        B, do = len(lens), h * d
        self.W_K, self.W_V = (new(d_model, do, std=d_model ** -0.5) for _ in range(2))
        self.W_Q, self.W_O = new(E, d_model, do, std=d_model ** -0.5), new(E, do, d_model, std=do ** -0.5)
        self.X, self.logits = new(B * N, d_model), torch.randn(B * N, E, generator=gen, device="cuda")
        table, pages = _table(lens, page, seed + 1)
        self.table = torch.cat([table, torch.zeros(B, spare_columns, dtype=torch.int32)], 1).cuda()
        self.cache = m.kv_cache(pages, page, h, d, quantised)
        seqs = torch.tensor([b for b, n in enumerate(lens) for _ in range(n)], dtype=torch.int32).cuda()
        pos = torch.tensor([p for n in lens for p in range(n)], dtype=torch.int32).cuda()
        m.cache_append(self.cache, new(len(seqs), h, d), new(len(seqs), h, d), self.table, seqs=seqs, positions=pos)
        self.at = dict(seqs=seqs, positions=pos)
        self.told = torch.tensor(lens, dtype=torch.int32).cuda()
        self.rot, self.rotary = rot, m.rotary_table(rot) if rot else None

    def run(self, **more):
        idx, gates = self.m.topk_gate(self.logits, self.k)
        return self.m.momha_decode(self.X, self.W_K, self.W_V, self.W_Q, self.W_O, self.m.route(idx, self.E), self.k, gates, self.cache, self.table, self.told,
                                   rotary=self.rotary, **more)

    def shares(self):
        """Shares of the contraction of the key and value projections; 0 where they run as the other products."""
        M, K, N = self.X.shape[0], self.X.shape[1], self.h * self.d
        return max(1, min(-(-(K // 32) // 8), -(-256 // (2 * -(-N // 128) * -(-M // 64))))) if M <= 512 and K % 32 == 0 else 0

    def wide(self):
        """Are Q and the slots' outputs kept in fp32?  Where decoding kernels make them: a tile of 32 rows an expert or less."""
        return self.shares() > 0 and self.X.shape[0] * self.k <= 32 * self.E

    def exact(self):
        """The pass in 64 bits over the keys and values that the cache holds after it."""
        N, k, h, d = self.N, self.k, self.h, self.d
        X, M = self.X.double(), self.X.shape[0]
        order = torch.argsort(self.logits, dim=1, descending=True, stable=True)[:, :k]
        gates = torch.softmax(self.logits.double().gather(1, order), 1)
        K, V = (t.double() for t in self.m.cache_read(self.cache, self.table, **self.at))
        out, start = torch.zeros(M, self.X.shape[1], dtype=torch.float64, device="cuda"), 0
        used = {int(e): (self.W_Q[e].double(), self.W_O[e].double()) for e in order.unique().tolist()} if M * k <= 512 else None
        weight = lambda e, i: used[e][i] if used else (self.W_Q, self.W_O)[i][e].double()
        q = torch.zeros(M, k, h * d, dtype=torch.float64, device="cuda")
        for e in range(self.E):
            row, slot = (order == e).nonzero(as_tuple=True)
            if len(row):
                q[row, slot] = torch.matmul(X[row], weight(e, 0))
        q = q.view(M, k * h, d)
        if self.rot:
            pos = (self.told.long()[:, None] - N + torch.arange(N, device="cuda")).reshape(-1)
            f = torch.from_numpy(oracle.rotary_frequencies(self.rot)[0]).cuda()
            w, n = (pos.double()[:, None] * f)[:, None], self.rot // 2
            a, b = q[..., :n].clone(), q[..., n:self.rot].clone()
            q[..., :n], q[..., n:self.rot] = a * w.cos() - b * w.sin(), a * w.sin() + b * w.cos()
        q = q.view(len(self.lens), N, k, h, d)
        att = torch.zeros(M, k, h * d, dtype=torch.float64, device="cuda")
        for b, n in enumerate(self.lens):
            kk, vv = (t[start:start + n].transpose(0, 1).contiguous() for t in (K, V))           # [h, n, d]
            start += n
            s = torch.matmul(q[b].permute(2, 0, 1, 3).reshape(h, N * k, d), kk.transpose(1, 2).contiguous()) / math.sqrt(d)
            hidden = torch.arange(n, device="cuda")[None] > (n - N + torch.arange(N, device="cuda")).repeat_interleave(k)[:, None]
            o = torch.matmul(torch.softmax(s.masked_fill(hidden, -math.inf), -1), vv)
            att[b * N:(b + 1) * N] = o.view(h, N, k, d).permute(1, 2, 0, 3).reshape(N, k, h * d)
        for e in range(self.E):
            row, slot = (order == e).nonzero(as_tuple=True)
            if len(row):
                out.index_add_(0, row, gates[row, slot, None] * torch.matmul(att[row, slot], weight(e, 1)))
        return out

    def errors(self, O):
        """(largest error over the largest entry, root mean square of the error over that of the entries)"""
        want = self.exact()
        err = O.double() - want
        return float(err.abs().max() / want.abs().max()), float(err.norm() / want.norm())


# A rounding to bf16 is uniform over a step of 2^-7 times the power of two under the value, so 2^-7 / sqrt(12) * E[1/x^2]^(1/2) = 1.6e-3 in the root mean
# square over mantissas x spread evenly from 1 to 2 (E = 1/2), and roundings on the way add up in squares: the outputs of a linear map of rounded rows have
# their relative error.  Where the pass keeps Q, the shares of K and V and the slots' outputs in fp32 there are two, Ohat's and O's: 2.3e-3.  A third
# would make 2.8e-3; the line is the root of two and a half.
TWO_ROUNDINGS = 2.0 ** -7 / math.sqrt(12) / math.sqrt(2) * math.sqrt(2.5)


@pytest.mark.parametrize("lens,N,d_model,E,k,h,d,rot,quantised", [
    ([1500, 3, 700], 1, 512, 16, 4, 2, 128, 128, False), ([1500, 3, 700], 3, 512, 16, 8, 2, 128, 128, False), ([1500, 4, 700], 3, 512, 16, 8, 1, 64, 32, True),
    ([1500, 3, 700], 1, 512, 16, 2, 4, 64, 64, True), ([600] * 40, 1, 256, 32, 4, 2, 128, 0, False), ([2100, 900, 33, 1], 1, 1024, 8, 4, 4, 128, 128, False)])
def test_layer_over_sequences_that_are_cut(smoe, lens, N, d_model, E, k, h, d, rot, quantised):
    _log(f"layer over cut sequences {lens[:4]} N={N} d_model={d_model} E={E} k={k} h={h} d={d} rot={rot} e4m3={quantised}")
    s = Step(smoe, lens, N, d_model, E, k, h, d, rot, quantised)
    assert s.table.shape[1] * s.page > 512 and s.wide()
    O = s.run()
    most, rms = s.errors(O)
    _log(f"  largest {most:.2e} rms {rms:.2e}")
    assert most <= TOL[torch.bfloat16] and rms <= TWO_ROUNDINGS
    need = smoe.lib.smoe_momha_decode_workspace_bytes(len(lens), N, k, d_model, h, d)
    ws = smoe._new(need, dtype=torch.uint8, device="cuda")               # exactly as large as the query says
    assert torch.equal(s.run(ws=ws), O)
    with pytest.raises(smoe.SmoeError):
        s.run(ws=ws[:-256])
    x = s.X.clone()
    s.X = x
    assert torch.equal(s.run(out=x), O)                                  # O over X


def test_layer_whose_weights_pass_the_caches(smoe):
    """Projections of more than 256 MB in all, by the decoding kernels into fp32."""
    d_model, E, h, d = 4096, 64, 4, 128
    assert 2 * d_model * h * d * 2 * (E + 1) > 256 << 20
    _log("layer past the caches")
    for lens, k in (([700, 3, 90, 1], 8), ([(i * 53) % 700 + 1 for i in range(64)], 8)):
        s = Step(smoe, lens, 1, d_model, E, k, h, d, 128, False, seed=521)
        assert s.wide()
        most, rms = s.errors(s.run())
        _log(f"  largest {most:.2e} rms {rms:.2e}")
        assert most <= TOL[torch.bfloat16] and rms <= TWO_ROUNDINGS


@pytest.mark.parametrize("B,N,d_model,E,k,h,d,rot,quantised", [(128, 1, 256, 8, 4, 2, 64, 64, False), (128, 1, 256, 8, 4, 1, 128, 20, True), (45, 3, 96, 4, 1, 2, 64, 64, False),
                                                               (300, 2, 96, 4, 2, 1, 64, 64, False), (70, 1, 104, 4, 2, 2, 64, 64, True)])
def test_layer_of_more_rows_than_the_decoding_kernels_take(smoe, B, N, d_model, E, k, h, d, rot, quantised):
    """More than 32 rows an expert on average (queries in bf16, keys and values in shares), more than 512 rows, contractions off 32 (neither)."""
    lens = [(i * 29) % 60 + N for i in range(B)]
    _log(f"layer of many rows B={B} N={N} d_model={d_model} E={E} k={k} rot={rot} e4m3={quantised}")
    s = Step(smoe, lens, N, d_model, E, k, h, d, rot, quantised, seed=531)
    assert not s.wide() and (s.shares() > 0) == (B * N <= 512 and d_model % 32 == 0)
    most, rms = s.errors(s.run())
    _log(f"  largest {most:.2e} rms {rms:.2e}")
    assert most <= TOL[torch.bfloat16]


@pytest.mark.parametrize("quantised", [False, True])
def test_captured_step_whose_cut_changes(smoe, quantised):
    """A table of 2048 positions and lengths that are cut into other pieces at every replay, or into none; two captured graphs with one workspace in turn and
    eager work between: the bits of the eager step."""
    _log(f"captured step with cuts e4m3={quantised}")
    B, N, k, h, d, d_model, E, page, width = 5, 1, 4, 2, 128, 256, 8, 16, 128
    steps = [Step(smoe, [page * width] * B, N, d_model, E, k, h, d, 128, quantised, seed=541) for _ in range(2)]
    ws = torch.empty(smoe.lib.smoe_momha_decode_workspace_bytes(B, N, k, d_model, h, d), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for s in steps:
            s.run(ws=ws)
    torch.cuda.synchronize()
    graphs, outs = [torch.cuda.CUDAGraph() for _ in steps], []
    for g, s in zip(graphs, steps):
        with torch.cuda.graph(g, stream=side):
            outs.append(s.run(ws=ws))
    for i, lens in enumerate(([2048, 3, 700, 513, 1], [5, 4, 3, 2, 1], [512, 2000, 512, 512, 2048], [2047, 0, 1999, 1300, 640], [2048] * 5)):
        for s in steps:
            s.told.copy_(torch.tensor(lens, dtype=torch.int32))
            s.X.copy_(_normal((B, d_model), 550 + i))
            s.logits.copy_(torch.randn(B, E, generator=_gen(560 + i)))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        kept = [s.cache.K.clone() for s in steps]
        for s, o, c in zip(steps, got, kept):
            assert torch.equal(s.run(ws=ws), o), lens
            assert torch.equal(s.cache.K.view(torch.uint8), c.view(torch.uint8))
        assert torch.equal(*got)
