"""What the block's entry points and their binding refuse (CPU: addresses stand for device memory and are never followed)."""
import ctypes
import math
import os
import re

import pytest
import torch

from test_cache_binding import Library, Tensor, ints

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3
STEP = 1 << 24


@pytest.fixture(scope="module")
def m():
    import paper_2403_08245_amd as m
    return m


def test_header_and_exports_agree(m):
    text = open(os.path.join(os.path.dirname(__file__), "..", "include", "smoe_block.h")).read()
    names = sorted(set(re.findall(r"\b(smoe_[a-z0-9_]+)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S))))
    assert sorted(m.BLOCK_EXPORTS) == names
    for n in names:
        assert hasattr(m.lib, n), n


@pytest.fixture(scope="module")
def call(m):
    """Calls an entry point with sound arguments, some of them replaced.  A call that nothing refuses would launch, so every call here has to be refused."""
    keep = (ctypes.c_char * 65536)()
    at = {n: (i + 1) * STEP for i, n in enumerate("x b i g dg dx R w S Y Yv Ye rstd dY dS dX dw ws Xv Xe W Wv We Vv Ve o off Yhat".split())}
    ref = ctypes.byref

    def rows(v, e):
        return ref(m.smoe_rows8(v, e))

    def go(name, **c):
        a = {**at, "ctx": ctypes.addressof(keep), "T": 4, "E": 8, "k": 2, "score": 1, "groups": 4, "kept": 2, "best": 2, "renorm": 1, "scale": 1.0, "dtype": 1, "rows": 4, "d": 256,
             "eps": 1e-6, "wsb": 1 << 20, "d_out": 64, "halves": 1, "x_rows": 4, "gates_k": 2, "gin": 0, "gout": 0, "act": 2, "d_model": 128, "d_expert": 64, "Tk": 8, **c}
        rule = None if a.get("norule") else ref(m.smoe_gate_rule(a["score"], a["groups"], a["kept"], a["best"], a["renorm"], a["scale"]))
        r = ref(m.smoe_routing(a["o"], a["o"], a["off"], a["Tk"], a["E"]))
        w = m.smoe_weights8(a["Wv"], a["We"], a.get("wE", a["E"]), a.get("w_in", a["d"]), a.get("w_out", a["d_out"]), a["halves"])
        lib = m.lib
        if name == "gate":
            return lib.smoe_score_gate(a["ctx"], None, a["x"], a["b"], a["T"], a["E"], a["k"], rule, a["i"], a["g"])
        if name == "gate_bwd":
            return lib.smoe_score_gate_bwd(a["ctx"], None, a["x"], a["i"], a["dg"], a["T"], a["E"], a["k"], rule, a["dx"])
        if name == "pack":
            return lib.smoe_rows8_pack(a["ctx"], None, a["dtype"], a["x"], a["rows"], a["d"], rows(a["Xv"], a["Xe"]))
        if name == "unpack":
            return lib.smoe_rows8_unpack(a["ctx"], None, a["dtype"], rows(a["Xv"], a["Xe"]), a["rows"], a["d"], a["x"])
        if name == "weights":
            return lib.smoe_weights8_pack(a["ctx"], None, a["dtype"], a["W"], ref(w))
        if name == "norm":
            return lib.smoe_add_norm_fwd(a["ctx"], None, a["dtype"], a["x"], a["R"], a["w"], a["rows"], a["d"], a["eps"], a["S"], a["Y"],
                                         rows(a["Yv"], a["Ye"]) if a["Yv"] else None, a["rstd"])
        if name == "norm_bwd":
            return lib.smoe_add_norm_bwd(a["ctx"], None, a["dtype"], a["dY"], a["dS"], a["S"], a["w"], a["rstd"], a["rows"], a["d"], a["dX"], a["dw"], a["ws"], a["wsb"])
        if name == "linear":
            return lib.smoe_plinear8_fwd(a["ctx"], None, rows(a["Xv"], a["Xe"]), a["x_rows"], a["d"], ref(w), a["d_out"], r, a["k"], a["g"], a["gates_k"], a["gin"], a["gout"], a["Yhat"], a["Y"])
        hidden = a["d_expert"] * (2 if a["act"] == 2 else 1)
        w1 = m.smoe_weights8(a["Wv"], a["We"], a.get("wE", a["E"]), a.get("w_in", a["d_model"]), a.get("w_out", hidden), a.get("w1_halves", 2 if a["act"] == 2 else 1))
        w2 = m.smoe_weights8(a["Vv"], a["Ve"], a["E"], a.get("v_in", a["d_expert"]), a["d_model"], a.get("v_halves", 1))
        return lib.smoe_mlp8_fwd(a["ctx"], None, a["act"], rows(a["Xv"], a["Xe"]), a["T"], a["d_model"], a["d_expert"], ref(w1), ref(w2), r, a["k"], a["g"], a["Y"], a["ws"], a["wsb"])
    go.at, go.keep = at, keep
    return go


ALL = ["gate", "gate_bwd", "pack", "unpack", "weights", "norm", "norm_bwd", "linear", "mlp"]


@pytest.mark.parametrize("name", ALL)
def test_no_context(call, name):
    assert call(name, ctx=None) == INVALID


GATE = [dict(norule=True), dict(T=-1), dict(E=0), dict(k=0), dict(k=9), dict(score=2), dict(score=-1), dict(groups=0), dict(groups=3), dict(kept=0), dict(kept=5), dict(best=0),
        dict(kept=1, k=3), dict(renorm=2), dict(scale=math.nan), dict(scale=math.inf), dict(x=None)]
TOO_MUCH = [dict(best=3), dict(E=1032, groups=1, kept=1), dict(E=256, groups=128, kept=128, k=2), dict(E=128, k=65, groups=1, kept=1), dict(T=2 ** 30, k=2), dict(T=2 ** 26 - 63, k=2), dict(x=STEP + 4)]


@pytest.mark.parametrize("name", ["gate", "gate_bwd"])
def test_gate(call, name):
    for bad in GATE + [dict(i=None)] + ([dict(g=None)] if name == "gate" else [dict(dg=None), dict(dx=None)]):
        assert call(name, **bad) == INVALID, bad
    for bad in TOO_MUCH:
        assert call(name, **bad) == UNSUPPORTED, bad
    over = [dict(i="x"), dict(g="x"), dict(i="b"), dict(g="b"), dict(i="g")] if name == "gate" else [dict(dx="i"), dict(dx="dg")]
    for pair in over:
        (a, b), = pair.items()
        for off in (0, 16):
            assert call(name, **{a: call.at[b] + off}) == INVALID, pair
    if name == "gate_bwd":
        assert call(name, dx=call.at["x"] + 16) == INVALID
    assert call(name, T=0, x=None, i=None, g=None, dg=None, dx=None) == OK


@pytest.mark.parametrize("name", ["pack", "unpack"])
def test_rows(call, name):
    for bad in (dict(dtype=7), dict(rows=-1), dict(d=0), dict(x=None), dict(Xv=None), dict(Xe=None)):
        assert call(name, **bad) == INVALID, bad
    for bad in (dict(d=(1 << 22) + 1), dict(x=STEP + 8), dict(Xv=STEP * 3 + 1), dict(Xe=STEP * 3 + 4)):
        assert call(name, **bad) == UNSUPPORTED, bad
    for bad in (dict(x=call.at["Xv"] + 16), dict(x=call.at["Xe"]), dict(Xe=call.at["x"] + 2032)):
        assert call(name, **bad) == INVALID, bad
    if name == "pack":
        assert call(name, Xe=call.at["Xv"] + 1008) == INVALID
    assert call(name, rows=0, x=None) == OK


def test_weights(m, call):
    for bad in (dict(dtype=5), dict(W=None), dict(Wv=None), dict(We=None), dict(E=0), dict(d=0), dict(d_out=0), dict(halves=0), dict(halves=3), dict(d_out=63, halves=2),
                dict(W=call.at["Wv"] + 32), dict(We=call.at["Wv"])):
        assert call("weights", **bad) == INVALID, bad
    for bad in (dict(E=65536), dict(d=(1 << 22) + 1), dict(W=STEP + 8)):
        assert call("weights", **bad) == UNSUPPORTED, bad
    size = m.lib.smoe_weights8_bytes
    assert size(0, 4, 4, 1) == size(1, 0, 4, 1) == size(1, 4, 0, 1) == size(1, 4, 3, 2) == size(1, 4, 4, 3) == size(65536, 4, 4, 1) == 0
    assert size(3, 129, 33, 1) == 3 * 256 * 64 and size(3, 128, 66, 2) == 3 * 128 * 128


def test_norm(call):
    for bad in (dict(dtype=9), dict(rows=-1), dict(d=0), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(Y=None, Yv=None), dict(x=None), dict(w=None), dict(Ye=None)):
        assert call("norm", **bad) == INVALID, bad
    for bad in (dict(d=32769), dict(rows=2 ** 31 - 63), dict(x=STEP + 8), dict(S=STEP + 2), dict(rstd=STEP + 4)):
        assert call("norm", **bad) == UNSUPPORTED, bad
    at = call.at
    for out in ("S", "Y"):
        for into in ("x", "R"):
            assert call("norm", **{out: at[into] + 16}) == INVALID
        assert call("norm", **{out: at["w"]}) == INVALID
    for a, b in (("S", "Y"), ("rstd", "x"), ("rstd", "S"), ("Yv", "x"), ("Yv", "R"), ("Ye", "Y"), ("Yv", "w"), ("Ye", "Yv"), ("rstd", "Ye")):
        assert call("norm", **{a: at[b]}) == INVALID, (a, b)
    assert call("norm", rows=0, x=None, S=None) == OK


def test_norm_gradient(m, call):
    for bad in (dict(dtype=9), dict(rows=-1), dict(d=0), dict(dY=None), dict(S=None), dict(w=None), dict(rstd=None), dict(dX=None), dict(dw=None)):
        assert call("norm_bwd", **bad) == INVALID, bad
    for bad in (dict(d=32769), dict(dY=STEP + 8)):
        assert call("norm_bwd", **bad) == UNSUPPORTED, bad
    need = m.lib.smoe_add_norm_bwd_workspace_bytes(1, 4, 256)
    assert need and need % 256 == 0
    for bad in (dict(ws=None), dict(ws=call.at["ws"] + 16), dict(wsb=need - 1)):
        assert call("norm_bwd", **bad) == WORKSPACE, bad
    at = call.at
    for into in ("dY", "S", "dS"):
        assert call("norm_bwd", dX=at[into] + 16) == INVALID
    for a, b in (("dX", "w"), ("dX", "rstd"), ("dw", "dY"), ("dw", "S"), ("dw", "w"), ("dw", "dX"), ("ws", "dY"), ("ws", "dS"), ("ws", "dX"), ("ws", "dw"), ("ws", "rstd")):
        assert call("norm_bwd", **{a: at[b]}) == INVALID, (a, b)
    size = m.lib.smoe_add_norm_bwd_workspace_bytes
    assert size(1, 4, 0) == size(1, -1, 8) == size(7, 4, 8) == size(1, 4, 32769) == 0


def test_linear(call):
    for bad in (dict(d=0), dict(d_out=0), dict(k=0), dict(x_rows=-1), dict(x_rows=5), dict(gin=1), dict(gout=1), dict(gates_k=0), dict(gates_k=3), dict(Y=None), dict(g=None), dict(wE=7),
                dict(w_in=128), dict(w_out=72), dict(halves=2), dict(Xv=None), dict(Yhat=None), dict(off=None), dict(o=None), dict(Tk=-1), dict(Wv=None)):
        assert call("linear", **bad) == INVALID, bad
    for bad in (dict(d_out=60), dict(Xv=STEP + 8), dict(Yhat=STEP + 8), dict(Tk=2 ** 31 - 2, x_rows=2 ** 30 - 1, d_out=2 ** 20)):
        assert call("linear", **bad) == UNSUPPORTED, bad
    at = call.at
    for a, b in (("Yhat", "Xv"), ("Yhat", "Xe"), ("Yhat", "Wv"), ("Yhat", "We"), ("Yhat", "g"), ("Y", "Xv"), ("Y", "g"), ("Y", "Yhat"), ("Y", "Wv"), ("Yhat", "o"), ("Y", "off")):
        assert call("linear", **{a: at[b]}) == INVALID, (a, b)
    assert call("linear", Tk=0, x_rows=0, Xv=None, Yhat=None) == OK


def test_mlp(m, call):
    for bad in (dict(T=-1), dict(d_model=0), dict(d_expert=0), dict(k=0), dict(act=5), dict(Tk=6), dict(wE=7), dict(w_in=256), dict(w_out=64), dict(w1_halves=1), dict(v_in=128), dict(v_halves=2),
                dict(act=1, w1_halves=2), dict(Xv=None), dict(g=None), dict(Y=None), dict(off=None)):
        assert call("mlp", **bad) == INVALID, bad
    for bad in (dict(act=0), dict(d_model=100), dict(Y=STEP + 8), dict(d_expert=(1 << 21) + 1)):
        assert call("mlp", **bad) == UNSUPPORTED, bad
    need = m.lib.smoe_mlp8_fwd_workspace_bytes(2, 4, 2, 128, 64)
    assert need and need % 256 == 0
    for bad in (dict(ws=None), dict(ws=call.at["ws"] + 16), dict(wsb=need - 1)):
        assert call("mlp", **bad) == WORKSPACE, bad
    at = call.at
    for a, b in (("Y", "Xv"), ("Y", "Xe"), ("Y", "Wv"), ("Y", "Ve"), ("Y", "g"), ("Y", "ws"), ("ws", "Xv"), ("ws", "Xe"), ("ws", "Vv"), ("ws", "We"), ("ws", "g"), ("ws", "o"), ("Y", "off")):
        assert call("mlp", **{a: at[b]}) == INVALID, (a, b)
    assert call("mlp", T=0, Tk=0, Xv=None, Y=None, ws=None) == OK
    size = m.lib.smoe_mlp8_fwd_workspace_bytes
    assert size(0, 4, 2, 128, 64) == size(2, -1, 2, 128, 64) == size(2, 4, 0, 128, 64) == size(2, 4, 2, 0, 64) == size(2, 2 ** 30, 2, 8, 8) == 0


# ------------------------------------------------------------------------------------------------------------- binding
class Real(Library):
    def smoe_weights8_bytes(self, E, d_in, d_out, halves):
        self.calls.append("smoe_weights8_bytes")
        return E * halves * 2 * -(-d_out // halves // 32) * -(-d_in // 128) * 2048



@pytest.fixture
def smoe(monkeypatch, m):
    monkeypatch.setattr(m, "lib", Real())
    monkeypatch.setattr(m, "_new", lambda *shape, dtype, device: Tensor(*shape, dtype=dtype))
    monkeypatch.setattr(m, "_device", lambda first: 0)
    monkeypatch.setattr(m, "_where", lambda dev: (None, None))
    return m


def floats(*shape, **kw):
    return Tensor(*shape, dtype=torch.float32, **kw)


def bytes_(*shape, **kw):
    return Tensor(*shape, dtype=torch.uint8, **kw)


def launches(m):
    return [c for c in m.lib.calls if not c.endswith("_bytes")]


def test_binding_of_the_gate(smoe):
    rule = smoe.gate_rule("sigmoid", 4, 2, 2)
    with pytest.raises(ValueError):
        smoe.gate_rule("tanh")
    with pytest.raises(AttributeError):
        rule.scale = 2.0
    for bad, error in ((lambda: smoe.score_gate(Tensor(4, 8), 2, rule), TypeError), (lambda: smoe.score_gate(floats(4, 2, 4), 2, rule), ValueError),
                       (lambda: smoe.score_gate(floats(4, 8), 9, rule), ValueError), (lambda: smoe.score_gate(floats(4, 8), 2, rule, floats(7)), ValueError),
                       (lambda: smoe.score_gate(floats(4, 8), 2, rule, floats(8, device=1)), ValueError), (lambda: smoe.score_gate(floats(4, 8, contiguous=False), 2, rule), ValueError),
                       (lambda: smoe.score_gate(floats(2 ** 32 + 4, 8), 2, rule), ValueError), (lambda: smoe.score_gate_bwd(floats(4, 8), ints(4, 2), floats(4, 3), rule), ValueError),
                       (lambda: smoe.score_gate_bwd(floats(4, 8), ints(3, 2), floats(3, 2), rule), ValueError), (lambda: smoe.score_gate_bwd(floats(4, 8), floats(4, 2), floats(4, 2), rule), TypeError)):
        with pytest.raises(error):
            bad()
    assert not launches(smoe)
    smoe.score_gate(floats(4, 8), 2, rule, floats(8))
    smoe.score_gate_bwd(floats(4, 8), ints(4, 2), floats(4, 2), rule)
    assert launches(smoe) == ["smoe_score_gate", "smoe_score_gate_bwd"]


def a_rows(m, *shape, device=0):
    P = -(-shape[-1] // 128) * 128
    r = m.Rows8.__new__(m.Rows8)
    v, e = bytes_(*shape[:-1], P, device=device), bytes_(*shape[:-1], P // 32, device=device)
    r.__init__(v, e, shape[-1])
    return r


def a_weights(m, E, d_in, d_out, halves=1, device=0):
    n = Real().smoe_weights8_bytes(E, d_in, d_out, halves)
    return m.Weights8(bytes_(n, device=device), bytes_(n // 32, device=device), E, d_in, d_out, halves)


def test_binding_of_rows_and_weights(smoe):
    for v, e, d in ((bytes_(4, 100), bytes_(4, 4), 100), (bytes_(4, 128), bytes_(4, 3), 100), (bytes_(4, 256), bytes_(4, 8), 128), (bytes_(4, 128), bytes_(5, 4), 128),
                    (bytes_(4, 128), bytes_(4, 4), 129), (bytes_(4, 128), bytes_(4, 4), 0), (bytes_(4, 128), bytes_(4, 4, device=1), 128)):
        with pytest.raises(ValueError):
            smoe.Rows8(v, e, d)
    with pytest.raises(TypeError):
        smoe.Rows8(Tensor(4, 128), bytes_(4, 4), 128)
    rows = a_rows(smoe, 4, 100)
    with pytest.raises(AttributeError):
        rows.values = bytes_(4, 128)
    for bad in (lambda: smoe.rows8_pack(Tensor(4, 100), out=a_rows(smoe, 5, 100)), lambda: smoe.rows8_pack(Tensor(4, 100), out=a_rows(smoe, 4, 101)), lambda: smoe.rows8_pack(Tensor(4, 0)),
                lambda: smoe.rows8_unpack(a_rows(smoe, 4, 100, device=1)), lambda: smoe.rows8_pack(Tensor(2 ** 32 + 1, 8)), lambda: smoe.weights8(Tensor(4, 8)),
                lambda: smoe.Weights8(bytes_(2048), bytes_(64), 1, 128, 32, 1)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        smoe.rows8_pack(Tensor(4, 100, dtype=torch.float16))
    assert not launches(smoe)
    smoe.rows8_pack(Tensor(2, 3, 100))
    smoe.weights8(Tensor(2, 64, 64), halves=2)
    assert launches(smoe) == ["smoe_rows8_pack", "smoe_weights8_pack"]


def test_binding_of_the_norm(smoe):
    X, w = Tensor(2, 3, 64), Tensor(64)
    kept = smoe.Norm(Tensor(2, 3, 64), Tensor(2, 3, 64), None, floats(6))
    for bad in (lambda: smoe.add_norm_fwd(X, Tensor(32)), lambda: smoe.add_norm_fwd(X, w, Tensor(3, 2, 64)), lambda: smoe.add_norm_fwd(X, w, plain=False),
                lambda: smoe.add_norm_fwd(X, w, Tensor(2, 3, 64, device=1)), lambda: smoe.add_norm_fwd(X, w, X, packed=True, out=kept), lambda: smoe.add_norm_fwd(Tensor(2, 4, 64), w, out=kept),
                lambda: smoe.add_norm_bwd(X, Tensor(6, 64), w, floats(6)), lambda: smoe.add_norm_bwd(X, X, w, floats(5)), lambda: smoe.add_norm_bwd(X, X, w, floats(6), dS=Tensor(6, 64)),
                lambda: smoe.add_norm_bwd(X, X, w, floats(6), out=(Tensor(6, 64), w)), lambda: smoe.add_norm_fwd(Tensor(2 ** 32 + 2, 1), Tensor(1))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: smoe.add_norm_fwd(X, floats(64)), lambda: smoe.add_norm_bwd(X, X, w, Tensor(6))):
        with pytest.raises(TypeError):
            bad()
    assert not launches(smoe)
    assert smoe.add_norm_fwd(X, w).S is X
    assert smoe.add_norm_fwd(X, w, out=kept).S is X                               # nothing added: the stream is X, whatever the kept one was
    assert smoe.add_norm_fwd(X, w, Tensor(2, 3, 64), out=kept) is kept
    smoe.add_norm_bwd(X, X, w, floats(6))
    assert launches(smoe) == ["smoe_add_norm_fwd"] * 3 + ["smoe_add_norm_bwd"]


def test_binding_of_the_products(smoe):
    r = smoe.Routing(ints(8), ints(8), ints(5), 8, 4)
    X, W1, W2, g = a_rows(smoe, 4, 96), a_weights(smoe, 4, 96, 128, 2), a_weights(smoe, 4, 64, 96), floats(4, 2)
    mlp = lambda **c: smoe.mlp8_fwd(**({"X": X, "W1": W1, "W2": W2, "r": r, "k": 2, "gates": g, "act": smoe.ACT_SWIGLU} | c))
    for bad in (dict(X=a_rows(smoe, 4, 95)), dict(X=a_rows(smoe, 5, 96)), dict(X=a_rows(smoe, 4, 96, device=1)), dict(W1=a_weights(smoe, 4, 96, 128)), dict(W1=a_weights(smoe, 3, 96, 128, 2)),
                dict(W2=a_weights(smoe, 4, 65, 96)), dict(W2=a_weights(smoe, 4, 64, 104)), dict(act=smoe.ACT_GELU), dict(k=3), dict(gates=floats(4, 3)), dict(gates=floats(4, 2, device=1)),
                dict(out=Tensor(4, 95)), dict(out=Tensor(96, 4)), dict(r=smoe.Routing(ints(8), ints(7), ints(5), 8, 4)), dict(r=smoe.Routing(ints(8), ints(8), ints(4), 8, 4)),
                dict(W2=a_weights(smoe, 4, 64, 96, device=1))):
        with pytest.raises(ValueError):
            mlp(**bad)
    with pytest.raises(TypeError):
        mlp(gates=Tensor(4, 2))
    for bad in (lambda: smoe.plinear8_fwd(a_rows(smoe, 4, 95), W2, r, 2), lambda: smoe.plinear8_fwd(a_rows(smoe, 4, 64), W2, r, 2, floats(4, 3)),
                lambda: smoe.plinear8_fwd(a_rows(smoe, 4, 64), a_weights(smoe, 5, 64, 96), r, 2)):
        with pytest.raises(ValueError):
            bad()
    assert not launches(smoe)
    assert mlp().shape == (4, 96)
    smoe.plinear8_fwd(a_rows(smoe, 4, 64), W2, r, 2, g)
    assert launches(smoe) == ["smoe_mlp8_fwd", "smoe_plinear8_fwd"]
