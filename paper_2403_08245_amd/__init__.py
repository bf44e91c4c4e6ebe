"""Python binding of libsmoe (ScatterMoE's ParallelLinear hot path on MI355X).

Argument marshalling only: every function here checks tensor dtypes/contiguity, allocates
outputs and scratch with torch, and calls the C entry point of the same name
(smoe_<name>, declared in include/smoe.h, in include/smoe_cache.h for positions and serving, or in include/smoe_block.h for the gate by
scores, the norm and the products in 8 bits) on torch's current HIP stream.  There is no
Python or PyTorch fallback: if libsmoe.so is missing, importing this package fails.
"""
from __future__ import annotations

import ctypes
import math
import os
from dataclasses import dataclass

import torch

ACT_NONE, ACT_GELU, ACT_SWIGLU = 0, 1, 2
F32, BF16 = 0, 1

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libsmoe.so")

EXPORTS = [
    "smoe_create", "smoe_destroy", "smoe_strerror", "smoe_abi_version", "smoe_set_kernel_mode", "smoe_set_clock_probe", "smoe_set_tile_group",
    "smoe_topk_gate", "smoe_topk_gate_bwd", "smoe_route_workspace_bytes", "smoe_route", "smoe_route_noalloc",
    "smoe_plinear_fwd", "smoe_plinear_bwd_workspace_bytes", "smoe_plinear_bwd",
    "smoe_plinear_act_fwd_workspace_bytes", "smoe_plinear_act_fwd", "smoe_mlp_fwd_workspace_bytes", "smoe_mlp_fwd", "smoe_mlp_saves_yhat", "smoe_mlp_bwd_workspace_bytes", "smoe_mlp_bwd",
    "smoe_group", "smoe_attention_fwd", "smoe_attention_bwd_workspace_bytes", "smoe_attention_bwd",
    "smoe_momha_fwd_workspace_bytes", "smoe_momha_fwd", "smoe_momha_bwd_workspace_bytes", "smoe_momha_bwd",
]

CACHE_EXPORTS = [
    "smoe_rotary_frequencies", "smoe_rotary_fwd", "smoe_rotary_bwd", "smoe_cache_append", "smoe_cache_read",
    "smoe_cached_attention_workspace_bytes", "smoe_cached_attention_fwd", "smoe_momha_decode_workspace_bytes", "smoe_momha_decode",
]

BLOCK_EXPORTS = [
    "smoe_score_gate", "smoe_score_gate_bwd", "smoe_rows8_pack", "smoe_rows8_unpack", "smoe_weights8_bytes", "smoe_weights8_pack", "smoe_add_norm_fwd",
    "smoe_add_norm_bwd_workspace_bytes", "smoe_add_norm_bwd", "smoe_plinear8_fwd", "smoe_mlp8_fwd_workspace_bytes", "smoe_mlp8_fwd",
]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} not found: build it first (python __graft_entry__.py); "
            "this package has no fallback path")
    return ctypes.CDLL(LIB_PATH)


lib = _load()

_vp, _i, _sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t


class smoe_routing(ctypes.Structure):
    _fields_ = [("sorted_expert_idxs", _vp), ("sorted_scattered_idxs", _vp), ("expert_offsets", _vp),
                ("Tk", ctypes.c_int32), ("E", ctypes.c_int32)]


_rp = ctypes.POINTER(smoe_routing)
lib.smoe_create.argtypes = [ctypes.POINTER(_vp), _i]
lib.smoe_destroy.argtypes = [_vp]
lib.smoe_destroy.restype = None
lib.smoe_strerror.argtypes = [_i]
lib.smoe_strerror.restype = ctypes.c_char_p
lib.smoe_set_kernel_mode.argtypes = [_vp, _i]
lib.smoe_set_clock_probe.argtypes = [_vp, _vp]
lib.smoe_set_tile_group.argtypes = [_vp, _i]
lib.smoe_topk_gate.argtypes = [_vp, _vp, _vp, _i, _i, _i, _vp, _vp]
lib.smoe_topk_gate_bwd.argtypes = [_vp, _vp, _vp, _vp, _vp, _i, _i, _i, _vp]
lib.smoe_attention_fwd.argtypes = [_vp, _vp, _i, _vp, _vp, _vp, _i, _i, _i, _i, _i, _vp, _vp]
lib.smoe_attention_bwd_workspace_bytes.argtypes = [_i, _i, _i, _i]
lib.smoe_attention_bwd_workspace_bytes.restype = _sz
lib.smoe_attention_bwd.argtypes = [_vp, _vp, _i, _vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _vp, _vp, _vp, _vp, _sz]
lib.smoe_momha_fwd_workspace_bytes.argtypes = [_i] * 7
lib.smoe_momha_fwd_workspace_bytes.restype = _sz
lib.smoe_momha_fwd.argtypes = [_vp, _vp, _i, _vp, _i, _i, _i, _i, _i, _vp, _vp, _vp, _vp, _rp, _i, _vp, _vp,
                               _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz]
lib.smoe_momha_bwd_workspace_bytes.argtypes = [_i] * 6
lib.smoe_momha_bwd_workspace_bytes.restype = _sz
lib.smoe_momha_bwd.argtypes = [_vp, _vp, _i, _vp, _vp, _i, _i, _i, _i, _i, _vp, _vp, _vp, _vp, _rp, _i, _vp,
                               _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz]
lib.smoe_route_workspace_bytes.argtypes = [_i, _i, _i]
lib.smoe_route_workspace_bytes.restype = _sz
lib.smoe_route.argtypes = [_vp, _vp, _vp, _i, _i, _i, _vp, _vp, _vp, _vp, _sz]
lib.smoe_route_noalloc.argtypes = [_vp, _vp, _vp, _i, _i, _i, _vp, _vp, _vp]
lib.smoe_plinear_fwd.argtypes = [_vp, _vp, _i, _vp, _i, _i, _vp, _i, _rp, _i, _vp, _i, _i, _i, _vp, _vp]
lib.smoe_plinear_bwd_workspace_bytes.argtypes = [_i] * 9
lib.smoe_plinear_bwd_workspace_bytes.restype = _sz
lib.smoe_plinear_bwd.argtypes = [_vp, _vp, _i, _vp, _vp, _i, _i, _vp, _i, _vp, _rp, _i, _vp, _i, _i, _i,
                                 _vp, _vp, _vp, _vp, _sz]
lib.smoe_plinear_act_fwd_workspace_bytes.argtypes = [_i] * 7
lib.smoe_plinear_act_fwd_workspace_bytes.restype = _sz
lib.smoe_plinear_act_fwd.argtypes = [_vp, _vp, _i, _i, _vp, _i, _i, _i, _vp, _rp, _i, _vp, _vp, _vp, _sz]
lib.smoe_mlp_fwd_workspace_bytes.argtypes = [_i] * 7
lib.smoe_mlp_fwd_workspace_bytes.restype = _sz
lib.smoe_mlp_fwd.argtypes = [_vp, _vp, _i, _i, _vp, _i, _i, _i, _vp, _vp, _rp, _i, _vp, _vp, _vp, _vp, _vp, _vp, _sz]
lib.smoe_mlp_bwd_workspace_bytes.argtypes = [_i] * 6
lib.smoe_mlp_saves_yhat.argtypes = [_vp, _i, _i, _i, _i, _i, _i, _i]
lib.smoe_mlp_bwd_workspace_bytes.restype = _sz
lib.smoe_mlp_bwd.argtypes = [_vp, _vp, _i, _i, _vp, _vp, _i, _i, _i, _vp, _vp, _rp, _i, _vp, _vp, _vp, _vp,
                             _vp, _vp, _vp, _vp, _vp, _sz]
lib.smoe_group.argtypes = [_vp, _vp, _i, _vp, _i, _rp, _i, _vp, _vp]


class smoe_rotary(ctypes.Structure):
    _fields_ = [("turns", _vp), ("rot", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("amplitude", ctypes.c_float)]


class smoe_cache(ctypes.Structure):
    _fields_ = [("K", _vp), ("V", _vp), ("K_exp", _vp), ("V_exp", _vp), ("pages", ctypes.c_int32), ("page", ctypes.c_int32),
                ("h", ctypes.c_int32), ("d_head", ctypes.c_int32), ("format", ctypes.c_int32)]


class smoe_places(ctypes.Structure):
    _fields_ = [("block_table", _vp), ("sequences", ctypes.c_int32), ("width", ctypes.c_int32), ("seqs", _vp), ("positions", _vp), ("lens", _vp)]


_op, _cp, _pp, _d = ctypes.POINTER(smoe_rotary), ctypes.POINTER(smoe_cache), ctypes.POINTER(smoe_places), ctypes.c_double
lib.smoe_rotary_frequencies.argtypes = [_i, _d, _i, _d, _d, _vp, _vp]
lib.smoe_rotary_fwd.argtypes = lib.smoe_rotary_bwd.argtypes = [_vp, _vp, _i, _vp, _i, _vp, _i, _i, _i, _i, _vp, _op, _vp, _vp]
lib.smoe_cache_append.argtypes = [_vp, _vp, _i, _cp, _pp, _vp, _vp, _i, _op, _vp, _i, _vp]
lib.smoe_cache_read.argtypes = [_vp, _vp, _i, _cp, _pp, _i, _vp, _vp]
lib.smoe_cached_attention_workspace_bytes.argtypes = [_cp, _pp, _i, _i]
lib.smoe_cached_attention_workspace_bytes.restype = _sz
lib.smoe_cached_attention_fwd.argtypes = [_vp, _vp, _i, _vp, _i, _i, _cp, _pp, _vp, _vp, _vp, _sz]
lib.smoe_momha_decode_workspace_bytes.argtypes = [_i] * 6
lib.smoe_momha_decode_workspace_bytes.restype = _sz
lib.smoe_momha_decode.argtypes = [_vp, _vp, _i, _vp, _i, _i, _vp, _vp, _vp, _vp, _rp, _i, _vp, _cp, _pp, _op, _vp, _vp, _sz]


class smoe_gate_rule(ctypes.Structure):
    _fields_ = [("score", ctypes.c_int32), ("groups", ctypes.c_int32), ("kept_groups", ctypes.c_int32), ("group_best", ctypes.c_int32),
                ("renormalise", ctypes.c_int32), ("scale", ctypes.c_float)]


class smoe_rows8(ctypes.Structure):
    _fields_ = [("values", _vp), ("exps", _vp)]


class smoe_weights8(ctypes.Structure):
    _fields_ = [("values", _vp), ("exps", _vp), ("E", ctypes.c_int32), ("d_in", ctypes.c_int32), ("d_out", ctypes.c_int32), ("halves", ctypes.c_int32)]


_gp, _r8, _w8 = ctypes.POINTER(smoe_gate_rule), ctypes.POINTER(smoe_rows8), ctypes.POINTER(smoe_weights8)
lib.smoe_score_gate.argtypes = [_vp, _vp, _vp, _vp, _i, _i, _i, _gp, _vp, _vp]
lib.smoe_score_gate_bwd.argtypes = [_vp, _vp, _vp, _vp, _vp, _i, _i, _i, _gp, _vp]
lib.smoe_rows8_pack.argtypes = [_vp, _vp, _i, _vp, _i, _i, _r8]
lib.smoe_rows8_unpack.argtypes = [_vp, _vp, _i, _r8, _i, _i, _vp]
lib.smoe_weights8_bytes.argtypes = [_i] * 4
lib.smoe_weights8_bytes.restype = _sz
lib.smoe_weights8_pack.argtypes = [_vp, _vp, _i, _vp, _w8]
lib.smoe_add_norm_fwd.argtypes = [_vp, _vp, _i, _vp, _vp, _vp, _i, _i, ctypes.c_float, _vp, _vp, _r8, _vp]
lib.smoe_add_norm_bwd_workspace_bytes.argtypes = [_i] * 3
lib.smoe_add_norm_bwd_workspace_bytes.restype = _sz
lib.smoe_add_norm_bwd.argtypes = [_vp, _vp, _i, _vp, _vp, _vp, _vp, _vp, _i, _i, _vp, _vp, _vp, _sz]
lib.smoe_plinear8_fwd.argtypes = [_vp, _vp, _r8, _i, _i, _w8, _i, _rp, _i, _vp, _i, _i, _i, _vp, _vp]
lib.smoe_mlp8_fwd_workspace_bytes.argtypes = [_i] * 5
lib.smoe_mlp8_fwd_workspace_bytes.restype = _sz
lib.smoe_mlp8_fwd.argtypes = [_vp, _vp, _i, _r8, _i, _i, _i, _w8, _w8, _rp, _i, _vp, _vp, _vp, _sz]


class SmoeError(RuntimeError):
    pass


def _check(rc: int, what: str):
    if rc != 0:
        raise SmoeError(f"{what}: {lib.smoe_strerror(rc).decode()} ({rc})")


_ctx_by_device: dict[int, ctypes.c_void_p] = {}


def ctx(device: int | None = None) -> ctypes.c_void_p:
    """The library context of a device (created on first use)."""
    dev = torch.cuda.current_device() if device is None else device
    if dev not in _ctx_by_device:
        h = _vp()
        _check(lib.smoe_create(ctypes.byref(h), dev), "smoe_create")
        _ctx_by_device[dev] = h
    return _ctx_by_device[dev]


def set_kernel_mode(mode: int):
    _check(lib.smoe_set_kernel_mode(ctx(), mode), "smoe_set_kernel_mode")


def set_tile_group(group_m: int):
    _check(lib.smoe_set_tile_group(ctx(), group_m), "smoe_set_tile_group")


def set_clock_probe(buf: torch.Tensor | None):
    """Device int64 tensor of 512 entries that the persistent scatter2scatter kernels report their clocks to
    (see smoe_set_clock_probe), or None to turn the probe off."""
    if buf is not None and (buf.dtype != torch.int64 or buf.numel() < 512 or not buf.is_cuda):
        raise ValueError("need a device int64 tensor of 512 entries")
    _check(lib.smoe_set_clock_probe(ctx(), _p(buf)), "smoe_set_clock_probe")


def _stream() -> int:
    # the handle of torch's current stream on the current device; torch.cuda.current_stream() makes a Stream object first, 2.8 us
    # a call of 0.2 (41 us of host work in a four-token forward pass with routing, three calls)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _p(t):
    return None if t is None else t.data_ptr()


def _chk(t: torch.Tensor, dtype=None):
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("tensors must be contiguous device tensors")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"expected {dtype}, got {t.dtype}")
    return t


def _new(*shape, dtype, device) -> torch.Tensor:
    """Every output and scratch tensor of this binding comes from here (uninitialised device memory).
    Tests replace this one function to poison new tensors and to put guard bands around them."""
    return torch.empty(*shape, dtype=dtype, device=device)


def _like(t: torch.Tensor) -> torch.Tensor:
    return _new(*t.shape, dtype=t.dtype, device=t.device)


def _ws(nbytes: int, device) -> torch.Tensor | None:
    return _new(max(nbytes, 256), dtype=torch.uint8, device=device)


@dataclass
class Routing:
    """Device arrays of Sec. 3.1 step 2 plus the ctypes view the C ABI takes."""
    sorted_expert_idxs: torch.Tensor
    sorted_scattered_idxs: torch.Tensor
    expert_offsets: torch.Tensor
    Tk: int
    E: int

    def c(self) -> smoe_routing:
        return smoe_routing(self.sorted_expert_idxs.data_ptr(), self.sorted_scattered_idxs.data_ptr(),
                            self.expert_offsets.data_ptr(), self.Tk, self.E)


def topk_gate(logits: torch.Tensor, k: int):
    _chk(logits, torch.float32)
    T, E = logits.shape
    idx = _new(T, k, dtype=torch.int32, device=logits.device)
    gates = _new(T, k, dtype=torch.float32, device=logits.device)
    _check(lib.smoe_topk_gate(ctx(), _stream(), _p(logits), T, E, k, _p(idx), _p(gates)), "smoe_topk_gate")
    return idx, gates


def topk_gate_bwd(expert_idxs: torch.Tensor, gates: torch.Tensor, dgates: torch.Tensor, E: int) -> torch.Tensor:
    _chk(expert_idxs, torch.int32)
    _chk(gates, torch.float32)
    _chk(dgates, torch.float32)
    T, k = expert_idxs.shape
    if gates.numel() != T * k or dgates.numel() != T * k:
        raise ValueError("gates and dgates must hold T*k entries")
    dlogits = _new(T, E, dtype=torch.float32, device=gates.device)
    _check(lib.smoe_topk_gate_bwd(ctx(), _stream(), _p(expert_idxs), _p(gates), _p(dgates), T, E, k, _p(dlogits)),
           "smoe_topk_gate_bwd")
    return dlogits


def attention_fwd(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor):
    """Q [B,T,G,h,d], K and V [B,T,h,d] (bf16) -> O like Q, LSE [B,T,G,h] fp32."""
    for t in (Q, K, V):
        _chk(t, torch.bfloat16)
    B, T, G, h, d = Q.shape
    if K.shape != (B, T, h, d) or V.shape != K.shape:
        raise ValueError("K and V must be [B, T, h, d]")
    O = _like(Q)
    LSE = _new(B, T, G, h, dtype=torch.float32, device=Q.device)
    _check(lib.smoe_attention_fwd(ctx(), _stream(), BF16, _p(Q), _p(K), _p(V), B, T, G, h, d, _p(O), _p(LSE)),
           "smoe_attention_fwd")
    return O, LSE


def attention_bwd(dO, Q, K, V, O, LSE):
    for t in (dO, Q, K, V, O):
        _chk(t, torch.bfloat16)
    _chk(LSE, torch.float32)
    B, T, G, h, d = Q.shape
    dQ, dK, dV = _like(Q), _like(K), _like(V)
    nb = lib.smoe_attention_bwd_workspace_bytes(B, T, G, h)
    ws = _ws(nb, Q.device)
    _check(lib.smoe_attention_bwd(ctx(), _stream(), BF16, _p(dO), _p(Q), _p(K), _p(V), _p(O), _p(LSE), B, T, G, h, d,
                                  _p(dQ), _p(dK), _p(dV), _p(ws), nb), "smoe_attention_bwd")
    return dQ, dK, dV


@dataclass
class MomhaBuffers:
    """Tensors smoe_momha_fwd keeps for the backward pass (Alg. 4's intermediates)."""
    K: torch.Tensor
    V: torch.Tensor
    Q: torch.Tensor
    Ohat: torch.Tensor
    LSE: torch.Tensor
    Yhat: torch.Tensor


def momha_fwd(X, W_K, W_V, W_Q, W_O, r: Routing, k: int, gates, B: int, T: int, h_expert: int, d_head: int):
    for t in (X, W_K, W_V, W_Q, W_O):
        _chk(t, torch.bfloat16)
    _chk(gates, torch.float32)
    N, d_model = X.shape
    d_out = h_expert * d_head
    dev = X.device
    bf = dict(dtype=torch.bfloat16, device=dev)
    buf = MomhaBuffers(_new(N, d_out, **bf), _new(N, d_out, **bf), _new(N * k, d_out, **bf),
                       _new(N * k, d_out, **bf), _new(N * k, h_expert, dtype=torch.float32, device=dev),
                       _new(N * k, d_model, **bf))
    O = _new(N, d_model, **bf)
    nb = lib.smoe_momha_fwd_workspace_bytes(B, T, k, d_model, h_expert, d_head, 1)
    ws = _ws(nb, dev)
    rc = r.c()
    _check(lib.smoe_momha_fwd(ctx(), _stream(), BF16, _p(X), B, T, d_model, h_expert, d_head, _p(W_K), _p(W_V),
                              _p(W_Q), _p(W_O), ctypes.byref(rc), k, _p(gates), _p(O), _p(buf.K), _p(buf.V),
                              _p(buf.Q), _p(buf.Ohat), _p(buf.LSE), _p(buf.Yhat), _p(ws), nb), "smoe_momha_fwd")
    return O, buf


def momha_bwd(dO, X, W_K, W_V, W_Q, W_O, r: Routing, k: int, gates, B: int, T: int, h_expert: int, d_head: int,
              buf: MomhaBuffers):
    _chk(dO, torch.bfloat16)
    N, d_model = X.shape
    dX, dW_K, dW_V = _like(X), _like(W_K), _like(W_V)
    dW_Q, dW_O = _like(W_Q), _like(W_O)
    dgates = _new(N, k, dtype=torch.float32, device=X.device)
    nb = lib.smoe_momha_bwd_workspace_bytes(B, T, k, d_model, h_expert, d_head)
    ws = _ws(nb, X.device)
    rc = r.c()
    _check(lib.smoe_momha_bwd(ctx(), _stream(), BF16, _p(dO), _p(X), B, T, d_model, h_expert, d_head, _p(W_K), _p(W_V),
                              _p(W_Q), _p(W_O), ctypes.byref(rc), k, _p(gates), _p(buf.K), _p(buf.V), _p(buf.Q),
                              _p(buf.Ohat), _p(buf.LSE), _p(buf.Yhat), _p(dX), _p(dW_K), _p(dW_V), _p(dW_Q), _p(dW_O),
                              _p(dgates), _p(ws), nb), "smoe_momha_bwd")
    return dX, dW_K, dW_V, dW_Q, dW_O, dgates


def route(expert_idxs: torch.Tensor, E: int) -> Routing:
    _chk(expert_idxs, torch.int32)
    T, k = expert_idxs.shape
    dev = expert_idxs.device
    se = _new(T * k, dtype=torch.int32, device=dev)
    so = _new(T * k, dtype=torch.int32, device=dev)
    off = _new(E + 1, dtype=torch.int32, device=dev)
    nb = lib.smoe_route_workspace_bytes(T, k, E)
    ws = _ws(nb, dev)
    _check(lib.smoe_route(ctx(), _stream(), _p(expert_idxs), T, k, E, _p(se), _p(so), _p(off), _p(ws), ws.numel()),
           "smoe_route")
    return Routing(se, so, off, T * k, E)


def route_noalloc(expert_idxs: torch.Tensor, E: int, out: Routing) -> Routing:
    """smoe_route_noalloc: routing into the caller's arrays `out`, scratch inside the library."""
    _chk(expert_idxs, torch.int32)
    T, k = expert_idxs.shape
    if out.sorted_expert_idxs.numel() < T * k or out.expert_offsets.numel() < E + 1:
        raise ValueError("output arrays too small")
    _check(lib.smoe_route_noalloc(ctx(), _stream(), _p(expert_idxs), T, k, E, _p(out.sorted_expert_idxs),
                                  _p(out.sorted_scattered_idxs), _p(out.expert_offsets)), "smoe_route_noalloc")
    return Routing(out.sorted_expert_idxs, out.sorted_scattered_idxs, out.expert_offsets, T * k, E)


def group(x: torch.Tensor, r: Routing, fan: int, gates: torch.Tensor | None = None) -> torch.Tensor:
    _chk(x)
    out = _new(r.Tk, x.shape[1], dtype=x.dtype, device=x.device)
    rc = r.c()
    _check(lib.smoe_group(ctx(), _stream(), _dt(x), _p(x), x.shape[1], ctypes.byref(rc), fan,
                          _p(None if gates is None else _chk(gates, torch.float32)), _p(out)), "smoe_group")
    return out


def plinear_fwd(X, W, r: Routing, k: int, gates=None, grouped_in=False, grouped_out=False):
    """Alg. 1.  Returns (Y, Yhat); Y is Yhat when no gates are given."""
    _chk(X); _chk(W, X.dtype)
    d_in, d_out = W.shape[1], W.shape[2]
    Yhat = _new(r.Tk, d_out, dtype=X.dtype, device=X.device)
    Y, gk = None, 0
    if gates is not None:
        _chk(gates, torch.float32)
        gk = gates.shape[1]
        Y = _new(r.Tk // gk, d_out, dtype=X.dtype, device=X.device)
    rc = r.c()
    _check(lib.smoe_plinear_fwd(ctx(), _stream(), _dt(X), _p(X), X.shape[0], d_in, _p(W), d_out, ctypes.byref(rc), k,
                                _p(gates), gk, int(grouped_in), int(grouped_out), _p(Yhat), _p(Y)), "smoe_plinear_fwd")
    return (Yhat if Y is None else Y), Yhat


def plinear_bwd(dY, X, W, Yhat, r: Routing, k: int, gates=None, grouped_in=False, grouped_out=False,
                need_dX=True, need_dW=True):
    """Alg. 2.  Returns (dX, dW, dgates)."""
    _chk(dY, X.dtype); _chk(X); _chk(W, X.dtype)
    d_in, d_out = W.shape[1], W.shape[2]
    dX = _like(X) if need_dX else None
    dW = _like(W) if need_dW else None
    dg, gk = None, 0
    if gates is not None:
        _chk(gates, torch.float32)
        gk = gates.shape[1]
        dg = _like(gates)
    nb = lib.smoe_plinear_bwd_workspace_bytes(_dt(X), X.shape[0], d_in, d_out, r.Tk, k, int(gates is not None),
                                              int(grouped_in), int(grouped_out))
    ws = _ws(nb, X.device)
    rc = r.c()
    _check(lib.smoe_plinear_bwd(ctx(), _stream(), _dt(X), _p(dY), _p(X), X.shape[0], d_in, _p(W), d_out, _p(Yhat),
                                ctypes.byref(rc), k, _p(gates), gk, int(grouped_in), int(grouped_out), _p(dX), _p(dW),
                                _p(dg), _p(ws), ws.numel()), "smoe_plinear_bwd")
    return dX, dW, dg


def hidden_width(act: int, d_expert: int) -> int:
    return 2 * d_expert if act == ACT_SWIGLU else d_expert


def plinear_act_fwd(X, W1, r: Routing, k: int, act: int, keep_hpre=True, out=None, ws=None):
    """Alg. 3 lines 1-2: returns (H, Hpre or None) in expert-sorted order.  `out` = (H, Hpre) and `ws` reuse
    preallocated tensors (repeated calls then allocate nothing)."""
    _chk(X); _chk(W1, X.dtype)
    T, d_model = X.shape
    d_expert = W1.shape[2] // 2 if act == ACT_SWIGLU else W1.shape[2]
    if out is None:
        H = _new(r.Tk, d_expert, dtype=X.dtype, device=X.device)
        Hpre = _new(r.Tk, W1.shape[2], dtype=X.dtype, device=X.device) if keep_hpre else None
    else:
        H, Hpre = out
    nb = lib.smoe_plinear_act_fwd_workspace_bytes(_dt(X), act, T, k, d_model, d_expert, int(Hpre is not None))
    if ws is None:
        ws = _ws(nb, X.device)
    rc = r.c()
    _check(lib.smoe_plinear_act_fwd(ctx(), _stream(), _dt(X), act, _p(X), T, d_model, d_expert, _p(W1), ctypes.byref(rc), k,
                                    _p(Hpre), _p(H), _p(ws), ws.numel()), "smoe_plinear_act_fwd")
    return H, Hpre


class MLPBuffers:
    """Preallocated outputs, saved activations and scratch of one SMoE MLP shape, so that
    repeated calls (training steps, benchmarks) do not allocate."""

    def __init__(self, T, k, E, d_model, d_expert, act, dtype, device, training=True):
        Tk, d_h = T * k, hidden_width(act, d_expert)
        dt = F32 if dtype == torch.float32 else BF16
        mk = lambda *s: _new(*s, dtype=dtype, device=device)
        self.T, self.k, self.E, self.d_model, self.d_expert, self.act, self.dtype = T, k, E, d_model, d_expert, act, dtype
        self.Y = mk(T, d_model)
        self.training = training
        mode = 0
        if training:
            needs = lib.smoe_mlp_saves_yhat(ctx(), dt, act, T, k, E, d_model, d_expert)
            _check(min(needs, 0), "smoe_mlp_saves_yhat")
            mode = 1 if needs else 2
            # the unweighted second product is kept only when the backward pass of this shape reads it
            self.Hpre, self.H, self.Yhat = mk(Tk, d_h), mk(Tk, d_expert), (mk(Tk, d_model) if needs else None)
            self.dX, self.dW1, self.dW2 = mk(T, d_model), mk(E, d_model, d_h), mk(E, d_expert, d_model)
            self.dgates = _new(T, k, dtype=torch.float32, device=device)
            self.ws_bwd = _ws(lib.smoe_mlp_bwd_workspace_bytes(dt, act, T, k, d_model, d_expert), device)
        else:
            self.Hpre = self.H = self.Yhat = None
        self.ws_fwd = _ws(lib.smoe_mlp_fwd_workspace_bytes(dt, act, T, k, d_model, d_expert, mode), device)


def mlp_fwd(X, W1, W2, r: Routing, k: int, gates, act: int, buf: MLPBuffers | None = None, training=True):
    """Alg. 3.  Returns (Y, buf); buf carries the tensors the backward pass needs."""
    _chk(X); _chk(W1, X.dtype); _chk(W2, X.dtype); _chk(gates, torch.float32)
    T, d_model = X.shape
    E, d_expert = W2.shape[0], W2.shape[1]
    if buf is None:
        buf = MLPBuffers(T, k, E, d_model, d_expert, act, X.dtype, X.device, training)
    rc = r.c()
    _check(lib.smoe_mlp_fwd(ctx(), _stream(), _dt(X), act, _p(X), T, d_model, d_expert, _p(W1), _p(W2),
                            ctypes.byref(rc), k, _p(gates), _p(buf.Y), _p(buf.Hpre), _p(buf.H), _p(buf.Yhat),
                            _p(buf.ws_fwd), buf.ws_fwd.numel()), "smoe_mlp_fwd")
    return buf.Y, buf


def mlp_bwd(dY, X, W1, W2, r: Routing, k: int, gates, act: int, buf: MLPBuffers):
    """Backward of mlp_fwd.  Returns (dX, dW1, dW2, dgates), views of buf."""
    _chk(dY, X.dtype)
    T, d_model = X.shape
    d_expert = W2.shape[1]
    rc = r.c()
    _check(lib.smoe_mlp_bwd(ctx(), _stream(), _dt(X), act, _p(dY), _p(X), T, d_model, d_expert, _p(W1), _p(W2),
                            ctypes.byref(rc), k, _p(gates), _p(buf.Hpre), _p(buf.H), _p(buf.Yhat), _p(buf.dX),
                            _p(buf.dW1), _p(buf.dW2), _p(buf.dgates), _p(buf.ws_bwd), buf.ws_bwd.numel()),
           "smoe_mlp_bwd")
    return buf.dX, buf.dW1, buf.dW2, buf.dgates


# ---- positions and serving (include/smoe_cache.h) ----------------------------------------------------------------------
# These calls are a few microseconds of work each, so their checks are written to cost little: the device is asked for once a call.
def _device(first: torch.Tensor) -> int:
    """The current device, on whose stream the launches go."""
    if not first.is_cuda:
        raise ValueError("tensors must be contiguous device tensors")
    return torch._C._cuda_getDevice()


def _here(dev: int, dtype, *tensors):
    """_chk, and that the tensors live on the current device."""
    for t in tensors:
        if not t.is_contiguous():
            raise ValueError("tensors must be contiguous device tensors")
        if t.dtype != dtype:
            raise TypeError(f"expected {dtype}, got {t.dtype}")
        if t.get_device() != dev:                 # -1 for one in host memory
            raise ValueError(f"tensor on {t.device}, but the current device is {dev}")


INT_MAX = 2 ** 31 - 1            # the library's sizes are 32 bits wide, and ctypes cuts a longer one down to them


def _where(dev: int):
    """Context and stream of a launch."""
    return _ctx_by_device.get(dev) or ctx(dev), torch._C._cuda_getCurrentRawStream(dev)


ROTARY_SCALINGS = {"none": 0, "linear": 1, "base": 2, "blend": 3}


class _Fixed:
    """Attributes are set once, at construction: the C view that the calls pass on is made of them there."""

    def __setattr__(self, name, value):
        raise AttributeError(f"{type(self).__name__}.{name} is fixed: make a new {type(self).__name__}")

    def __delattr__(self, name):
        self.__setattr__(name, None)


class RotaryTable(_Fixed):
    """Frequencies of the rotated pairs, on the device (made once, attributes fixed; see smoe_rotary)."""

    def __init__(self, turns: torch.Tensor, rot: int, interleaved: bool, amplitude: float):
        self.__dict__.update(turns=turns, rot=rot, interleaved=interleaved, amplitude=amplitude,
                             _c=ctypes.byref(smoe_rotary(turns.data_ptr(), rot, int(interleaved), amplitude)))


def rotary_table(rot: int, layout: str = "half", base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                 trained_length: float = 4096.0, device=None) -> RotaryTable:
    """Table of a rotation of the first `rot` elements of a row: pairs (i, i + rot/2) for layout "half", (2i, 2i+1) for "interleaved";
    scaling "none", "linear", "base" or "blend" by `factor` (see smoe_rotary_scaling)."""
    if layout not in ("half", "interleaved") or scaling not in ROTARY_SCALINGS:
        raise ValueError(f"layout {layout!r}, scaling {scaling!r}")
    turns = torch.zeros(max(rot, 2) // 2, dtype=torch.int64)
    amplitude = ctypes.c_float(1.0)
    _check(lib.smoe_rotary_frequencies(rot, base, ROTARY_SCALINGS[scaling], factor, trained_length, turns.data_ptr(), ctypes.byref(amplitude)),
           "smoe_rotary_frequencies")
    return RotaryTable(turns.to(torch.device("cuda", torch.cuda.current_device()) if device is None else device), rot, layout == "interleaved",
                       amplitude.value)


def _turn(entry, what, Q, K, table, positions, out):
    dev, dtype = _device(Q), Q.dtype
    _here(dev, dtype, Q)
    shape = Q.shape
    if len(shape) < 3:
        raise ValueError("rows must be [B, T, heads..., d]")
    B, T, d = shape[0], shape[1], shape[-1]
    hq, hk = math.prod(shape[2:-1]), 0
    if table.turns.get_device() != dev:
        raise ValueError(f"table on {table.turns.device}, but the current device is {dev}")
    if K is not None:
        _here(dev, dtype, K)
        like = K.shape
        if len(like) < 3 or like[0] != B or like[1] != T or like[-1] != d:
            raise ValueError("K must be [B, T, heads..., d] like Q")
        hk = math.prod(like[2:-1])
    if (B * T | hq | hk | d) > INT_MAX:           # any of them
        raise ValueError("more rows, heads or elements than 32 bits count")
    if positions is not None:
        _here(dev, torch.int32, positions)
        if positions.numel() != B * T:
            raise ValueError("positions must hold B*T entries")
    if out is None:
        Qr, Kr = _new(*shape, dtype=dtype, device=Q.device), None if K is None else _new(*like, dtype=dtype, device=K.device)
    else:
        Qr, Kr = out
        for t, x in ((Qr, Q), (Kr, K)):
            if (t is None) != (x is None) or (t is not None and t.shape != x.shape):
                raise ValueError("out must be a pair like (Q, K)")
            if t is not None:
                _here(dev, dtype, t)
    c, stream = _where(dev)
    _check(entry(c, stream, _dt(Q), Q.data_ptr(), hq, _p(K), hk, B * T, d, T or 1, _p(positions), table._c, Qr.data_ptr(), _p(Kr)), what)
    return Qr, Kr


def rotary_fwd(Q, K, table: RotaryTable, positions=None, out=None):
    """Q [B, T, ..., d] and K [B, T, ..., d] (or None), F32 or BF16, turned by their positions: positions [B, T] int32, or 0..T-1 of every
    sequence.  out = (Qr, Kr) may be (Q, K) themselves.  Returns (Qr, Kr)."""
    return _turn(lib.smoe_rotary_fwd, "smoe_rotary_fwd", Q, K, table, positions, out)


def rotary_bwd(dQ, dK, table: RotaryTable, positions=None, out=None):
    """Gradient of rotary_fwd: (dQ, dK) of its inputs from those of its outputs."""
    return _turn(lib.smoe_rotary_bwd, "smoe_rotary_bwd", dQ, dK, table, positions, out)


class KVCache(_Fixed):
    """A paged cache of keys and values: K and V [pages, h, page, d_head], bf16, or uint8 holding e4m3 with the rows' exponents
    K_exp and V_exp [pages, h, page] uint8 (see smoe_cache).  The tensors stay the caller's and are written in place; which they are is
    fixed (a larger cache is a new KVCache), and so is where they lie."""

    def __init__(self, K: torch.Tensor, V: torch.Tensor, K_exp: torch.Tensor | None = None, V_exp: torch.Tensor | None = None):
        quantised = K_exp is not None
        for t in (K, V):
            _chk(t, torch.uint8 if quantised else torch.bfloat16)
        if K.dim() != 4 or V.shape != K.shape or (V_exp is not None) != quantised:
            raise ValueError("K and V must be [pages, h, page, d_head], with exponents for both or neither")
        for t in (K_exp, V_exp) if quantised else ():
            _chk(t, torch.uint8)
            if t.shape != K.shape[:3]:
                raise ValueError("exponents must be [pages, h, page]")
        if len({t.device for t in (K, V, K_exp, V_exp) if t is not None}) != 1:
            raise ValueError("the cache's tensors must be on one device")
        pages, h, page, d_head = K.shape
        self.__dict__.update(K=K, V=V, K_exp=K_exp, V_exp=V_exp, pages=pages, h=h, page=page, d_head=d_head, device=K.get_device(),
                             _c=ctypes.byref(smoe_cache(_p(K), _p(V), _p(K_exp), _p(V_exp), pages, page, h, d_head, int(quantised))))


def kv_cache(pages: int, page: int, h: int, d_head: int, quantised: bool = False, device=None) -> KVCache:
    """An empty cache (contents unspecified: positions that were not written are never read)."""
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else device
    K, V = (_new(pages, h, page, d_head, dtype=torch.uint8 if quantised else torch.bfloat16, device=device) for _ in "KV")
    exps = [_new(pages, h, page, dtype=torch.uint8, device=device) for _ in "KV"] if quantised else [None, None]
    return KVCache(K, V, *exps)


def _places(dev: int, cache: KVCache, block_table, lens=None, seqs=None, positions=None):
    """The ctypes view of where rows live, how many sequences the table has and how many rows `seqs` names (None with lens)."""
    if cache.device != dev:
        raise ValueError(f"cache on device {cache.device}, but the current device is {dev}")
    _here(dev, torch.int32, block_table)
    if block_table.dim() != 2:
        raise ValueError("block_table must be [sequences, width]")
    B, width = block_table.shape
    if (B | width) > INT_MAX:                     # either
        raise ValueError("block_table has more sequences or pages than 32 bits count")
    if lens is not None:
        _here(dev, torch.int32, lens)
        if seqs is not None or positions is not None or lens.numel() != B:
            raise ValueError("give lens [sequences], or seqs and positions")
        return ctypes.byref(smoe_places(block_table.data_ptr(), B, width, None, None, lens.data_ptr())), B, None
    if seqs is None or positions is None or seqs.numel() != positions.numel():
        raise ValueError("give lens [sequences], or seqs and positions of the same length")
    _here(dev, torch.int32, seqs, positions)
    return ctypes.byref(smoe_places(block_table.data_ptr(), B, width, seqs.data_ptr(), positions.data_ptr(), None)), B, seqs.numel()


def _rows_of(cache: KVCache, t) -> bool:
    """Does a row of t end as [h, d_head], or as both in one?  (Any other order of as many elements would be read as other rows.)"""
    shape = t.shape
    last = shape[-1]
    return (last == cache.d_head and len(shape) > 1 and shape[-2] == cache.h) or last == cache.h * cache.d_head


def cache_append(cache: KVCache, K, V, block_table, lens=None, seqs=None, positions=None, rotary: RotaryTable | None = None, Q=None, out=None):
    """Writes the rows K, V [rows, h, d_head] (bf16) to the last places of every sequence (lens), or to the listed ones; with `rotary` K is
    turned first, and Q [rows, ..., d_head] into the returned tensor (`out`, which may be Q)."""
    dev = _device(K)
    where, B, rows = _places(dev, cache, block_table, lens, seqs, positions)
    _here(dev, torch.bfloat16, K, V)
    row, n = cache.h * cache.d_head, K.numel()
    M = n // row
    if n != M * row or (M != rows if rows is not None else B == 0 or M % B) or not _rows_of(cache, K) or \
            (V.shape != K.shape and (V.numel() != n or not _rows_of(cache, V))):
        raise ValueError("K and V must be [rows, h, d_head], as many rows for each sequence")
    if rotary is not None and rotary.turns.get_device() != dev:
        raise ValueError(f"table on {rotary.turns.device}, but the current device is {dev}")
    hq, Qr = 0, None
    if Q is not None:
        _here(dev, torch.bfloat16, Q)
        of_q, of_head = Q.numel(), M * cache.d_head
        hq = of_q // max(1, of_head)
        if rotary is None or of_q != of_head * hq or Q.shape[-1] != cache.d_head:
            raise ValueError("Q must be [rows, heads..., d_head], and goes with rotary")
        if out is None:
            Qr = _like(Q)
        else:
            Qr = out
            _here(dev, torch.bfloat16, out)
            if out.shape != Q.shape:
                raise ValueError("out must be like Q")
    ask_q = Q is not None and M > 0       # without rows there is nothing to turn
    c, stream = _where(dev)
    _check(lib.smoe_cache_append(c, stream, BF16, cache._c, where, K.data_ptr(), V.data_ptr(), M, None if rotary is None else rotary._c,
                                 Q.data_ptr() if ask_q else None, hq, Qr.data_ptr() if ask_q else None), "smoe_cache_append")
    return Qr


def cache_read(cache: KVCache, block_table, lens=None, seqs=None, positions=None, N: int = 1, out=None):
    """K, V [rows, h, d_head] (bf16) of the listed places, or of the last N of every sequence (lens)."""
    dev = _device(cache.K)
    where, B, rows = _places(dev, cache, block_table, lens, seqs, positions)
    rows = B * N if rows is None else rows
    if out is None:
        K, V = (_new(rows, cache.h, cache.d_head, dtype=torch.bfloat16, device=cache.K.device) for _ in "KV")
    else:
        K, V = out
        _here(dev, torch.bfloat16, K, V)
        if K.numel() != rows * cache.h * cache.d_head or V.numel() != K.numel() or not _rows_of(cache, K) or not _rows_of(cache, V):
            raise ValueError("out must be two tensors [rows, h, d_head]")
    c, stream = _where(dev)
    _check(lib.smoe_cache_read(c, stream, BF16, cache._c, where, rows, K.data_ptr(), V.data_ptr()), "smoe_cache_read")
    return K, V


def cached_attention_fwd(Q, cache: KVCache, block_table, lens, out=None, ws=None):
    """Q [B, N, G, h, d_head] (bf16), the last N positions of every sequence, over the cache -> O like Q, LSE [B, N, G, h] fp32.
    out = (O, LSE) and ws reuse tensors; O may be Q."""
    dev = _device(Q)
    where, sequences, _ = _places(dev, cache, block_table, lens)
    _here(dev, torch.bfloat16, Q)
    if Q.dim() != 5:
        raise ValueError("Q must be [sequences, N, G, h, d_head]")
    B, N, G, h, d = Q.shape
    if h != cache.h or d != cache.d_head or B != sequences:
        raise ValueError("Q must be [sequences, N, G, h, d_head] with the cache's h and d_head")
    if out is None:
        O, LSE = _new(B, N, G, h, d, dtype=torch.bfloat16, device=Q.device), _new(B, N, G, h, dtype=torch.float32, device=Q.device)
    else:
        O, LSE = out
        _here(dev, torch.bfloat16, O)
        _here(dev, torch.float32, LSE)
        if O.shape != Q.shape or LSE.numel() != B * N * G * h:
            raise ValueError("out must be a tensor like Q and one [B, N, G, h]")
    if ws is None:
        nb = lib.smoe_cached_attention_workspace_bytes(cache._c, where, N, G)
        ws = _ws(nb, Q.device) if nb else None
    else:
        _here(dev, torch.uint8, ws)
    c, stream = _where(dev)
    _check(lib.smoe_cached_attention_fwd(c, stream, BF16, Q.data_ptr(), N, G, cache._c, where, O.data_ptr(), LSE.data_ptr(), _p(ws),
                                         0 if ws is None else ws.numel()), "smoe_cached_attention_fwd")
    return O, LSE


def momha_decode(X, W_K, W_V, W_Q, W_O, r: Routing, k: int, gates, cache: KVCache, block_table, lens, rotary: RotaryTable | None = None,
                 out=None, ws=None):
    """The SMoE attention layer on the last N positions of every sequence, X [B*N, d_model], over a cache that holds the earlier ones and
    receives these; W_K and W_V [d_model, h * d_head], W_Q [E, d_model, h * d_head], W_O [E, h * d_head, d_model].  Returns O [B*N, d_model]."""
    dev = _device(X)
    where, B, _ = _places(dev, cache, block_table, lens)
    _here(dev, torch.bfloat16, X, W_K, W_V, W_Q, W_O)
    _here(dev, torch.float32, gates)
    _here(dev, torch.int32, r.sorted_expert_idxs, r.sorted_scattered_idxs, r.expert_offsets)
    if rotary is not None and rotary.turns.get_device() != dev:
        raise ValueError(f"table on {rotary.turns.device}, but the current device is {dev}")
    M, d_model = X.shape
    d_out = cache.h * cache.d_head
    if B == 0 or M == 0 or M % B or gates.numel() != M * k:
        raise ValueError("X must be [sequences * N, d_model] and gates hold k for each row")
    for W in (W_K, W_V):
        if W.shape != (d_model, d_out) and W.shape != (d_model, cache.h, cache.d_head):
            raise ValueError("W_K and W_V must be [d_model, h * d_head]")
    if W_Q.shape != (r.E, d_model, d_out) or W_O.shape != (r.E, d_out, d_model):
        raise ValueError("weights do not fit d_model and the cache's h * d_head")
    N = M // B
    O = _like(X) if out is None else out
    if out is not None:
        _here(dev, torch.bfloat16, out)
        if out.shape != X.shape:
            raise ValueError("out must be like X")
    if ws is None:
        ws = _ws(lib.smoe_momha_decode_workspace_bytes(B, N, k, d_model, cache.h, cache.d_head), X.device)
    else:
        _here(dev, torch.uint8, ws)
    rc = r.c()
    c, stream = _where(dev)
    _check(lib.smoe_momha_decode(c, stream, BF16, _p(X), N, d_model, _p(W_K), _p(W_V), _p(W_Q), _p(W_O), ctypes.byref(rc), k, _p(gates),
                                 cache._c, where, None if rotary is None else rotary._c, _p(O), _p(ws), ws.numel()), "smoe_momha_decode")
    return O


# ---- the block around the experts (include/smoe_block.h) ------------------------------------------------------------------
def _held(*numbers: int):
    """Numbers that come from the caller as they are: none that 32 bits would cut down to another."""
    for n in numbers:
        if not -INT_MAX <= n <= INT_MAX:
            raise ValueError(f"{n} does not fit 32 bits")


SCORES = {"softmax": 0, "sigmoid": 1}
FLOAT_MAX = (2 - 2.0 ** -23) * 2.0 ** 127


class GateRule(_Fixed):
    """How a router's scores become a choice and weights (attributes fixed; see smoe_gate_rule)."""

    def __init__(self, score: str, groups: int, kept_groups: int, group_best: int, renormalise: bool, scale: float):
        if score not in SCORES:
            raise ValueError(f"score {score!r}")
        _held(groups, kept_groups, group_best)
        if not abs(scale) <= FLOAT_MAX:
            raise ValueError(f"scale {scale} is not a finite number of 32 bits")
        self.__dict__.update(score=score, groups=groups, kept_groups=kept_groups, group_best=group_best, renormalise=renormalise, scale=scale,
                             _c=ctypes.byref(smoe_gate_rule(SCORES[score], groups, kept_groups, group_best, int(renormalise), scale)))


def gate_rule(score: str = "softmax", groups: int = 1, kept_groups: int = 1, group_best: int = 1, renormalise: bool = True, scale: float = 1.0) -> GateRule:
    """Scores "softmax" or "sigmoid"; of `groups` groups of experts the kept_groups whose group_best largest ranks sum to most; weights divided by
    their sum with `renormalise`, times `scale`."""
    return GateRule(score, groups, kept_groups, group_best, renormalise, scale)


def score_gate(logits: torch.Tensor, k: int, rule: GateRule, bias: torch.Tensor | None = None):
    """logits [T, E] fp32, bias [E] fp32 (moves the choice only) -> expert_idxs [T, k] int32, gates [T, k] fp32."""
    dev = _device(logits)
    _here(dev, torch.float32, logits)
    if logits.dim() != 2:
        raise ValueError("logits must be [T, E]")
    T, E = logits.shape
    if (T | E) > INT_MAX or not 0 < k <= E:
        raise ValueError("more tokens or experts than 32 bits count, or k outside 1 .. E")
    if bias is not None:
        _here(dev, torch.float32, bias)
        if bias.numel() != E:
            raise ValueError("bias must be [E]")
    idx, gates = _new(T, k, dtype=torch.int32, device=logits.device), _new(T, k, dtype=torch.float32, device=logits.device)
    c, stream = _where(dev)
    _check(lib.smoe_score_gate(c, stream, logits.data_ptr(), _p(bias), T, E, k, rule._c, idx.data_ptr(), gates.data_ptr()), "smoe_score_gate")
    return idx, gates


def score_gate_bwd(logits: torch.Tensor, expert_idxs: torch.Tensor, dgates: torch.Tensor, rule: GateRule) -> torch.Tensor:
    """dlogits [T, E] from the gradient of score_gate's gates."""
    dev = _device(logits)
    _here(dev, torch.float32, logits, dgates)
    _here(dev, torch.int32, expert_idxs)
    if logits.dim() != 2 or expert_idxs.dim() != 2 or expert_idxs.shape[0] != logits.shape[0] or dgates.shape != expert_idxs.shape:
        raise ValueError("logits must be [T, E], expert_idxs and dgates [T, k]")
    (T, E), k = logits.shape, expert_idxs.shape[1]
    if (T | E | k) > INT_MAX:
        raise ValueError("more tokens or experts than 32 bits count")
    dlogits = _new(T, E, dtype=torch.float32, device=logits.device)
    c, stream = _where(dev)
    _check(lib.smoe_score_gate_bwd(c, stream, logits.data_ptr(), expert_idxs.data_ptr(), dgates.data_ptr(), T, E, k, rule._c, dlogits.data_ptr()),
           "smoe_score_gate_bwd")
    return dlogits


class Rows8(_Fixed):
    """Rows of d elements in 8 bits: values [..., P] and exps [..., P / 32] uint8, P = 128 * ceil(d / 128) (see smoe_rows8).  The tensors stay
    the caller's; which they are is fixed."""

    def __init__(self, values: torch.Tensor, exps: torch.Tensor, d: int):
        for t in (values, exps):
            _chk(t, torch.uint8)
        P = values.shape[-1]
        if not 0 < d <= P or P != -(-d // 128) * 128 or exps.shape != (*values.shape[:-1], P // 32) or exps.device != values.device:
            raise ValueError("rows in 8 bits must be values [..., 128 * ceil(d / 128)] and exps [..., 4 * ceil(d / 128)] on one device")
        self.__dict__.update(values=values, exps=exps, d=d, rows=values.numel() // P, shape=(*values.shape[:-1], d), device=values.get_device(),
                             _c=ctypes.byref(smoe_rows8(_p(values), _p(exps))))


def _new_rows8(shape, device) -> Rows8:
    P = -(-shape[-1] // 128) * 128
    return Rows8(_new(*shape[:-1], P, dtype=torch.uint8, device=device), _new(*shape[:-1], P // 32, dtype=torch.uint8, device=device), shape[-1])


def _rows_on(dev: int, *rows: Rows8):
    for r in rows:
        if r.device != dev:
            raise ValueError(f"rows on device {r.device}, but the current device is {dev}")
        if r.rows > INT_MAX:
            raise ValueError("more rows than 32 bits count")


def _row_sizes(X: torch.Tensor):
    """Rows and width of X [..., d]."""
    d = X.shape[-1] if X.dim() else 0
    rows = X.numel() // d if d else 0
    if X.dim() < 1 or d < 1 or (rows | d) > INT_MAX:
        raise ValueError("rows must be [..., d], as many as 32 bits count")
    return rows, d


def rows8_pack(X: torch.Tensor, out: Rows8 | None = None) -> Rows8:
    """X [..., d] (F32 or BF16) in 8 bits."""
    dev = _device(X)
    _here(dev, X.dtype, X)
    rows, d = _row_sizes(X)
    if out is None:
        out = _new_rows8(X.shape, X.device)
    _rows_on(dev, out)
    if out.rows != rows or out.d != d:
        raise ValueError("out must be rows like X")
    c, stream = _where(dev)
    _check(lib.smoe_rows8_pack(c, stream, _dt(X), X.data_ptr(), rows, d, out._c), "smoe_rows8_pack")
    return out


def rows8_unpack(rows: Rows8, dtype=torch.bfloat16) -> torch.Tensor:
    """The values that rows in 8 bits stand for, [..., d]."""
    dev = _device(rows.values)
    _rows_on(dev, rows)
    X = _new(*rows.shape, dtype=dtype, device=rows.values.device)
    c, stream = _where(dev)
    _check(lib.smoe_rows8_unpack(c, stream, _dt(X), rows._c, rows.rows, rows.d, X.data_ptr()), "smoe_rows8_unpack")
    return X


class Weights8(_Fixed):
    """Weights of E experts [d_in, d_out] in 8 bits, as the products read them (made by weights8; see smoe_weights8)."""

    def __init__(self, values: torch.Tensor, exps: torch.Tensor, E: int, d_in: int, d_out: int, halves: int):
        for t in (values, exps):
            _chk(t, torch.uint8)
        _held(E, d_in, d_out, halves)
        nb = lib.smoe_weights8_bytes(E, d_in, d_out, halves)
        if not nb or values.numel() != nb or exps.numel() * 32 != nb or exps.device != values.device:
            raise ValueError("weights in 8 bits must be values of smoe_weights8_bytes and a 32nd as many exps, on one device")
        self.__dict__.update(values=values, exps=exps, E=E, d_in=d_in, d_out=d_out, halves=halves, device=values.get_device(),
                             _c=ctypes.byref(smoe_weights8(_p(values), _p(exps), E, d_in, d_out, halves)))


def weights8(W: torch.Tensor, halves: int = 1) -> Weights8:
    """W [E, d_in, d_out] (F32 or BF16) in 8 bits, laid out for the products; halves = 2 where the columns are SwiGLU's [gate | up].  Made once."""
    dev = _device(W)
    _here(dev, W.dtype, W)
    if W.dim() != 3 or max(W.shape) > INT_MAX:
        raise ValueError("weights must be [E, d_in, d_out]")
    E, d_in, d_out = W.shape
    _held(halves)
    nb = lib.smoe_weights8_bytes(E, d_in, d_out, halves)
    if not nb:
        raise ValueError(f"no layout for {E} experts of {d_in} x {d_out} in {halves} halves")
    out = Weights8(_new(nb, dtype=torch.uint8, device=W.device), _new(nb // 32, dtype=torch.uint8, device=W.device), E, d_in, d_out, halves)
    c, stream = _where(dev)
    _check(lib.smoe_weights8_pack(c, stream, _dt(W), W.data_ptr(), out._c), "smoe_weights8_pack")
    return out


@dataclass
class Norm:
    """What add_norm_fwd leaves: the stream S that goes on (X itself where nothing was added), Y in its dtype, Y8 in 8 bits, rstd [rows] for the
    backward pass; None for what was not asked for."""
    S: torch.Tensor
    Y: torch.Tensor | None
    Y8: Rows8 | None
    rstd: torch.Tensor


def add_norm_fwd(X: torch.Tensor, weight: torch.Tensor, R: torch.Tensor | None = None, eps: float = 1e-6, plain: bool = True, packed: bool = False,
                 out: Norm | None = None) -> Norm:
    """The root-mean-square norm of X + R [..., d] (F32 or BF16, weight [d] in the same): Y with `plain`, Y8 with `packed`.  `out` reuses the
    tensors of an earlier call; its S, where R is given, may be X or R itself."""
    dev, dtype = _device(X), X.dtype
    _here(dev, dtype, X, weight)
    rows, d = _row_sizes(X)
    if weight.numel() != d:
        raise ValueError("weight must be [d]")
    if not plain and not packed:
        raise ValueError("ask for plain or packed rows, or both")
    if R is not None:
        _here(dev, dtype, R)
        if R.shape != X.shape:
            raise ValueError("R must be like X")
    if out is None:
        out = Norm(X if R is None else _like(X), _like(X) if plain else None, _new_rows8(X.shape, X.device) if packed else None,
                   _new(rows, dtype=torch.float32, device=X.device))
    else:
        _here(dev, dtype, out.S)
        _here(dev, torch.float32, out.rstd)
        if out.S.shape != X.shape or out.rstd.numel() != rows or (out.Y is not None) != plain or (out.Y8 is not None) != packed:
            raise ValueError("out must be what such a call leaves")
        if plain:
            _here(dev, dtype, out.Y)
            if out.Y.shape != X.shape:
                raise ValueError("out must be what such a call leaves")
        if packed:
            _rows_on(dev, out.Y8)
            if out.Y8.rows != rows or out.Y8.d != d:
                raise ValueError("out must be what such a call leaves")
        if R is None and out.S is not X:
            out = Norm(X, out.Y, out.Y8, out.rstd)
    c, stream = _where(dev)
    _check(lib.smoe_add_norm_fwd(c, stream, _dt(X), X.data_ptr(), _p(R), weight.data_ptr(), rows, d, eps, None if R is None else out.S.data_ptr(), _p(out.Y),
                                 out.Y8._c if packed else None, out.rstd.data_ptr()), "smoe_add_norm_fwd")
    return out


def add_norm_bwd(dY: torch.Tensor, S: torch.Tensor, weight: torch.Tensor, rstd: torch.Tensor, dS: torch.Tensor | None = None, out=None, ws=None):
    """(dX, dweight) of add_norm_fwd from the gradients of Y and, where the stream goes on, of S; that of R is dX.  out = (dX, dweight), whose dX
    may be dY, S or dS itself."""
    dev, dtype = _device(dY), dY.dtype
    _here(dev, dtype, dY, S, weight)
    _here(dev, torch.float32, rstd)
    rows, d = _row_sizes(dY)
    if S.shape != dY.shape or weight.numel() != d or rstd.numel() != rows:
        raise ValueError("dY and S must be [..., d], weight [d] and rstd one for each row")
    if dS is not None:
        _here(dev, dtype, dS)
        if dS.shape != dY.shape:
            raise ValueError("dS must be like dY")
    if out is None:
        dX, dweight = _like(dY), _like(weight)
    else:
        dX, dweight = out
        _here(dev, dtype, dX, dweight)
        if dX.shape != dY.shape or dweight.numel() != d:
            raise ValueError("out must be a tensor like dY and one like weight")
    if ws is None:
        ws = _ws(lib.smoe_add_norm_bwd_workspace_bytes(_dt(dY), rows, d), dY.device)
    else:
        _here(dev, torch.uint8, ws)
    c, stream = _where(dev)
    _check(lib.smoe_add_norm_bwd(c, stream, _dt(dY), dY.data_ptr(), _p(dS), S.data_ptr(), weight.data_ptr(), rstd.data_ptr(), rows, d, dX.data_ptr(),
                                 dweight.data_ptr(), ws.data_ptr(), ws.numel()), "smoe_add_norm_bwd")
    return dX, dweight


def _experts8(dev: int, r: Routing, *weights: Weights8):
    _here(dev, torch.int32, r.sorted_expert_idxs, r.sorted_scattered_idxs, r.expert_offsets)
    for w in weights:
        if w.device != dev:
            raise ValueError(f"weights on device {w.device}, but the current device is {dev}")
        if w.E != r.E:
            raise ValueError("weights and routing must be of as many experts")
    if r.sorted_scattered_idxs.numel() < r.Tk or r.expert_offsets.numel() < r.E + 1:
        raise ValueError("routing arrays are too short")


def plinear8_fwd(X: Rows8, W: Weights8, r: Routing, k: int, gates=None, grouped_in=False, grouped_out=False):
    """Alg. 1 on rows and weights in 8 bits, bf16 out.  Returns (Y, Yhat); Y is Yhat when no gates are given."""
    dev = _device(X.values)
    _rows_on(dev, X)
    _experts8(dev, r, W)
    _held(k)
    if X.d != W.d_in:
        raise ValueError("rows and weights differ in d_in")
    Y, gk = None, 0
    Yhat = _new(r.Tk, W.d_out, dtype=torch.bfloat16, device=X.values.device)
    if gates is not None:
        _here(dev, torch.float32, gates)
        gk = gates.shape[-1]
        if gates.numel() != r.Tk:
            raise ValueError("gates must hold one entry for each routed slot")
        Y = _new(r.Tk // gk if gk else 0, W.d_out, dtype=torch.bfloat16, device=X.values.device)
    rc = r.c()
    c, stream = _where(dev)
    _check(lib.smoe_plinear8_fwd(c, stream, X._c, X.rows, X.d, W._c, W.d_out, ctypes.byref(rc), k, _p(gates), gk, int(grouped_in), int(grouped_out),
                                 Yhat.data_ptr(), _p(Y)), "smoe_plinear8_fwd")
    return (Yhat if Y is None else Y), Yhat


def mlp8_fwd(X: Rows8, W1: Weights8, W2: Weights8, r: Routing, k: int, gates, act: int, out=None, ws=None) -> torch.Tensor:
    """Alg. 3's forward pass on rows and weights in 8 bits (W1 of two halves for SwiGLU).  Returns Y [..., d_model] bf16."""
    dev = _device(X.values)
    _rows_on(dev, X)
    _experts8(dev, r, W1, W2)
    _held(k, act)
    _here(dev, torch.float32, gates)
    T, d_model, d_expert = X.rows, X.d, W2.d_in
    if W1.d_in != d_model or W2.d_out != d_model or W1.d_out != hidden_width(act, d_expert) or W1.halves != hidden_width(act, 1) or W2.halves != 1:
        raise ValueError("weights do not fit the rows, one another or the activation")
    if r.Tk != T * k or gates.numel() != T * k:
        raise ValueError("gates and routing must hold k slots for each row")
    if out is None:
        out = _new(*X.shape, dtype=torch.bfloat16, device=X.values.device)
    else:
        _here(dev, torch.bfloat16, out)
        if out.numel() != T * d_model or out.shape[-1] != d_model:
            raise ValueError("out must be [..., d_model] like the rows")
    if ws is None:
        ws = _ws(lib.smoe_mlp8_fwd_workspace_bytes(act, T, k, d_model, d_expert), X.values.device)
    else:
        _here(dev, torch.uint8, ws)
    rc = r.c()
    c, stream = _where(dev)
    _check(lib.smoe_mlp8_fwd(c, stream, act, X._c, T, d_model, d_expert, W1._c, W2._c, ctypes.byref(rc), k, gates.data_ptr(), out.data_ptr(), ws.data_ptr(),
                             ws.numel()), "smoe_mlp8_fwd")
    return out
