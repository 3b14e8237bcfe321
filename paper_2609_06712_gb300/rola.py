"""Thin Python binding of the C ABI in include/rola.h.

Argument marshalling only: every step of the module runs in the CUDA kernels
of librola.so.  Torch tensors supply device memory and the current stream.
Importing this module loads librola.so and raises if it is missing -- there is
no CPU fallback.
"""
from __future__ import annotations

import ctypes
import os

import torch
from torch.autograd.function import once_differentiable

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "librola.so")

ROLA_OK, ROLA_ERR_INVALID_ARG, ROLA_ERR_UNSUPPORTED, ROLA_ERR_WORKSPACE, ROLA_ERR_CUDA, ROLA_ERR_TIMEOUT = range(6)
ROLA_BF16, ROLA_FP32 = 0, 1


class RolaConfig(ctypes.Structure):
    """Mirror of rola_config_t."""
    _fields_ = [
        ("B", ctypes.c_int32), ("H", ctypes.c_int32), ("N", ctypes.c_int32), ("d_h", ctypes.c_int32),
        ("T", ctypes.c_int32), ("Hh", ctypes.c_int32), ("Ww", ctypes.c_int32),
        ("pos_offset", ctypes.c_int32 * 3),
        ("rope_split", ctypes.c_int32 * 3),
        ("rope_theta", ctypes.c_double),
        ("block", ctypes.c_int32),
        ("keep_ratio", ctypes.c_float),
        ("r", ctypes.c_int32),
        ("eps_lr", ctypes.c_float),
        ("eps_fuse", ctypes.c_float),
        ("gate_bias", ctypes.c_float),
        ("dtype", ctypes.c_int32),
        ("wait_limit_ms", ctypes.c_int32),
        ("debug_flags", ctypes.c_int32),
        ("lowrank_rope", ctypes.c_int32),
        ("lowrank_act", ctypes.c_int32),
        ("block_geometry", ctypes.c_int32),
        ("query_block", ctypes.c_int32),
    ]


class RolaFfnConfig(ctypes.Structure):
    """Mirror of rola_ffn_config_t."""
    _fields_ = [(n, ctypes.c_int32) for n in ("tokens", "d_model", "d_ff", "act", "dtype", "wait_limit_ms",
                                              "debug_flags")]


class RolaAttentionConfig(ctypes.Structure):
    """Mirror of rola_attention_config_t."""
    _fields_ = [
        ("B", ctypes.c_int32), ("H", ctypes.c_int32), ("H_kv", ctypes.c_int32),
        ("Lq", ctypes.c_int32), ("Lk", ctypes.c_int32), ("d_h", ctypes.c_int32),
        ("causal", ctypes.c_int32),
        ("scale", ctypes.c_float),
        ("dtype", ctypes.c_int32),
        ("wait_limit_ms", ctypes.c_int32),
        ("debug_flags", ctypes.c_int32),
    ]


class RolaLinearConfig(ctypes.Structure):
    """Mirror of rola_linear_config_t."""
    _fields_ = [(n, ctypes.c_int32) for n in ("tokens", "d_in", "d_out", "act", "dtype", "wait_limit_ms",
                                              "debug_flags")]


class RolaResidualNormConfig(ctypes.Structure):
    """Mirror of rola_residual_norm_config_t."""
    _fields_ = [(n, ctypes.c_int32) for n in ("groups", "rows", "d", "norm", "branch_norm", "mod_stride")] + [
        ("eps", ctypes.c_float)] + [(n, ctypes.c_int32) for n in ("dtype", "wait_limit_ms", "debug_flags")]


ROLA_DEBUG_SKIP_FIRST_K_COPY = 1
# rola_lowrank_rope_t: where the truncated RoPE sits in the low-rank features
ROLA_LOWRANK_ROPE_OUTSIDE, ROLA_LOWRANK_ROPE_INSIDE, ROLA_LOWRANK_ROPE_NONE = 0, 1, 2
# rola_lowrank_act_t: the feature map of the low-rank features, and the names a config dict uses
(ROLA_LOWRANK_ACT_SILU, ROLA_LOWRANK_ACT_IDENTITY, ROLA_LOWRANK_ACT_TANH, ROLA_LOWRANK_ACT_RELU,
 ROLA_LOWRANK_ACT_GELU) = 0, 1, 2, 3, 4
LOWRANK_ACTS = {"silu": ROLA_LOWRANK_ACT_SILU, "identity": ROLA_LOWRANK_ACT_IDENTITY,
                "tanh": ROLA_LOWRANK_ACT_TANH, "relu": ROLA_LOWRANK_ACT_RELU, "gelu": ROLA_LOWRANK_ACT_GELU}
# rola_block_geometry_t: contiguous 64-token chunks, or 4 x 4 x 4 cubes of the latent grid
ROLA_BLOCK_FLAT, ROLA_BLOCK_CUBE = 0, 1
BLOCK_GEOMETRIES = {"flat": ROLA_BLOCK_FLAT, "cube": ROLA_BLOCK_CUBE}
# rola_norm_t: the norms of a residual norm, and the names that its binding takes
ROLA_NORM_NONE, ROLA_NORM_LAYER, ROLA_NORM_RMS = 0, 1, 2
NORMS = {"none": ROLA_NORM_NONE, "layer": ROLA_NORM_LAYER, "rms": ROLA_NORM_RMS}


class RolaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {_lib.rola_status_string(status).decode()}")


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with paper_2609_06712_gb300.build.build() "
                          "(the RoLA module has no CPU fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    P, S = ctypes.c_void_p, ctypes.c_size_t
    I32, I64 = ctypes.c_int32, ctypes.c_int64
    cfgp = ctypes.POINTER(RolaConfig)
    ffnp, attnp = ctypes.POINTER(RolaFfnConfig), ctypes.POINTER(RolaAttentionConfig)
    rnp, linp = ctypes.POINTER(RolaResidualNormConfig), ctypes.POINTER(RolaLinearConfig)
    st = ctypes.c_int
    sig = {
        "rola_config_init": (st, [cfgp]),
        "rola_num_blocks": (ctypes.c_int32, [cfgp]),
        "rola_num_keep": (ctypes.c_int32, [cfgp]),
        "rola_num_query_blocks": (ctypes.c_int32, [cfgp]),
        "rola_workspace_bytes": (S, [cfgp]),
        "rola_block_mask": (st, [cfgp, P, P, P, P, S, P]),
        "rola_sparse_attn": (st, [cfgp, P, P, P, P, P, P, S, P]),
        "rola_lowrank_summary": (st, [cfgp, P, P, P, P, P, P, S, P]),
        "rola_lowrank_summary_static": (st, [cfgp, P, P, P, P, P, P]),
        "rola_lowrank_apply": (st, [cfgp, P, P, P, P, P, P, P, S, P]),
        "rola_forward": (st, [cfgp, P, P, P, P, P, P, P, P, P, S, P]),
        "rola_forward_timed": (st, [cfgp, P, P, P, P, P, P, P, P, P, S, P, P]),
        "rola_forward_train": (st, [cfgp, P, P, P, P, P, P, P, P, P, P, P, P, S, P]),
        "rola_backward_workspace_bytes": (S, [cfgp]),
        "rola_backward": (st, [cfgp] + [P] * 18 + [S, P]),
        "rola_gate": (st, [cfgp, P, P, ctypes.c_float, ctypes.c_int32, P, P]),
        "rola_out_proj": (st, [cfgp, P, P, P, ctypes.c_int32, P, P, S, P]),
        "rola_attention_block": (st, [cfgp, P, P, ctypes.c_float, ctypes.c_int32] + [P] * 12 + [S, P]),
        "rola_layer_norm": (st, [I64, I32, I32, P, P, P, ctypes.c_float, P, P, P, P]),
        "rola_layer_norm_backward_workspace_bytes": (S, [I64, I32, I32]),
        "rola_layer_norm_backward": (st, [I64, I32, I32] + [P] * 9 + [S, P]),
        "rola_ffn_config_init": (st, [ffnp]),
        "rola_ffn_workspace_bytes": (S, [ffnp]),
        "rola_ffn_backward_workspace_bytes": (S, [ffnp]),
        "rola_ffn": (st, [ffnp] + [P] * 6 + [S, P]),
        "rola_ffn_train": (st, [ffnp] + [P] * 8 + [S, P]),
        "rola_ffn_backward": (st, [ffnp] + [P] * 12 + [S, P]),
        "rola_attention_config_init": (st, [attnp]),
        "rola_attention_workspace_bytes": (S, [attnp]),
        "rola_attention_backward_workspace_bytes": (S, [attnp]),
        "rola_attention": (st, [attnp] + [P] * 7 + [S, P]),
        "rola_attention_backward": (st, [attnp] + [P] * 11 + [S, P]),
        "rola_linear_config_init": (st, [linp]),
        "rola_linear_workspace_bytes": (S, [linp]),
        "rola_linear_backward_workspace_bytes": (S, [linp]),
        "rola_linear": (st, [linp] + [P] * 6 + [S, P]),
        "rola_linear_train": (st, [linp] + [P] * 7 + [S, P]),
        "rola_linear_backward": (st, [linp] + [P] * 8 + [S, P]),
        "rola_residual_norm_config_init": (st, [rnp]),
        "rola_residual_norm": (st, [rnp] + [P] * 12),
        "rola_residual_norm_backward_workspace_bytes": (S, [rnp]),
        "rola_residual_norm_backward": (st, [rnp] + [P] * 19 + [S, P]),
        "rola_get_device_status": (st, [P, P]),
        "rola_status_string": (ctypes.c_char_p, [st]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


_lib = _load()


def library():
    """The loaded ctypes library (for tests that call the ABI directly)."""
    return _lib


def make_config(cfg: dict, dtype: int = ROLA_BF16) -> RolaConfig:
    """rola_config_t from a plain dict of layer sizes (see configs.py)."""
    c = RolaConfig()
    _lib.rola_config_init(ctypes.byref(c))
    c.B, c.H, c.N = cfg["B"], cfg["H"], cfg["N"]
    c.d_h = cfg.get("d_h", 128)
    c.T, c.Hh, c.Ww = cfg["T"], cfg["Hh"], cfg["Ww"]
    c.pos_offset[:] = list(cfg.get("pos_offset", (0, 0, 0)))
    c.rope_split[:] = list(cfg.get("rope_split", (44, 42, 42)))
    c.rope_theta = float(cfg.get("rope_theta", 10000.0))
    c.block = cfg.get("block", 64)
    c.keep_ratio = float(cfg["keep"])
    c.r = cfg["r"]
    c.eps_lr = float(cfg.get("eps_lr", 1e-6))
    c.eps_fuse = float(cfg.get("eps_fuse", 1e-6))
    c.gate_bias = float(cfg.get("gate_bias", -1.946))
    c.dtype = dtype
    c.lowrank_rope = int(cfg.get("lowrank_rope", ROLA_LOWRANK_ROPE_OUTSIDE))
    act = cfg.get("lowrank_act", "silu")
    c.lowrank_act = LOWRANK_ACTS[act] if isinstance(act, str) else int(act)
    geom = cfg.get("block_geometry", "flat")
    c.block_geometry = BLOCK_GEOMETRIES[geom] if isinstance(geom, str) else int(geom)
    c.query_block = int(cfg.get("qblock", 0))
    return c


def _p(t):
    if t is None:
        return None
    if not (t.is_cuda and t.is_contiguous()):
        raise ValueError("RoLA tensors must be contiguous CUDA tensors")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _check(status: int, where: str):
    if status != ROLA_OK:
        raise RolaError(status, where)


def num_blocks(c: RolaConfig) -> int:
    return _lib.rola_num_blocks(ctypes.byref(c))


def num_query_blocks(c: RolaConfig) -> int:
    """Rows of kv_idx: 128-token query chunks when c.query_block is 128, else the key blocks."""
    return _lib.rola_num_query_blocks(ctypes.byref(c))


def num_keep(c: RolaConfig) -> int:
    return _lib.rola_num_keep(ctypes.byref(c))


def workspace_bytes(c: RolaConfig) -> int:
    return _lib.rola_workspace_bytes(ctypes.byref(c))


def workspace(c: RolaConfig, device="cuda") -> torch.Tensor:
    """A workspace tensor of rola_workspace_bytes(c) bytes (torch allocations are 256-byte aligned)."""
    n = workspace_bytes(c)
    if n == 0:
        raise RolaError(ROLA_ERR_INVALID_ARG, "rola_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def block_mask(c, q, k, kv_idx, ws, stream=None):
    _check(_lib.rola_block_mask(ctypes.byref(c), _p(q), _p(k), _p(kv_idx), _p(ws), ws.numel(), _stream(stream)),
           "rola_block_mask")


def sparse_attn(c, q, k, v, kv_idx, o_s, ws, stream=None):
    _check(_lib.rola_sparse_attn(ctypes.byref(c), _p(q), _p(k), _p(v), _p(kv_idx), _p(o_s), _p(ws), ws.numel(),
                                 _stream(stream)), "rola_sparse_attn")


def lowrank_summary(c, k, v, P_k, C, z, ws, stream=None):
    _check(_lib.rola_lowrank_summary(ctypes.byref(c), _p(k), _p(v), _p(P_k), _p(C), _p(z), _p(ws), ws.numel(),
                                     _stream(stream)), "rola_lowrank_summary")


def lowrank_summary_static(c, k, v, P_k, C, z, stream=None):
    """The summary with no workspace: scratch lives in the library's static device array."""
    _check(_lib.rola_lowrank_summary_static(ctypes.byref(c), _p(k), _p(v), _p(P_k), _p(C), _p(z),
                                            _stream(stream)), "rola_lowrank_summary_static")


def lowrank_apply(c, q, P_q, C, gate, o_s, o, ws, stream=None):
    _check(_lib.rola_lowrank_apply(ctypes.byref(c), _p(q), _p(P_q), _p(C), _p(gate), _p(o_s), _p(o), _p(ws),
                                   ws.numel(), _stream(stream)), "rola_lowrank_apply")


def forward(c, q, k, v, P_q, P_k, gate, o, kv_idx_out, ws, stream=None):
    _check(_lib.rola_forward(ctypes.byref(c), _p(q), _p(k), _p(v), _p(P_q), _p(P_k), _p(gate), _p(o),
                             _p(kv_idx_out), _p(ws), ws.numel(), _stream(stream)), "rola_forward")


def forward_train(c, q, k, v, P_q, P_k, gate, o, kv_idx_out, o_s, lse, C, ws, stream=None):
    """rola_forward keeping O^s, the per-row log-sum-exp and C for backward()."""
    _check(_lib.rola_forward_train(ctypes.byref(c), _p(q), _p(k), _p(v), _p(P_q), _p(P_k), _p(gate), _p(o),
                                   _p(kv_idx_out), _p(o_s), _p(lse), _p(C), _p(ws), ws.numel(), _stream(stream)),
           "rola_forward_train")


def backward_workspace(c: RolaConfig, device="cuda") -> torch.Tensor:
    n = _lib.rola_backward_workspace_bytes(ctypes.byref(c))
    if n == 0:
        raise RolaError(ROLA_ERR_UNSUPPORTED, "rola_backward_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def backward(c, q, k, v, P_q, P_k, gate, kv_idx, o_s, lse, C, dO, dq, dk, dv, dP_q, dP_k, dgate, ws, stream=None):
    _check(_lib.rola_backward(ctypes.byref(c), _p(q), _p(k), _p(v), _p(P_q), _p(P_k), _p(gate), _p(kv_idx),
                              _p(o_s), _p(lse), _p(C), _p(dO), _p(dq), _p(dk), _p(dv), _p(dP_q), _p(dP_k),
                              _p(dgate), _p(ws), ws.numel(), _stream(stream)), "rola_backward")


def gate(c, X, w_g, b_g: float, gate_out, stream=None):
    """Token gate g = sigmoid(X w_g + b_g) into gate_out (fp32 [B][N]); X [B][N][d_model]."""
    _check(_lib.rola_gate(ctypes.byref(c), _p(X), _p(w_g), float(b_g), int(X.shape[-1]), _p(gate_out),
                          _stream(stream)), "rola_gate")


def out_proj(c, O, W_o, b_o, Y, ws, stream=None):
    """Y = concat_h(O) W_o^T (+ b_o): O [B][H][N][128], W_o [d_model][H*128], b_o fp32 [d_model] or
    None, Y [B][N][d_model] (the block's output projection)."""
    _check(_lib.rola_out_proj(ctypes.byref(c), _p(O), _p(W_o), _p(b_o), int(W_o.shape[0]), _p(Y), _p(ws),
                              ws.numel(), _stream(stream)), "rola_out_proj")


def attention_block(c, X, w_g, b_g: float, q, k, v, P_q, P_k, W_o, b_o, gate, o, Y, kv_idx_out, ws, stream=None):
    """The block after the QKV projection: gate from X, the RoLA module, the output projection."""
    _check(_lib.rola_attention_block(ctypes.byref(c), _p(X), _p(w_g), float(b_g), int(X.shape[-1]), _p(q), _p(k),
                                     _p(v), _p(P_q), _p(P_k), _p(W_o), _p(b_o), _p(gate), _p(o), _p(Y),
                                     _p(kv_idx_out), _p(ws), ws.numel(), _stream(stream)), "rola_attention_block")


def forward_timed(c, q, k, v, P_q, P_k, gate, o, kv_idx_out, ws, events, stream=None):
    """rola_forward recording 5 stage events (torch.cuda.Event, already created)."""
    arr = (ctypes.c_void_p * 5)(*[ctypes.c_void_p(e.cuda_event) for e in events])
    _check(_lib.rola_forward_timed(ctypes.byref(c), _p(q), _p(k), _p(v), _p(P_q), _p(P_k), _p(gate), _p(o),
                                   _p(kv_idx_out), _p(ws), ws.numel(), _stream(stream), arr),
           "rola_forward_timed")


# ---------------------------------------------------------------- the block around the module

_DTYPES = {torch.bfloat16: ROLA_BF16, torch.float32: ROLA_FP32}
_TORCH_DTYPES = {v: k for k, v in _DTYPES.items()}


def _dtype_of(t, where: str) -> int:
    if t.dtype not in _DTYPES:
        raise ValueError(f"{where}: tensors must be bfloat16 or float32, not {t.dtype}")
    return _DTYPES[t.dtype]


def _gpu(t, where: str, name: str) -> int:
    """The number of the GPU that the call's first tensor is on, where all the others have to be."""
    dev = -1 if t is None else t.get_device()
    if dev < 0:
        raise ValueError(f"{where}: {name} must be a CUDA tensor")
    return dev


def _a(t, dtype, shape, where: str, name: str, dev: int):
    """The address of tensor `t` (None: NULL, which the library judges), checked against its dtype, shape and GPU."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != dev:
        raise ValueError(f"{where}: {name} must be a contiguous tensor on GPU {dev}, {dtype} of shape {tuple(shape)}, "
                         f"not {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _bytes(n: int, where: str, device) -> torch.Tensor:
    if n == 0:
        raise RolaError(ROLA_ERR_INVALID_ARG, where)
    return torch.empty(n, dtype=torch.uint8, device=device)


def _ws(ws, where: str, dev: int):
    return _a(ws, torch.uint8, ws.shape, where, "ws", dev), ws.numel()


def _run(fn, where: str, dev: int, stream, *args):
    """fn(*args, stream) with GPU `dev` current, which the library launches on; stream None: its current one."""
    if stream is not None and stream.device_index != dev:
        raise ValueError(f"{where}: the stream is on GPU {stream.device_index}, the tensors on GPU {dev}")
    handle = torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream
    if torch._C._cuda_getDevice() == dev:
        st = fn(*args, handle)
    else:
        with torch.cuda.device(dev):
            st = fn(*args, handle)
    if st:
        raise RolaError(st, where)


_F32 = torch.float32


def layer_norm(x, gamma, beta, eps: float, y, mean=None, rstd=None, stream=None):
    """y = (x - mean) rstd gamma + beta over the last axis of x; gamma and beta [d] in x's dtype or None.
    mean and rstd (fp32, one per row), if given, receive what layer_norm_backward reads."""
    w, dt, shape = "rola_layer_norm", x.dtype, x.shape
    d, code = shape[-1], _dtype_of(x, "rola_layer_norm")
    dev = _gpu(x, w, "x")
    _run(_lib.rola_layer_norm, w, dev, stream, x.numel() // max(d, 1), d, code, _a(x, dt, shape, w, "x", dev),
         _a(gamma, dt, (d,), w, "gamma", dev), _a(beta, dt, (d,), w, "beta", dev), eps, _a(y, dt, shape, w, "y", dev),
         _a(mean, _F32, shape[:-1], w, "mean", dev), _a(rstd, _F32, shape[:-1], w, "rstd", dev))


def layer_norm_backward_workspace(x) -> torch.Tensor:
    w, d = "rola_layer_norm_backward_workspace_bytes", x.shape[-1]
    return _bytes(_lib.rola_layer_norm_backward_workspace_bytes(x.numel() // max(d, 1), d, _dtype_of(x, w)), w, x.device)


def layer_norm_backward(x, gamma, mean, rstd, dy, dx, dgamma, dbeta, ws, stream=None):
    """dx of layer_norm, and dgamma, dbeta (fp32 [d], or both None)."""
    w, dt, shape = "rola_layer_norm_backward", x.dtype, x.shape
    d, code = shape[-1], _dtype_of(x, "rola_layer_norm_backward")
    dev = _gpu(x, w, "x")
    _run(_lib.rola_layer_norm_backward, w, dev, stream, x.numel() // max(d, 1), d, code,
         _a(x, dt, shape, w, "x", dev), _a(gamma, dt, (d,), w, "gamma", dev),
         _a(mean, _F32, shape[:-1], w, "mean", dev), _a(rstd, _F32, shape[:-1], w, "rstd", dev),
         _a(dy, dt, shape, w, "dy", dev), _a(dx, dt, shape, w, "dx", dev), _a(dgamma, _F32, (d,), w, "dgamma", dev),
         _a(dbeta, _F32, (d,), w, "dbeta", dev), *_ws(ws, w, dev))


def make_ffn_config(tokens: int, d_model: int, d_ff: int, act="silu", dtype: int = ROLA_BF16) -> RolaFfnConfig:
    """rola_ffn_config_t of a gated feed-forward; act is a name in LOWRANK_ACTS or its number."""
    c = RolaFfnConfig()
    _lib.rola_ffn_config_init(ctypes.byref(c))
    c.tokens, c.d_model, c.d_ff, c.dtype = tokens, d_model, d_ff, dtype
    c.act = LOWRANK_ACTS[act] if isinstance(act, str) else int(act)
    return c


def ffn_workspace(c: RolaFfnConfig, device="cuda") -> torch.Tensor:
    return _bytes(_lib.rola_ffn_workspace_bytes(c), "rola_ffn_workspace_bytes", device)


def ffn_backward_workspace(c: RolaFfnConfig, device="cuda") -> torch.Tensor:
    return _bytes(_lib.rola_ffn_backward_workspace_bytes(c), "rola_ffn_backward_workspace_bytes", device)


def ffn(c, X, W_gate, W_up, W_down, Y, ws, stream=None):
    """Y = (phi(X W_gate^T) * (X W_up^T)) W_down^T; X, Y [tokens][d_model], weights in the nn.Linear layout."""
    w, dt, m, d, f = "rola_ffn", _TORCH_DTYPES.get(c.dtype), c.tokens, c.d_model, c.d_ff
    dev = _gpu(X, w, "X")
    _run(_lib.rola_ffn, w, dev, stream, c, _a(X, dt, (m, d), w, "X", dev), _a(W_gate, dt, (f, d), w, "W_gate", dev),
         _a(W_up, dt, (f, d), w, "W_up", dev), _a(W_down, dt, (d, f), w, "W_down", dev),
         _a(Y, dt, (m, d), w, "Y", dev), *_ws(ws, w, dev))


def ffn_train(c, X, W_gate, W_up, W_down, Y, G, U, ws, stream=None):
    """ffn keeping G = X W_gate^T and U = X W_up^T (fp32 [tokens][d_ff]) for ffn_backward."""
    w, dt, m, d, f = "rola_ffn_train", _TORCH_DTYPES.get(c.dtype), c.tokens, c.d_model, c.d_ff
    dev = _gpu(X, w, "X")
    _run(_lib.rola_ffn_train, w, dev, stream, c, _a(X, dt, (m, d), w, "X", dev),
         _a(W_gate, dt, (f, d), w, "W_gate", dev), _a(W_up, dt, (f, d), w, "W_up", dev),
         _a(W_down, dt, (d, f), w, "W_down", dev), _a(Y, dt, (m, d), w, "Y", dev), _a(G, _F32, (m, f), w, "G", dev),
         _a(U, _F32, (m, f), w, "U", dev), *_ws(ws, w, dev))


def ffn_backward(c, X, W_gate, W_up, W_down, G, U, dY, dX, dW_gate, dW_up, dW_down, ws, stream=None):
    """Gradients of ffn_train: dX and the three weights', in the weights' dtype."""
    w, dt, m, d, f = "rola_ffn_backward", _TORCH_DTYPES.get(c.dtype), c.tokens, c.d_model, c.d_ff
    dev = _gpu(X, w, "X")
    _run(_lib.rola_ffn_backward, w, dev, stream, c, _a(X, dt, (m, d), w, "X", dev),
         _a(W_gate, dt, (f, d), w, "W_gate", dev), _a(W_up, dt, (f, d), w, "W_up", dev),
         _a(W_down, dt, (d, f), w, "W_down", dev), _a(G, _F32, (m, f), w, "G", dev), _a(U, _F32, (m, f), w, "U", dev),
         _a(dY, dt, (m, d), w, "dY", dev), _a(dX, dt, (m, d), w, "dX", dev),
         _a(dW_gate, dt, (f, d), w, "dW_gate", dev), _a(dW_up, dt, (f, d), w, "dW_up", dev),
         _a(dW_down, dt, (d, f), w, "dW_down", dev), *_ws(ws, w, dev))


def make_attention_config(B: int, H: int, H_kv: int, Lq: int, Lk: int, causal: bool = False, scale: float = 0.0,
                          dtype: int = ROLA_BF16) -> RolaAttentionConfig:
    """rola_attention_config_t; scale 0 is 1 / sqrt(d_h)."""
    c = RolaAttentionConfig()
    _lib.rola_attention_config_init(ctypes.byref(c))
    c.B, c.H, c.H_kv, c.Lq, c.Lk, c.causal, c.scale, c.dtype = B, H, H_kv, Lq, Lk, int(causal), scale, dtype
    return c


def attention_workspace(c: RolaAttentionConfig, device="cuda") -> torch.Tensor:
    return _bytes(_lib.rola_attention_workspace_bytes(c), "rola_attention_workspace_bytes", device)


def attention_backward_workspace(c: RolaAttentionConfig, device="cuda") -> torch.Tensor:
    return _bytes(_lib.rola_attention_backward_workspace_bytes(c), "rola_attention_backward_workspace_bytes", device)


def attention(c, q, k, v, kv_len, o, lse, ws, stream=None):
    """o = softmax(scale q k^T) v over the first kv_len[b] keys (int32 [B]; None: all), causal if c.causal;
    q, o [B][H][Lq][128], k, v [B][H_kv][Lk][128].  lse (fp32 [B][H][Lq]) is what attention_backward reads."""
    w, dt = "rola_attention", _TORCH_DTYPES.get(c.dtype)
    rows, keys = (c.B, c.H, c.Lq, c.d_h), (c.B, c.H_kv, c.Lk, c.d_h)
    dev = _gpu(q, w, "q")
    _run(_lib.rola_attention, w, dev, stream, c, _a(q, dt, rows, w, "q", dev), _a(k, dt, keys, w, "k", dev),
         _a(v, dt, keys, w, "v", dev), _a(kv_len, torch.int32, rows[:1], w, "kv_len", dev),
         _a(o, dt, rows, w, "o", dev), _a(lse, _F32, rows[:3], w, "lse", dev), *_ws(ws, w, dev))


def attention_backward(c, q, k, v, kv_len, o, lse, dO, dq, dk, dv, ws, stream=None):
    """Gradients of attention from its o and lse; the probabilities are recomputed."""
    w, dt = "rola_attention_backward", _TORCH_DTYPES.get(c.dtype)
    rows, keys = (c.B, c.H, c.Lq, c.d_h), (c.B, c.H_kv, c.Lk, c.d_h)
    dev = _gpu(q, w, "q")
    _run(_lib.rola_attention_backward, w, dev, stream, c, _a(q, dt, rows, w, "q", dev), _a(k, dt, keys, w, "k", dev),
         _a(v, dt, keys, w, "v", dev), _a(kv_len, torch.int32, rows[:1], w, "kv_len", dev),
         _a(o, dt, rows, w, "o", dev), _a(lse, _F32, rows[:3], w, "lse", dev), _a(dO, dt, rows, w, "dO", dev),
         _a(dq, dt, rows, w, "dq", dev), _a(dk, dt, keys, w, "dk", dev), _a(dv, dt, keys, w, "dv", dev),
         *_ws(ws, w, dev))


def make_linear_config(tokens: int, d_in: int, d_out: int, act="identity", dtype: int = ROLA_BF16) -> RolaLinearConfig:
    """rola_linear_config_t; act is a name in LOWRANK_ACTS or its number."""
    c = RolaLinearConfig()
    _lib.rola_linear_config_init(ctypes.byref(c))
    c.tokens, c.d_in, c.d_out, c.dtype = tokens, d_in, d_out, dtype
    c.act = LOWRANK_ACTS[act] if isinstance(act, str) else int(act)
    return c


def linear_workspace(c: RolaLinearConfig, device="cuda") -> torch.Tensor:
    return _bytes(_lib.rola_linear_workspace_bytes(c), "rola_linear_workspace_bytes", device)


def linear_backward_workspace(c: RolaLinearConfig, device="cuda") -> torch.Tensor:
    return _bytes(_lib.rola_linear_backward_workspace_bytes(c), "rola_linear_backward_workspace_bytes", device)


def linear(c, X, W, b, residual, Y, ws, stream=None):
    """Y = residual + phi(X W^T + b); X [tokens][d_in], W [d_out][d_in], b [d_out] or None, residual (or None) and
    Y [tokens][d_out]; Y may be residual."""
    w, dt, m, k, n = "rola_linear", _TORCH_DTYPES.get(c.dtype), c.tokens, c.d_in, c.d_out
    dev = _gpu(X, w, "X")
    _run(_lib.rola_linear, w, dev, stream, c, _a(X, dt, (m, k), w, "X", dev), _a(W, dt, (n, k), w, "W", dev),
         _a(b, dt, (n,), w, "b", dev), _a(residual, dt, (m, n), w, "residual", dev), _a(Y, dt, (m, n), w, "Y", dev),
         *_ws(ws, w, dev))


def linear_train(c, X, W, b, residual, Y, Z, ws, stream=None):
    """linear keeping Z = X W^T + b (fp32 [tokens][d_out]; None with the identity) for linear_backward."""
    w, dt, m, k, n = "rola_linear_train", _TORCH_DTYPES.get(c.dtype), c.tokens, c.d_in, c.d_out
    dev = _gpu(X, w, "X")
    _run(_lib.rola_linear_train, w, dev, stream, c, _a(X, dt, (m, k), w, "X", dev), _a(W, dt, (n, k), w, "W", dev),
         _a(b, dt, (n,), w, "b", dev), _a(residual, dt, (m, n), w, "residual", dev), _a(Y, dt, (m, n), w, "Y", dev),
         _a(Z, _F32, (m, n), w, "Z", dev), *_ws(ws, w, dev))


def linear_backward(c, X, W, Z, dY, dX, dW, db, ws, stream=None):
    """Gradients of linear_train: dX and dW in the tensors' dtype, db (fp32 [d_out]); each may be None (not wanted).  The
    residual's is dY."""
    w, dt, m, k, n = "rola_linear_backward", _TORCH_DTYPES.get(c.dtype), c.tokens, c.d_in, c.d_out
    dev = _gpu(X, w, "X")
    _run(_lib.rola_linear_backward, w, dev, stream, c, _a(X, dt, (m, k), w, "X", dev), _a(W, dt, (n, k), w, "W", dev),
         _a(Z, _F32, (m, n), w, "Z", dev), _a(dY, dt, (m, n), w, "dY", dev), _a(dX, dt, (m, k), w, "dX", dev),
         _a(dW, dt, (n, k), w, "dW", dev), _a(db, _F32, (n,), w, "db", dev), *_ws(ws, w, dev))


def make_residual_norm_config(groups: int, rows: int, d: int, norm="layer", branch_norm="none", eps: float = 1e-6,
                              mod_stride: int = 0, dtype: int = ROLA_BF16) -> RolaResidualNormConfig:
    """rola_residual_norm_config_t; the norms are names in NORMS or their numbers, mod_stride 0 is d."""
    c = RolaResidualNormConfig()
    _lib.rola_residual_norm_config_init(ctypes.byref(c))
    c.groups, c.rows, c.d, c.eps, c.mod_stride, c.dtype = groups, rows, d, eps, mod_stride, dtype
    c.norm, c.branch_norm = (NORMS[n] if isinstance(n, str) else int(n) for n in (norm, branch_norm))
    return c


def residual_norm_backward_workspace(c: RolaResidualNormConfig, device="cuda") -> torch.Tensor:
    return _bytes(_lib.rola_residual_norm_backward_workspace_bytes(c), "rola_residual_norm_backward_workspace_bytes", device)


def _mod(t, shape, apart: int, dt, where: str, name: str, dev: int):
    """The address of a vector of each sample, of shape (groups, d), whose samples are `apart` elements from each other."""
    if t is None:
        return None
    if t.dtype is not dt or t.shape != shape or t.get_device() != dev or (
            t.stride() != (apart, 1) and ((shape[0] > 1 and t.stride(0) != apart) or (shape[1] > 1 and t.stride(1) != 1))):
        raise ValueError(f"{where}: {name} must be a tensor on GPU {dev}, {dt} of shape {shape} with strides "
                         f"{(apart, 1)}, not {t.dtype} {tuple(t.shape)} with {t.stride()} on {t.device}")
    return t.data_ptr()


def residual_norm(c, x, h, out, y, *, gate=None, gamma_h=None, gamma=None, beta=None, scale=None, shift=None, stats=None,
                  stream=None):
    """out = x + gate a with a = h or norm_b(h) gamma_h, and y = (norm(out) gamma + beta) (1 + scale) + shift.
    x, h, out, y [groups][rows][d]; gate, scale, shift [groups][d] with c.mod_stride between the samples; gamma_h, gamma,
    beta [d]; every vector may be None.  h and out None: the norm of x; y None: no norm.  stats (fp32
    [groups][rows][4]), if given, receives what residual_norm_backward reads."""
    w, dt, B, n, width = "rola_residual_norm", _TORCH_DTYPES.get(c.dtype), c.groups, c.rows, c.d
    shape, per, d, apart = (B, n, width), (B, width), (width,), c.mod_stride or width
    dev = _gpu(x, w, "x")
    _run(_lib.rola_residual_norm, w, dev, stream, c, _a(x, dt, shape, w, "x", dev), _a(h, dt, shape, w, "h", dev),
         _mod(gate, per, apart, dt, w, "gate", dev), _a(gamma_h, dt, d, w, "gamma_h", dev), _a(gamma, dt, d, w, "gamma", dev),
         _a(beta, dt, d, w, "beta", dev), _mod(scale, per, apart, dt, w, "scale", dev), _mod(shift, per, apart, dt, w, "shift", dev),
         _a(out, dt, shape, w, "out", dev), _a(y, dt, shape, w, "y", dev),
         _a(stats, _F32, shape[:2] + (4,), w, "stats", dev))


def residual_norm_backward(c, x, h, stats, dout, dy, dx, dh, ws, *, gate=None, gamma_h=None, gamma=None, beta=None,
                           scale=None, dgate=None, dgamma_h=None, dgamma=None, dbeta=None, dscale=None, dshift=None,
                           stream=None):
    """dx, dh of residual_norm from the gradients dout and dy of its results (None: 0 / no y), and those of its vectors
    (fp32, dense, in the vectors' shapes; None: not wanted)."""
    w, dt, B, n, width = "rola_residual_norm_backward", _TORCH_DTYPES.get(c.dtype), c.groups, c.rows, c.d
    shape, per, d, apart = (B, n, width), (B, width), (width,), c.mod_stride or width
    dev = _gpu(x, w, "x")
    _run(_lib.rola_residual_norm_backward, w, dev, stream, c, _a(x, dt, shape, w, "x", dev), _a(h, dt, shape, w, "h", dev),
         _mod(gate, per, apart, dt, w, "gate", dev), _a(gamma_h, dt, d, w, "gamma_h", dev), _a(gamma, dt, d, w, "gamma", dev),
         _a(beta, dt, d, w, "beta", dev), _mod(scale, per, apart, dt, w, "scale", dev),
         _a(stats, _F32, shape[:2] + (4,), w, "stats", dev), _a(dout, dt, shape, w, "dout", dev),
         _a(dy, dt, shape, w, "dy", dev), _a(dx, dt, shape, w, "dx", dev), _a(dh, dt, shape, w, "dh", dev),
         _a(dgate, _F32, per, w, "dgate", dev), _a(dgamma_h, _F32, d, w, "dgamma_h", dev),
         _a(dgamma, _F32, d, w, "dgamma", dev), _a(dbeta, _F32, d, w, "dbeta", dev),
         _a(dscale, _F32, per, w, "dscale", dev), _a(dshift, _F32, per, w, "dshift", dev), *_ws(ws, w, dev))


def get_device_status(ws, stream=None) -> int:
    p = _p(ws)
    with torch.cuda.device(ws.device):
        return _lib.rola_get_device_status(p, _stream(stream))


class RoLAAttention:
    """Convenience wrapper: owns the workspace for one layer shape and runs rola_forward.

    ``__call__(q, k, v, P_q, P_k, gate=None)`` returns (o, kv_idx) as new tensors."""

    def __init__(self, cfg: dict, dtype: int = ROLA_BF16, device="cuda"):
        self.cfg = make_config(cfg, dtype)
        self.ws = workspace(self.cfg, device)
        self.nB = num_blocks(self.cfg)
        self.n_keep = num_keep(self.cfg)

    def __call__(self, q, k, v, P_q, P_k, gate=None, out=None, kv_idx=None, stream=None):
        c = self.cfg
        if out is None:
            out = torch.empty_like(q)
        if kv_idx is None:
            kv_idx = torch.empty((c.B, c.H, self.nB, self.n_keep), dtype=torch.int32, device=q.device)
        forward(c, q, k, v, P_q, P_k, gate, out, kv_idx, self.ws, stream)
        return out, kv_idx


class RoLAFunction(torch.autograd.Function):
    """The module as a differentiable torch op on this library's kernels:
    rola_forward_train in forward, rola_backward in backward (torch allocates the
    buffers and casts the fp32 P gradients to P's dtype; it computes nothing else).

    ``RoLAFunction.apply(c, q, k, v, P_q, P_k, gate)`` returns O; ``gate`` may be None."""

    @staticmethod
    def forward(ctx, c, q, k, v, P_q, P_k, gate):
        B, H, N = c.B, c.H, c.N
        dev = q.device
        ws = workspace(c, dev)
        o = torch.empty_like(q)
        o_s = torch.empty_like(q)
        kv = torch.empty((B, H, num_blocks(c), num_keep(c)), dtype=torch.int32, device=dev)
        lse = torch.empty((B, H, N), dtype=torch.float32, device=dev)
        C = torch.empty((B, H, c.r, 128), dtype=torch.float32, device=dev)
        forward_train(c, q, k, v, P_q, P_k, gate, o, kv, o_s, lse, C, ws)
        ctx.c = c
        ctx.has_gate = gate is not None
        ctx.save_for_backward(q, k, v, P_q, P_k, gate if gate is not None else torch.empty(0, device=dev),
                              kv, o_s, lse, C)
        return o

    @staticmethod
    @once_differentiable
    def backward(ctx, dO):
        q, k, v, P_q, P_k, gate, kv, o_s, lse, C = ctx.saved_tensors
        c = ctx.c
        gate = gate if ctx.has_gate else None
        dO = dO.contiguous()
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        dP_q = torch.empty(P_q.shape, dtype=torch.float32, device=q.device)
        dP_k = torch.empty(P_k.shape, dtype=torch.float32, device=q.device)
        dgate = torch.empty((c.B, c.N), dtype=torch.float32, device=q.device) if ctx.has_gate else None
        ws = backward_workspace(c, q.device)
        backward(c, q, k, v, P_q, P_k, gate, kv, o_s, lse, C, dO, dq, dk, dv, dP_q, dP_k, dgate, ws)
        return None, dq, dk, dv, dP_q.to(P_q.dtype), dP_k.to(P_k.dtype), dgate



class LayerNormFunction(torch.autograd.Function):
    """Layer norm over the last axis as a differentiable torch op: ``apply(x, gamma, beta, eps)``;
    gamma and beta are both tensors or both None."""

    @staticmethod
    def forward(ctx, x, gamma, beta, eps):
        if (gamma is None) != (beta is None):
            raise ValueError("LayerNormFunction: gamma and beta are both tensors or both None")
        x = x.contiguous()
        y = torch.empty_like(x)
        mean, rstd = (torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device) for _ in range(2))
        layer_norm(x, gamma, beta, eps, y, mean, rstd)
        ctx.save_for_backward(x, gamma, mean, rstd)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, gamma, mean, rstd = ctx.saved_tensors
        dx, dgamma, dbeta = torch.empty_like(x), None, None
        if gamma is not None:
            dgamma, dbeta = (torch.empty_like(gamma, dtype=torch.float32) for _ in range(2))
        layer_norm_backward(x, gamma, mean, rstd, dy.contiguous(), dx, dgamma, dbeta, layer_norm_backward_workspace(x))
        if gamma is not None:
            dgamma, dbeta = dgamma.to(gamma.dtype), dbeta.to(gamma.dtype)
        return dx, dgamma, dbeta, None


class FfnFunction(torch.autograd.Function):
    """The gated feed-forward as a differentiable torch op: ``apply(X, W_gate, W_up, W_down, act)``;
    X [..., d_model]."""

    @staticmethod
    def forward(ctx, X, W_gate, W_up, W_down, act):
        x = X.contiguous().view(-1, X.shape[-1])
        c = make_ffn_config(x.shape[0], x.shape[1], W_gate.shape[0], act, _dtype_of(x, "rola_ffn"))
        Y = torch.empty_like(x)
        G, U = (torch.empty((c.tokens, c.d_ff), dtype=torch.float32, device=x.device) for _ in range(2))
        ffn_train(c, x, W_gate, W_up, W_down, Y, G, U, ffn_workspace(c, x.device))
        ctx.c = c
        ctx.save_for_backward(x, W_gate, W_up, W_down, G, U)
        return Y.view(X.shape)

    @staticmethod
    @once_differentiable
    def backward(ctx, dY):
        x, W_gate, W_up, W_down, G, U = ctx.saved_tensors
        dX, dWg, dWu, dWd = (torch.empty_like(t) for t in (x, W_gate, W_up, W_down))
        ffn_backward(ctx.c, x, W_gate, W_up, W_down, G, U, dY.contiguous().view_as(x), dX, dWg, dWu, dWd,
                     ffn_backward_workspace(ctx.c, x.device))
        return dX.view(dY.shape), dWg, dWu, dWd, None


class AttentionFunction(torch.autograd.Function):
    """Attention over a dense key set as a differentiable torch op: ``apply(q, k, v, kv_len, causal)``;
    kv_len int32 [B] or None."""

    @staticmethod
    def forward(ctx, q, k, v, kv_len, causal):
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        B, H, Lq, _ = q.shape
        c = make_attention_config(B, H, k.shape[1], Lq, k.shape[2], causal, dtype=_dtype_of(q, "rola_attention"))
        o, lse = torch.empty_like(q), torch.empty((B, H, Lq), dtype=torch.float32, device=q.device)
        attention(c, q, k, v, kv_len, o, lse, attention_workspace(c, q.device))
        ctx.c = c
        ctx.save_for_backward(q, k, v, kv_len, o, lse)
        return o

    @staticmethod
    @once_differentiable
    def backward(ctx, dO):
        q, k, v, kv_len, o, lse = ctx.saved_tensors
        dq, dk, dv = (torch.empty_like(t) for t in (q, k, v))
        attention_backward(ctx.c, q, k, v, kv_len, o, lse, dO.contiguous(), dq, dk, dv,
                           attention_backward_workspace(ctx.c, q.device))
        return dq, dk, dv, None, None


class LinearFunction(torch.autograd.Function):
    """A linear layer with its epilogue as a differentiable torch op: ``apply(X, W, b, residual, act)``;
    X [..., d_in], residual [..., d_out] or [tokens, d_out]; b and residual may be None."""

    @staticmethod
    def forward(ctx, X, W, b, residual, act):
        x, W = X.contiguous().view(-1, X.shape[-1]), W.contiguous()
        shapes = (*X.shape[:-1], W.shape[0]), (x.shape[0], W.shape[0])
        if residual is not None and residual.shape not in shapes:    # another order of the tokens has as many elements
            raise ValueError(f"rola_linear: residual must be {shapes[0]} or {shapes[1]}, not {tuple(residual.shape)}")
        c = make_linear_config(x.shape[0], x.shape[1], W.shape[0], act, _dtype_of(x, "rola_linear"))
        Y = torch.empty((c.tokens, c.d_out), dtype=x.dtype, device=x.device)
        Z = None
        if c.act != ROLA_LOWRANK_ACT_IDENTITY:
            Z = torch.empty((c.tokens, c.d_out), dtype=torch.float32, device=x.device)
        r = None if residual is None else residual.contiguous().view(-1, residual.shape[-1])
        linear_train(c, x, W, None if b is None else b.contiguous(), r, Y, Z, linear_workspace(c, x.device))
        ctx.c, ctx.bias_dtype = c, None if b is None else b.dtype
        ctx.residual_shape = None if residual is None else residual.shape
        ctx.save_for_backward(x, W, Z)
        return Y.view(*X.shape[:-1], c.d_out)

    @staticmethod
    @once_differentiable
    def backward(ctx, dY):
        c = ctx.c
        x, W, Z = ctx.saved_tensors
        need = ctx.needs_input_grad
        dX, dW = (torch.empty_like(t) if need[i] else None for i, t in enumerate((x, W)))
        db = torch.empty((c.d_out,), dtype=torch.float32, device=x.device) if need[2] else None
        if any(need[:3]):
            linear_backward(c, x, W, Z, dY.contiguous().view(c.tokens, c.d_out), dX, dW, db,
                            linear_backward_workspace(c, x.device))
        return (None if dX is None else dX.view(*dY.shape[:-1], c.d_in), dW, None if db is None else db.to(ctx.bias_dtype),
                dY.reshape(ctx.residual_shape) if need[3] else None, None)


class ResidualNormFunction(torch.autograd.Function):
    """The gated residual sum and its norms as a differentiable torch op:
    ``apply(x, h, gate, gamma_h, gamma, beta, scale, shift, norm, branch_norm, eps)`` returns (out, y).

    x, h [groups, rows, d]; gate, scale, shift [groups, d]; gamma_h, gamma, beta [d]; h and every vector may be None.
    With h None, out is None; with norm "none", y is None."""

    @staticmethod
    def forward(ctx, x, h, gate, gamma_h, gamma, beta, scale, shift, norm, branch_norm, eps):
        B, n, d = x.shape
        x, h = x.contiguous(), None if h is None else h.contiguous()
        gamma_h, gamma, beta = (None if t is None else t.contiguous() for t in (gamma_h, gamma, beta))
        gate, scale, shift, apart = _same_stride((gate, scale, shift), d)
        c = make_residual_norm_config(B, n, d, norm, branch_norm, eps, apart, _dtype_of(x, "rola_residual_norm"))
        out = None if h is None else torch.empty_like(x)
        y = None if c.norm == ROLA_NORM_NONE else torch.empty_like(x)
        stats = torch.empty((B, n, 4), dtype=torch.float32, device=x.device)
        residual_norm(c, x, h, out, y, gate=gate, gamma_h=gamma_h, gamma=gamma, beta=beta, scale=scale, shift=shift,
                      stats=stats)
        ctx.c, ctx.shifted = c, None if shift is None else shift.dtype
        ctx.save_for_backward(x, h, gate, gamma_h, gamma, beta, scale, stats)
        ctx.set_materialize_grads(False)
        return out, y

    @staticmethod
    @once_differentiable
    def backward(ctx, dout, dy):
        c = ctx.c
        x, h, gate, gamma_h, gamma, beta, scale, stats = ctx.saved_tensors
        if dout is None and dy is None:
            return (None,) * 11
        if c.norm != ROLA_NORM_NONE and dy is None:          # out alone was used
            dy = torch.zeros_like(x)
        dout, dy = (None if t is None else t.contiguous() for t in (dout, dy))
        dx, dh = torch.empty_like(x), None if h is None else torch.empty_like(h)
        want = ctx.needs_input_grad
        named = dict(dgate=(gate, 2), dgamma_h=(gamma_h, 3), dgamma=(gamma, 4), dbeta=(beta, 5), dscale=(scale, 6))
        grads = {k: torch.empty(t.shape, dtype=torch.float32, device=x.device) if t is not None and want[i] else None
                 for k, (t, i) in named.items()}
        grads["dshift"] = torch.empty((c.groups, c.d), dtype=torch.float32, device=x.device) if want[7] else None
        residual_norm_backward(c, x, h, stats, dout, dy, dx, dh, residual_norm_backward_workspace(c, x.device), gate=gate,
                               gamma_h=gamma_h, gamma=gamma, beta=beta, scale=scale, **grads)
        return (dx, dh, *(None if grads[k] is None else grads[k].to(t.dtype) for k, (t, _) in named.items()),
                None if grads["dshift"] is None else grads["dshift"].to(ctx.shifted), None, None, None)


def _same_stride(vectors, d: int):
    """Vectors of each sample, as they are where they are slices of one modulation (one distance between the samples of
    all), else dense; and that distance."""
    there = [t for t in vectors if t is not None]
    apart = {t.stride(0) if t.shape[0] > 1 else d for t in there}
    if len(apart) == 1 and d <= min(apart) < 2 ** 31 and all(t.stride(1) == 1 for t in there):
        return (*vectors, apart.pop())
    return (*(None if t is None else t.contiguous() for t in vectors), d)
