"""Python binding of the MI355X greedy speculative-verification library.

A thin ctypes layer over the C ABI of ``include/ee.h``: it allocates device
memory with PyTorch (weights, packed-weight arena, KV pool, workspace),
passes raw pointers and the current HIP stream, and converts arguments and
results.  Every step of the verification path runs in the HIP kernels of
``libee.so``; nothing here computes any part of it.  If the library has not
been built, importing this package raises.
"""

from __future__ import annotations

import ctypes
import functools
import os
import struct

import numpy as np
import torch  # loaded first so the HIP runtime it ships is the one libee.so binds to
from torch.autograd import forward_ad as _forward_ad

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libee.so")

EE_OK, EE_EINVAL, EE_ECAPACITY, EE_ESTATE, EE_EHIP = 0, -1, -2, -3, -4
EE_F32, EE_BF16 = 0, 1

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'`")
_lib = ctypes.CDLL(LIB_PATH)

_i32, _vp, _sz = ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t
_pi32 = ctypes.POINTER(ctypes.c_int32)


class EEModelConfig(ctypes.Structure):
    _fields_ = [("n_layers", _i32), ("d_model", _i32), ("n_heads", _i32), ("n_kv_heads", _i32),
                ("head_dim", _i32), ("ffn", _i32), ("vocab", _i32), ("dtype", _i32),
                ("rms_eps", ctypes.c_float), ("rope_theta", ctypes.c_float),
                ("max_ctx", _i32), ("max_seqs", _i32), ("k_max", _i32), ("page_size", _i32)]


class EEWeights(ctypes.Structure):
    _fields_ = [("embed", _vp), ("lm_head", _vp), ("final_gain", _vp),
                ("wq", ctypes.POINTER(_vp)), ("wk", ctypes.POINTER(_vp)), ("wv", ctypes.POINTER(_vp)),
                ("wo", ctypes.POINTER(_vp)), ("w_gate", ctypes.POINTER(_vp)),
                ("w_up", ctypes.POINTER(_vp)), ("w_down", ctypes.POINTER(_vp)),
                ("attn_gain", ctypes.POINTER(_vp)), ("ffn_gain", ctypes.POINTER(_vp))]


class EEMoeConfig(ctypes.Structure):
    _fields_ = [("n_experts", _i32), ("top_k", _i32), ("score", _i32), ("renormalize", _i32), ("n_groups", _i32),
                ("top_groups", _i32), ("group_top", _i32), ("scale", ctypes.c_float)]


class EEMoeWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.POINTER(_vp)) for n in ("router", "router_bias", "w_gate_up", "w_down")]


def _sig(name, res, args):
    f = getattr(_lib, name)
    f.restype, f.argtypes = res, args
    return f


ee_packed_weight_bytes = _sig("ee_packed_weight_bytes", _sz, [ctypes.POINTER(EEModelConfig)])
ee_kv_pool_bytes = _sig("ee_kv_pool_bytes", _sz, [ctypes.POINTER(EEModelConfig)])
ee_workspace_bytes = _sig("ee_workspace_bytes", _sz, [ctypes.POINTER(EEModelConfig)])
ee_create = _sig("ee_create", _i32, [ctypes.POINTER(EEModelConfig), ctypes.POINTER(EEWeights),
                                     _vp, _vp, _vp, _vp, ctypes.POINTER(_vp)])
ee_moe_packed_weight_bytes = _sig("ee_moe_packed_weight_bytes", _sz,
                                  [ctypes.POINTER(EEModelConfig), ctypes.POINTER(EEMoeConfig)])
ee_moe_workspace_bytes = _sig("ee_moe_workspace_bytes", _sz, [ctypes.POINTER(EEModelConfig), ctypes.POINTER(EEMoeConfig)])
ee_moe_create = _sig("ee_moe_create", _i32, [ctypes.POINTER(EEModelConfig), ctypes.POINTER(EEMoeConfig),
                                             ctypes.POINTER(EEWeights), ctypes.POINTER(EEMoeWeights),
                                             _vp, _vp, _vp, _vp, ctypes.POINTER(_vp)])
ee_destroy = _sig("ee_destroy", _i32, [_vp])
ee_prefill = _sig("ee_prefill", _i32, [_vp, _i32, _pi32, _i32, _pi32])
ee_verify = _sig("ee_verify", _i32, [_vp, _i32, _pi32, _i32, _pi32, _pi32, _pi32, _pi32])
ee_verify_noalloc = _sig("ee_verify_noalloc", _i32, [_vp, _i32, _pi32, _i32, _pi32, _pi32, _pi32, _pi32])
ee_verify_batch = _sig("ee_verify_batch", _i32, [_vp, _i32, _pi32, _pi32, _i32, _pi32, _pi32, _pi32, _pi32])
ee_verify_topk = _sig("ee_verify_topk", _i32, [_vp, _i32, _pi32, _pi32, _i32, _i32, _i32, _pi32, _pi32, _pi32])
_pf32 = ctypes.POINTER(ctypes.c_float)
ee_verify_sample = _sig("ee_verify_sample", _i32, [_vp, _i32, _pi32, _i32, _vp, _pf32, _pf32, ctypes.c_float, _i32,
                                                   _pi32, _pi32])
ee_extend = _sig("ee_extend", _i32, [_vp, _i32, _pi32, _i32, _pi32])
ee_kv_rollback = _sig("ee_kv_rollback", _i32, [_vp, _i32, _i32, _i32])
ee_seq_state = _sig("ee_seq_state", _i32, [_vp, _i32, _pi32, _pi32])
ee_match_reuse_c = _sig("ee_match_reuse", _i32, [_pi32, _i32, _pi32, _i32, _i32, _i32, _i32, _pi32, _pi32])
ee_get_logits = _sig("ee_get_logits", _i32, [_vp, ctypes.POINTER(ctypes.c_float), _i32])
ee_read_kv = _sig("ee_read_kv", _i32, [_vp, _i32, _i32, _vp, _vp])
ee_load_kv = _sig("ee_load_kv", _i32, [_vp, _i32, _i32, _i32, _vp, _vp])
ee_capture_bytes = _sig("ee_capture_bytes", _sz, [ctypes.POINTER(EEModelConfig), _i32])
ee_capture = _sig("ee_capture", _i32, [_vp, _vp, _sz])
ee_last_error = _sig("ee_last_error", ctypes.c_char_p, [_vp])
ee_profile = _sig("ee_profile", _i32, [_vp, ctypes.c_uint32])
ee_use_graphs = _sig("ee_use_graphs", _i32, [_vp, _i32])
ee_time_gemm = _sig("ee_time_gemm", _i32, [_vp, ctypes.c_uint32, _i32, _i32, ctypes.POINTER(ctypes.c_double)])
ee_time_stream_read = _sig("ee_time_stream_read", _i32, [_vp, _vp, _sz, _i32, ctypes.POINTER(ctypes.c_double)])
ee_profile_read = _sig("ee_profile_read", _i32, [_vp, ctypes.POINTER(ctypes.c_double),
                                                 ctypes.POINTER(ctypes.c_int64), _i32])

_i64 = ctypes.c_int64


class EELinearArgs(ctypes.Structure):
    _fields_ = [("x", _vp), ("w", _vp), ("bias", _vp), ("residual", _vp), ("y", _vp),
                ("ldx", _i64), ("ldw", _i64), ("ldr", _i64), ("ldy", _i64),
                ("rows", _i32), ("in_", _i32), ("out", _i32), ("dtype", _i32), ("out_dtype", _i32), ("act", _i32)]


class EEMoeRouteArgs(ctypes.Structure):
    _fields_ = [("logits", _vp), ("bias", _vp), ("ids", _vp), ("weights", _vp), ("ld", _i64),
                ("rows", _i32), ("n_experts", _i32), ("top_k", _i32), ("dtype", _i32),
                ("score", _i32), ("renormalize", _i32), ("n_groups", _i32), ("top_groups", _i32), ("group_top", _i32),
                ("scale", ctypes.c_float)]


class EEMoeFfnArgs(ctypes.Structure):
    _fields_ = [("x", _vp), ("w_gate_up", _vp), ("w_down", _vp), ("ids", _vp), ("weights", _vp), ("residual", _vp),
                ("out", _vp), ("workspace", _vp), ("workspace_bytes", _sz), ("ldx", _i64), ("ldr", _i64), ("ldo", _i64),
                ("rows", _i32), ("n_experts", _i32), ("top_k", _i32), ("d_model", _i32), ("ffn", _i32),
                ("dtype", _i32), ("out_dtype", _i32)]


class EEFp8QuantArgs(ctypes.Structure):
    _fields_ = [("x", _vp), ("codes", _vp), ("scales", _vp), ("ldx", _i64), ("ldc", _i64),
                ("rows", _i32), ("in_", _i32), ("block_rows", _i32), ("dtype", _i32)]


class EEFp8LinearArgs(ctypes.Structure):
    _fields_ = [("x", _vp), ("x_scales", _vp), ("w", _vp), ("w_scales", _vp), ("bias", _vp), ("residual", _vp), ("y", _vp),
                ("ldx", _i64), ("ldw", _i64), ("ldr", _i64), ("ldy", _i64),
                ("rows", _i32), ("in_", _i32), ("out", _i32), ("out_dtype", _i32), ("act", _i32)]


# (ee_paged_cache, a member of both: its fields stand in its place)
_CACHE = [("k_cache", _vp), ("v_cache", _vp), ("tables", _vp), ("k_page", _i64), ("k_slot", _i64), ("k_head", _i64),
          ("v_page", _i64), ("v_slot", _i64), ("v_head", _i64), ("ld", _i64),
          ("n_seqs", _i32), ("n_pages", _i32), ("max_pages", _i32), ("page_size", _i32)]


class EEKvAppendArgs(ctypes.Structure):
    _fields_ = [("q", _vp), ("k", _vp), ("v", _vp), ("q_out", _vp), *_CACHE,
                ("seqs", _vp), ("positions", _vp), ("inv_freq", _vp), ("ldq", _i64), ("ldk", _i64), ("ldv", _i64), ("ldqo", _i64),
                ("rows", _i32), ("n_heads", _i32), ("n_kv_heads", _i32), ("head_dim", _i32), ("rot_dim", _i32),
                ("interleaved", _i32), ("dtype", _i32)]


class EEPagedAttentionArgs(ctypes.Structure):
    _fields_ = [("q", _vp), *_CACHE, ("lens", _vp), ("out", _vp), ("lse", _vp), ("workspace", _vp), ("workspace_bytes", _sz),
                ("ldq", _i64), ("ldo", _i64), ("rows", _i32), ("n_heads", _i32), ("n_kv_heads", _i32), ("head_dim", _i32),
                ("window", _i32), ("dtype", _i32), ("out_dtype", _i32), ("scale", ctypes.c_float)]


ee_linear = _sig("ee_linear", _i32, [ctypes.POINTER(EELinearArgs), _vp])
ee_moe_route = _sig("ee_moe_route", _i32, [ctypes.POINTER(EEMoeRouteArgs), _vp])
ee_moe_ffn = _sig("ee_moe_ffn", _i32, [ctypes.POINTER(EEMoeFfnArgs), _vp])
ee_fp8_quant = _sig("ee_fp8_quant", _i32, [ctypes.POINTER(EEFp8QuantArgs), _vp])
ee_fp8_linear = _sig("ee_fp8_linear", _i32, [ctypes.POINTER(EEFp8LinearArgs), _vp])
ee_kv_append = _sig("ee_kv_append", _i32, [ctypes.POINTER(EEKvAppendArgs), _vp])
ee_paged_attention = _sig("ee_paged_attention", _i32, [ctypes.POINTER(EEPagedAttentionArgs), _vp])


def _packed(name: str, args):
    """An operator's C call for arguments packed into bytes: (packer, call).  A third of
    a microsecond less than filling ``args``, a twentieth of a small call."""
    layout = "@" + "".join(t._type_ for _, t in args._fields_) + "0P"   # (padded at its end as in C)
    return struct.Struct(layout).pack, ctypes.CFUNCTYPE(_i32, ctypes.c_char_p, _vp)((name, _lib))


_OP_LINEAR = _packed("ee_linear", EELinearArgs)
_OP_ROUTE = _packed("ee_moe_route", EEMoeRouteArgs)
_OP_FFN = _packed("ee_moe_ffn", EEMoeFfnArgs)
_OP_FP8_QUANT = _packed("ee_fp8_quant", EEFp8QuantArgs)
_OP_FP8_LINEAR = _packed("ee_fp8_linear", EEFp8LinearArgs)
_OP_KV_APPEND = _packed("ee_kv_append", EEKvAppendArgs)
_OP_PAGED_ATTENTION = _packed("ee_paged_attention", EEPagedAttentionArgs)
ee_paged_attention_workspace_bytes = _sig("ee_paged_attention_workspace_bytes", _sz, [_i32] * 8)
ee_moe_ffn_workspace_bytes = _sig("ee_moe_ffn_workspace_bytes", _sz, [_i32] * 6)

ACTIVATIONS = ("none", "silu", "gelu", "gelu_tanh", "relu")
SCORES = ("softmax", "sigmoid")

PROF_CLASSES = ("norm", "qkv", "attn", "combine", "oproj", "gateup", "down", "lmhead", "argmax",
                "accept", "compact", "finish")


EE_PHASE_REUSE, EE_PHASE_GENERATE = 0, 1


class EEEditParams(ctypes.Structure):
    _fields_ = [("k_reuse", _i32), ("gamma", _i32), ("top_k", _i32), ("dynamic", _i32),
                ("min_match", _i32), ("max_match", _i32)]


class EEEditState(ctypes.Structure):
    _fields_ = [("phase", _i32), ("cursor", _i32), ("last_phase", _i32), ("last_accept", _i32),
                ("steps", ctypes.c_int64 * 2), ("emitted", ctypes.c_int64 * 2),
                ("draft_tokens", ctypes.c_int64), ("draft_forwards", ctypes.c_int64)]


ee_edit_begin = _sig("ee_edit_begin", _i32, [_vp, _i32, _vp, _i32, ctypes.POINTER(EEEditState)])
ee_edit_step = _sig("ee_edit_step", _i32, [_vp, _i32, _vp, _i32, _pi32, _i32, ctypes.POINTER(EEEditParams),
                                           ctypes.POINTER(EEEditState), _pi32, _i32, _i32, _pi32])


class EEError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"ee error {code}: {msg}")
        self.code = code


def _check(rc: int, ctx=None):
    if rc != EE_OK:
        raise EEError(rc, ee_last_error(ctx).decode())


def _i32arr(x):
    a = np.ascontiguousarray(np.asarray(x, dtype=np.int32))
    return a, a.ctypes.data_as(_pi32)


def make_config(shape, max_ctx: int, max_seqs: int = 1, k_max: int = 64) -> EEModelConfig:
    return EEModelConfig(shape.n_layers, shape.d_model, shape.n_heads, shape.n_kv_heads,
                         shape.head_dim, shape.ffn, shape.vocab,
                         EE_BF16 if shape.dtype == "bf16" else EE_F32,
                         shape.rms_eps, shape.rope_theta, max_ctx, max_seqs, k_max, 64)


def make_moe_config(shape) -> EEMoeConfig:
    """The routing of a shape with sparse layers."""
    return EEMoeConfig(shape.n_experts, shape.top_k, SCORES.index(shape.score), int(shape.renormalize),
                       shape.n_groups, shape.top_groups, shape.group_top, shape.route_scale)


# -- stand-alone operators ---------------------------------------------------
#
# Device tensors in, device tensors out, on the tensors' device and its current
# stream; nothing synchronizes.  Outputs are allocated with PyTorch unless given; one
# that is given counts as written in place (its version grows).
# They have no backward pass and no forward-mode derivative: operands that require a
# gradient are refused while gradients are recorded, and operands that carry a tangent.

_TYPES = {torch.float32: EE_F32, torch.bfloat16: EE_BF16}
_ACT_OF = {a: i for i, a in enumerate(ACTIVATIONS)}
_SCORE_OF = {a: i for i, a in enumerate(SCORES)}
# (the plain call where the raw one is missing: it is 1.8 us slower, a seventh of a small call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _refuse(what: str, shape, dtype, dev, t):
    if isinstance(t, torch.Tensor) and t.requires_grad and torch.is_grad_enabled():
        raise EEError(EE_EINVAL, f"{what} requires a gradient, which these operators do not have (use torch.no_grad)")
    got = f"{list(t.shape)} {t.dtype} on {t.device}" if isinstance(t, torch.Tensor) else type(t).__name__
    raise EEError(EE_EINVAL, f"{what} must be {list(shape)} {dtype} on cuda:{dev} (rows of unit column stride), not {got}")


def _refuse_tangents(**operands):
    for what, t in operands.items():
        if isinstance(t, torch.Tensor) and _forward_ad.unpack_dual(t).tangent is not None:
            raise EEError(EE_EINVAL, f"{what} carries a tangent (forward_ad), which these operators do not propagate")


def _tangents() -> bool:
    """Whether operands may carry tangents (inside forward_ad.dual_level)."""
    return getattr(_forward_ad, "_current_level", 0) >= 0


def _rows_of(t, what: str, shape, dtype, dev) -> int:
    """Checks a [rows, cols] operand of unit column stride; returns its row stride."""
    if (isinstance(t, torch.Tensor) and t.shape == shape and t.dtype is dtype and t.get_device() == dev
            and not (t.requires_grad and torch.is_grad_enabled())):
        rs, cs = t.stride()
        if cs == 1 or shape[1] <= 1:
            # (a single row may carry any stride: the last position of a batch of one, a view
            # whose stride the library might refuse)
            return rs if shape[0] > 1 else shape[1]
    _refuse(what, shape, dtype, dev, t)


def _whole(t, what: str, shape, dtype, dev) -> int:
    """Checks a contiguous operand; returns its address."""
    if (isinstance(t, torch.Tensor) and t.shape == shape and t.dtype is dtype and t.get_device() == dev
            and t.is_contiguous() and not (t.requires_grad and torch.is_grad_enabled())):
        return t.data_ptr()
    _refuse(what, shape, dtype, dev, t)


def _operand(x, what: str):
    """Checks a call's first operand, [rows, cols] of unit column stride: (device
    index, EE_* type, rows, cols, row stride)."""
    if not isinstance(x, torch.Tensor) or x.dim() != 2 or not x.is_cuda:
        raise EEError(EE_EINVAL, f"{what} must be a two-dimensional tensor on a GPU")
    dt = _TYPES.get(x.dtype)
    if dt is None:
        raise EEError(EE_EINVAL, f"{what} must be float32 or bfloat16")
    dev = x.get_device()
    rows, cols = x.shape
    ld, cs = x.stride()
    if (cs != 1 and cols > 1) or (x.requires_grad and torch.is_grad_enabled()):
        _refuse(what, (rows, cols), x.dtype, dev, x)
    return dev, dt, rows, cols, ld if rows > 1 else cols


def _out_type(out_dtype, out, x):
    if out_dtype is None:
        out_dtype = x.dtype if out is None else getattr(out, "dtype", None)
    if out_dtype not in _TYPES:
        raise EEError(EE_EINVAL, "out_dtype must be float32 or bfloat16")
    return out_dtype


_current_device = torch.cuda.current_device
_written = torch.autograd.graph.increment_version


def _operator(op, dev: int, *args):
    """Calls an operator on GPU ``dev`` and its current stream."""
    pack, fn = op
    try:
        packed = pack(*args)
    except (struct.error, OverflowError) as e:
        raise EEError(EE_EINVAL, f"an argument does not fit its type: {e}") from None
    if dev == _current_device():
        rc = fn(packed, _raw_stream(dev))
    else:
        with torch.cuda.device(dev):
            rc = fn(packed, _raw_stream(dev))
    if rc != EE_OK:
        _check(rc)


def linear(x, w, bias=None, act: str = "none", residual=None, out=None, out_dtype=None):
    """act(x w^T + bias) + residual (ee_linear).  x [rows, in] and w [out, in]
    in float32 or bfloat16, bias [out] float32, residual [rows, out] in the
    output's dtype (``out_dtype``: x's, or float32).  ``out`` may be the residual."""
    dev, dt, rows, cols, ldx = _operand(x, "x")
    if _tangents():
        _refuse_tangents(x=x, w=w, bias=bias, residual=residual, out=out)
    code = _ACT_OF.get(act)
    if code is None:
        raise EEError(EE_EINVAL, f"act must be one of {ACTIVATIONS}")
    if not isinstance(w, torch.Tensor) or w.dim() != 2:
        raise EEError(EE_EINVAL, "w must be [out, in]")
    n = w.shape[0]
    ldw = _rows_of(w, "w", (n, cols), x.dtype, dev)
    odt = _out_type(out_dtype, out, x)
    shape = (rows, n)
    given = out is not None
    if given:
        ldy = _rows_of(out, "out", shape, odt, dev)
    else:
        out, ldy = x.new_empty(shape, dtype=odt), n
    ldr = 0 if residual is None else _rows_of(residual, "residual", shape, odt, dev)
    _operator(_OP_LINEAR, dev, x.data_ptr(), w.data_ptr(), 0 if bias is None else _whole(bias, "bias", (n,), torch.float32, dev),
              0 if residual is None else residual.data_ptr(), out.data_ptr(), ldx, ldw, ldr, ldy, rows, cols, n, dt,
              _TYPES[odt], code)
    if given:
        _written(out)
    return out


def moe_route(logits, top_k: int, score: str = "softmax", bias=None, renormalize: bool = True, scale: float = 1.0,
              n_groups: int = 1, top_groups: int = 1, group_top: int = 1):
    """Experts and weights of every row of the router's logits [rows, experts]
    (ee_moe_route): (ids int32, weights float32), both [rows, top_k]."""
    dev, dt, rows, n, ld = _operand(logits, "logits")
    if _tangents():
        _refuse_tangents(logits=logits, bias=bias)
    code = _SCORE_OF.get(score)
    if code is None:
        raise EEError(EE_EINVAL, f"score must be one of {SCORES}")
    k = int(top_k)
    shape = (rows, k if 0 < k <= n else 0)   # (refused below)
    ids = logits.new_empty(shape, dtype=torch.int32)
    weights = logits.new_empty(shape, dtype=torch.float32)
    _operator(_OP_ROUTE, dev, logits.data_ptr(), 0 if bias is None else _whole(bias, "bias", (n,), torch.float32, dev),
              ids.data_ptr(), weights.data_ptr(), ld, rows, n, k, dt, code, 1 if renormalize else 0, int(n_groups),
              int(top_groups), int(group_top), scale)
    return ids, weights


_ffn_workspace = functools.lru_cache(maxsize=1024)(ee_moe_ffn_workspace_bytes)   # (a function of its arguments)


def moe_ffn(x, w_gate_up, w_down, ids, weights, residual=None, out=None, out_dtype=None, workspace=None):
    """residual + the weighted sum of the experts' SwiGLU products of every row
    (ee_moe_ffn).  x [rows, d], w_gate_up [experts, 2 ffn, d] (gate rows, then
    up rows) and w_down [experts, d, ffn] in float32 or bfloat16; ids int32 and
    weights float32 [rows, top_k] as from ``moe_route``; residual and out
    [rows, d] in ``out_dtype`` (x's, or float32).  ``workspace``: a uint8 tensor
    of at least ee_moe_ffn_workspace_bytes, else one is allocated."""
    dev, dt, rows, d, ldx = _operand(x, "x")
    if _tangents():
        _refuse_tangents(x=x, w_gate_up=w_gate_up, w_down=w_down, weights=weights, residual=residual, out=out)
    if not (isinstance(w_down, torch.Tensor) and w_down.dim() == 3 and isinstance(ids, torch.Tensor) and ids.dim() == 2):
        raise EEError(EE_EINVAL, "w_down must be [experts, d, ffn], ids [rows, top_k]")
    E, _, f = w_down.shape
    k = ids.shape[1]
    pointers = (x.data_ptr(), _whole(w_gate_up, "w_gate_up", (E, 2 * f, d), x.dtype, dev),
                _whole(w_down, "w_down", (E, d, f), x.dtype, dev), _whole(ids, "ids", (rows, k), torch.int32, dev),
                _whole(weights, "weights", (rows, k), torch.float32, dev))
    odt = _out_type(out_dtype, out, x)
    shape = (rows, d)
    given = out is not None
    if given:
        ldo = _rows_of(out, "out", shape, odt, dev)
    else:
        out, ldo = x.new_empty(shape, dtype=odt), d
    ldr = 0 if residual is None else _rows_of(residual, "residual", shape, odt, dev)
    if workspace is None:
        workspace = x.new_empty(_ffn_workspace(rows, E, k, d, f, dt), dtype=torch.uint8)
    elif (not isinstance(workspace, torch.Tensor) or workspace.dtype != torch.uint8 or workspace.get_device() != dev
          or not workspace.is_contiguous()):
        raise EEError(EE_EINVAL, f"workspace must be contiguous uint8 on cuda:{dev}")
    _operator(_OP_FFN, dev, *pointers, 0 if residual is None else residual.data_ptr(), out.data_ptr(), workspace.data_ptr(),
              workspace.numel(), ldx, ldr, ldo, rows, E, k, d, f, dt, _TYPES[odt])
    if given:
        _written(out)
    return out


def _codes(t, what: str):
    """Checks e4m3 codes [rows, cols] of unit column stride: (device index, rows, cols, row stride)."""
    if not isinstance(t, torch.Tensor) or t.dim() != 2 or not t.is_cuda or t.dtype is not torch.float8_e4m3fn:
        raise EEError(EE_EINVAL, f"{what} must be a two-dimensional float8_e4m3fn tensor on a GPU")
    rows, cols = t.shape
    dev = t.get_device()
    return dev, rows, cols, _rows_of(t, what, t.shape, t.dtype, dev)


def fp8_quant(x, block_rows: int = 1, codes=None, scales=None):
    """e4m3 codes of x [rows, in] (float32 or bfloat16) and their scales, one per
    block of ``block_rows`` (1, or 128 for weights) rows and 128 columns
    (ee_fp8_quant): (float8_e4m3fn [rows, in], float32 [ceil(rows / block_rows), ceil(in / 128)])."""
    dev, dt, rows, cols, ldx = _operand(x, "x")
    if _tangents():
        _refuse_tangents(x=x)
    if block_rows not in (1, 128):
        raise EEError(EE_EINVAL, "block_rows must be 1 or 128")
    shape = (-(-rows // block_rows), -(-cols // 128))
    given = codes, scales
    if codes is None:
        codes, ldc = x.new_empty((rows, cols), dtype=torch.float8_e4m3fn), cols
    else:
        ldc = _rows_of(codes, "codes", (rows, cols), torch.float8_e4m3fn, dev)
    if scales is None:
        scales = x.new_empty(shape, dtype=torch.float32)
    _operator(_OP_FP8_QUANT, dev, x.data_ptr(), codes.data_ptr(), _whole(scales, "scales", shape, torch.float32, dev), ldx, ldc,
              rows, cols, block_rows, dt)
    for t in given:
        if t is not None:
            _written(t)
    return codes, scales


def fp8_linear(x, x_scales, w, w_scales, bias=None, act: str = "none", residual=None, out=None, out_dtype=None):
    """act(x w^T + bias) + residual of e4m3 codes and their scales (ee_fp8_linear): x
    [rows, in] with a scale per row and 128 columns, w [out, in] with one per 128
    rows and 128 columns, as ``fp8_quant`` makes them with ``block_rows`` 1 and 128.  ``out_dtype``:
    bfloat16 (the default), or float32, whose products are summed in float32
    throughout.  ``out`` may be the residual."""
    dev, rows, cols, ldx = _codes(x, "x")
    if _tangents():
        _refuse_tangents(x_scales=x_scales, w_scales=w_scales, bias=bias, residual=residual, out=out)
    code = _ACT_OF.get(act)
    if code is None:
        raise EEError(EE_EINVAL, f"act must be one of {ACTIVATIONS}")
    if not isinstance(w, torch.Tensor) or w.dim() != 2:
        raise EEError(EE_EINVAL, "w must be [out, in]")
    n, blocks = w.shape[0], -(-cols // 128)
    ldw = _rows_of(w, "w", (n, cols), x.dtype, dev)
    if out_dtype is None and out is None:
        odt = torch.bfloat16
    else:
        odt = _out_type(out_dtype, out, x)
    shape = (rows, n)
    given = out is not None
    if given:
        ldy = _rows_of(out, "out", shape, odt, dev)
    else:
        out, ldy = x.new_empty(shape, dtype=odt), n
    ldr = 0 if residual is None else _rows_of(residual, "residual", shape, odt, dev)
    _operator(_OP_FP8_LINEAR, dev, x.data_ptr(), _whole(x_scales, "x_scales", (rows, blocks), torch.float32, dev), w.data_ptr(),
              _whole(w_scales, "w_scales", (-(-n // 128), blocks), torch.float32, dev),
              0 if bias is None else _whole(bias, "bias", (n,), torch.float32, dev),
              0 if residual is None else residual.data_ptr(), out.data_ptr(), ldx, ldw, ldr, ldy, rows, cols, n, _TYPES[odt], code)
    if given:
        _written(out)
    return out


def _cache(k_cache, v_cache, tables, dtype, dev: int):
    """Checks a paged cache: (its arguments, page size, KV heads, head_dim, max_pages, sequences)."""
    if not (isinstance(k_cache, torch.Tensor) and isinstance(v_cache, torch.Tensor) and k_cache.dim() == 4
            and k_cache.shape == v_cache.shape and k_cache.dtype is dtype and v_cache.dtype is dtype
            and k_cache.get_device() == dev and v_cache.get_device() == dev):
        raise EEError(EE_EINVAL, f"k_cache and v_cache must be [pages, page size, KV heads, head_dim] {dtype} on cuda:{dev}")
    if (k_cache.requires_grad or v_cache.requires_grad) and torch.is_grad_enabled():
        raise EEError(EE_EINVAL, "the cache requires a gradient, which these operators do not have (use torch.no_grad)")
    pages, page, heads, hd = k_cache.shape
    kp, ks, kh, kd = k_cache.stride()
    vp, vs, vh, vd = v_cache.stride()
    if kd != 1 or vd != 1:
        raise EEError(EE_EINVAL, "k_cache and v_cache must have unit stride within a vector")
    if not isinstance(tables, torch.Tensor) or tables.dim() != 2:
        raise EEError(EE_EINVAL, "tables must be [sequences, pages of one]")
    n, most = tables.shape
    ld = _rows_of(tables, "tables", (n, most), torch.int32, dev)
    # (a dimension of one element may carry any stride)
    if pages <= 1:
        kp = vp = 0
    if heads <= 1:
        kh = vh = 0
    return (k_cache.data_ptr(), v_cache.data_ptr(), tables.data_ptr(), kp, ks, kh, vp, vs, vh, ld, n, pages, most, page), page, heads, hd, most, n


def kv_append(k, v, k_cache, v_cache, tables, positions, seqs=None, q=None, inv_freq=None, interleaved: bool = False, q_out=None):
    """Writes the rows of k and v [rows, KV heads * head_dim] to their sequences'
    pages, k rotated by its row's position; q [rows, heads * head_dim], if given, is rotated
    too and returned (``q_out``, which may be q; else None) (ee_kv_append).  k_cache and
    v_cache [pages, page size, KV heads, head_dim] of any strides, tables int32 [sequences,
    pages of one], positions int32 [rows], seqs int32 [rows] (the default: equally many
    consecutive rows of every sequence), inv_freq float64 [rotated dimensions / 2] (None: no
    rotation).  Operands are float32 or bfloat16, all of one type."""
    dev, dt, rows, kd, ldk = _operand(k, "k")
    if _tangents():
        _refuse_tangents(q=q, k=k, v=v, k_cache=k_cache, v_cache=v_cache, inv_freq=inv_freq, q_out=q_out)
    cache, _, heads, hd, _, _ = _cache(k_cache, v_cache, tables, k.dtype, dev)
    if kd != heads * hd:
        raise EEError(EE_EINVAL, f"k must be [rows, {heads} * {hd}]")
    ldv = _rows_of(v, "v", (rows, kd), k.dtype, dev)
    n_heads, ldq, ldqo, given = heads, 0, 0, q_out is not None
    if q is None:
        if given:
            raise EEError(EE_EINVAL, "q_out needs q")
    else:
        if not isinstance(q, torch.Tensor) or q.dim() != 2 or hd < 1 or q.shape[1] % hd:
            raise EEError(EE_EINVAL, f"q must be [rows, heads * {hd}]")
        qd = q.shape[1]
        n_heads = qd // hd
        ldq = _rows_of(q, "q", (rows, qd), k.dtype, dev)
        if given:
            ldqo = _rows_of(q_out, "q_out", (rows, qd), k.dtype, dev)
        else:
            q_out, ldqo = q.new_empty((rows, qd)), qd
    rot, freq = 0, 0
    if inv_freq is not None:
        if not isinstance(inv_freq, torch.Tensor) or inv_freq.dim() != 1:
            raise EEError(EE_EINVAL, "inv_freq must be [rotated dimensions / 2]")
        rot = 2 * inv_freq.shape[0]
        freq = _whole(inv_freq, "inv_freq", inv_freq.shape, torch.float64, dev)
    _operator(_OP_KV_APPEND, dev, 0 if q is None else q.data_ptr(), k.data_ptr(), v.data_ptr(), 0 if q is None else q_out.data_ptr(),
              *cache, 0 if seqs is None else _whole(seqs, "seqs", (rows,), torch.int32, dev),
              _whole(positions, "positions", (rows,), torch.int32, dev), freq, ldq, ldk, ldv, ldqo,
              rows, n_heads, heads, hd, rot, 1 if interleaved else 0, dt)
    _written((k_cache, v_cache))
    if given:
        _written(q_out)
    return q_out


_attention_workspace = functools.lru_cache(maxsize=1024)(ee_paged_attention_workspace_bytes)   # (a function of its arguments)


def paged_attention(q, k_cache, v_cache, tables, lens, window: int = 0, scale=None, out=None, out_dtype=None, lse=None, workspace=None):
    """Attention of the newest rows of every sequence over its pages (ee_paged_attention):
    q [sequences * rows, heads * head_dim], a sequence's rows one after another, the
    cache and tables as ``kv_append`` writes them, lens int32 [sequences] (positions
    held, these rows' among them).  ``window``: positions a row sees, its own last (0:
    all).  ``scale``: of the scores, 1 / sqrt(head_dim) unless given.  ``lse``: a float32
    tensor [sequences * rows, heads] for the logarithms of the softmax's sums.
    ``workspace``: a uint8 tensor of at least ee_paged_attention_workspace_bytes, else one is allocated."""
    dev, dt, total, qd, ldq = _operand(q, "q")
    if _tangents():
        _refuse_tangents(q=q, k_cache=k_cache, v_cache=v_cache, out=out, lse=lse)
    cache, page, heads, hd, most, n = _cache(k_cache, v_cache, tables, q.dtype, dev)
    if hd < 1 or qd % hd or (total % n if n else total):
        raise EEError(EE_EINVAL, f"q must be [{n} * rows, heads * {hd}]")
    if total:
        seqs, rows = n, total // n
    else:   # no rows of however many sequences: the same checks, and no work
        seqs, rows, cache = 0, 1, (*cache[:10], 0, *cache[11:])
    odt = _out_type(out_dtype, out, q)
    shape = (total, qd)
    given = out is not None
    if given:
        ldo = _rows_of(out, "out", shape, odt, dev)
    else:
        out, ldo = q.new_empty(shape, dtype=odt), qd
    window, n_heads = int(window), qd // hd
    if workspace is None:
        workspace = q.new_empty(_attention_workspace(seqs, rows, n_heads, heads, hd, page, most, window), dtype=torch.uint8)
    elif (not isinstance(workspace, torch.Tensor) or workspace.dtype != torch.uint8 or workspace.get_device() != dev
          or not workspace.is_contiguous()):
        raise EEError(EE_EINVAL, f"workspace must be contiguous uint8 on cuda:{dev}")
    _operator(_OP_PAGED_ATTENTION, dev, q.data_ptr(), *cache, _whole(lens, "lens", (n,), torch.int32, dev), out.data_ptr(),
              0 if lse is None else _whole(lse, "lse", (total, n_heads), torch.float32, dev), workspace.data_ptr(), workspace.numel(),
              ldq, ldo, rows, n_heads, heads, hd, window, dt, _TYPES[odt], hd ** -0.5 if scale is None else scale)
    if given:
        _written(out)
    if lse is not None:
        _written(lse)
    return out


def match_reuse(generated, original, cursor: int, min_ngram: int = 1, max_ngram: int = 8):
    """Reuse-phase matcher: (draft_start, match_len), (-1, 0) if nothing matches."""
    g, gp = _i32arr(generated)
    o, op = _i32arr(original)
    ds, ml = ctypes.c_int32(), ctypes.c_int32()
    _check(ee_match_reuse_c(gp, len(g), op, len(o), cursor, min_ngram, max_ngram,
                            ctypes.byref(ds), ctypes.byref(ml)))
    return ds.value, ml.value


def _to_device(a: np.ndarray, device) -> torch.Tensor:
    if a.dtype == np.uint16:
        t = torch.from_numpy(np.ascontiguousarray(a).view(np.int16))
    else:
        t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32))
    return t.to(device, non_blocking=False)


class Engine:
    """One library context: packed weights, a paged KV pool, one workspace.

    ``weights`` provides numpy arrays in the model dtype (``embed``,
    ``lm_head``, ``final_gain``, ``layer(l)`` mapping), as drawn by
    ``workloads.gen_weights``.  A shape with ``n_experts`` has sparse layers
    (ee_moe_create): its layers map router, w_gate_up, w_down and, optionally,
    router_bias.
    """

    def __init__(self, shape, weights, max_ctx: int, max_seqs: int = 1, k_max: int = 64,
                 device: str = "cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("the verification library needs a ROCm GPU")
        self.shape, self.device = shape, torch.device(device)
        self.cfg = make_config(shape, max_ctx, max_seqs, k_max)
        cfgp = ctypes.byref(self.cfg)
        moe = make_moe_config(shape) if getattr(shape, "n_experts", 0) else None
        nb_packed, nb_kv, nb_ws = ee_packed_weight_bytes(cfgp), ee_kv_pool_bytes(cfgp), ee_workspace_bytes(cfgp)
        if moe is not None:
            nb_packed, nb_ws = (f(cfgp, ctypes.byref(moe)) for f in (ee_moe_packed_weight_bytes, ee_moe_workspace_bytes))
        if not (nb_packed and nb_kv and nb_ws):
            raise EEError(EE_EINVAL, "invalid model config for the library")
        with torch.cuda.device(self.device):
            self.packed = torch.empty(nb_packed, dtype=torch.uint8, device=self.device)
            self.kv_pool = torch.empty(nb_kv, dtype=torch.uint8, device=self.device)
            self.workspace = torch.empty(nb_ws, dtype=torch.uint8, device=self.device)
            self.stream = torch.cuda.current_stream(self.device)
            keep = []

            def dev(a):
                t = _to_device(a, self.device)
                keep.append(t)
                return t.data_ptr()

            L = shape.n_layers
            arr = lambda: (_vp * L)()
            names = ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down", "attn_gain", "ffn_gain")
            sparse = ("router", "router_bias", "w_gate_up", "w_down") if moe is not None else ()
            own = [k for k in names if not sparse or not k.startswith("w_")]   # (sparse layers: no dense FFN)
            ptrs = {k: arr() for k in (*own, *sparse)}
            for l in range(L):
                lw = weights.layer(l)
                for k in ptrs:
                    ptrs[k][l] = dev(lw[k]) if k != "router_bias" or k in lw else None
            cast = lambda k: ctypes.cast(ptrs[k], ctypes.POINTER(_vp)) if k in ptrs else None
            w = EEWeights(dev(weights.embed), dev(weights.lm_head), dev(weights.final_gain),
                          *[cast(k) if k in own else None for k in names])
            torch.cuda.synchronize(self.device)
            ctx = _vp()
            buffers = (self.packed.data_ptr(), self.kv_pool.data_ptr(), self.workspace.data_ptr(),
                       self.stream.cuda_stream, ctypes.byref(ctx))
            if moe is None:
                _check(ee_create(cfgp, ctypes.byref(w), *buffers))
            else:
                mw = EEMoeWeights(*[cast(k) for k in sparse])
                _check(ee_moe_create(cfgp, ctypes.byref(moe), ctypes.byref(w), ctypes.byref(mw), *buffers))
            self.ctx = ctx
            del keep
        self._last_rows = 0

    # -- calls ---------------------------------------------------------------
    def prefill(self, seq: int, tokens) -> int:
        t, tp = _i32arr(tokens)
        nxt = ctypes.c_int32()
        _check(ee_prefill(self.ctx, seq, tp, len(t), ctypes.byref(nxt)), self.ctx)
        self._last_rows = min(len(t) - (len(t) - 1) // (self.cfg.k_max + 1) * (self.cfg.k_max + 1),
                              self.cfg.k_max + 1)
        return nxt.value

    def extend(self, seq: int, tokens) -> int:
        """Commit [pending, tokens...] without verification; returns the new
        pending token (the greedy token after the last one)."""
        t, tp = _i32arr(tokens)
        nxt = ctypes.c_int32()
        _check(ee_extend(self.ctx, seq, tp if len(t) else None, len(t), ctypes.byref(nxt)), self.ctx)
        self._last_rows = (len(t) + 1) - len(t) // (self.cfg.k_max + 1) * (self.cfg.k_max + 1)
        return nxt.value

    def verify(self, seq: int, draft, parent=None):
        """Returns (accept_len, next_token, accepted_nodes or None)."""
        d, dp = _i32arr(draft)
        k = len(d)
        a, nxt = ctypes.c_int32(), ctypes.c_int32()
        if parent is not None:
            p, pp = _i32arr(parent)
            if len(p) != k:
                raise EEError(EE_EINVAL, "parent must have one entry per draft node")
            nodes = np.zeros(max(k, 1), dtype=np.int32)
            _check(ee_verify(self.ctx, seq, dp, k, pp, ctypes.byref(a), ctypes.byref(nxt),
                             nodes.ctypes.data_as(_pi32)), self.ctx)
            self._last_rows = k + 1
            return a.value, nxt.value, nodes[:a.value].copy()
        _check(ee_verify(self.ctx, seq, dp, k, None, ctypes.byref(a), ctypes.byref(nxt), None), self.ctx)
        self._last_rows = k + 1
        return a.value, nxt.value, None

    def verify_noalloc(self, seq: int, draft, parent=None):
        """ee_verify_noalloc: ee_verify with the step's scratch in the
        library's static device array (no allocation, no graph).  Returns
        (accept_len, next_token, accepted_nodes or None)."""
        d, dp = _i32arr(draft)
        k = len(d)
        a, nxt = ctypes.c_int32(), ctypes.c_int32()
        pp, nodes = None, None
        if parent is not None:
            p, pp = _i32arr(parent)
            if len(p) != k:
                raise EEError(EE_EINVAL, "parent must have one entry per draft node")
            nodes = np.zeros(max(k, 1), dtype=np.int32)
        _check(ee_verify_noalloc(self.ctx, seq, dp, k, pp, ctypes.byref(a), ctypes.byref(nxt),
                                 nodes.ctypes.data_as(_pi32) if nodes is not None else None), self.ctx)
        self._last_rows = k + 1
        return a.value, nxt.value, (nodes[:a.value].copy() if nodes is not None else None)

    def verify_batch(self, seqs, drafts, parents=None):
        """One block for several sequences; drafts (and parents) are equal-length
        lists, one per sequence.  Returns [(accept_len, next_token,
        accepted_nodes or None)] in the order of ``seqs``."""
        n = len(seqs)
        k = len(drafts[0]) if n else 0
        if len(drafts) != n or any(len(d) != k for d in drafts):
            raise EEError(EE_EINVAL, "one draft per sequence, all of the same length")
        sq, sp = _i32arr(seqs)
        d, dp = _i32arr(np.concatenate([np.asarray(x, dtype=np.int32).reshape(-1) for x in drafts])
                        if n else np.zeros(0, np.int32))
        acc = np.zeros(max(n, 1), dtype=np.int32)
        nxt = np.zeros(max(n, 1), dtype=np.int32)
        nodes = np.zeros(max(n * k, 1), dtype=np.int32)
        pp = None
        if parents is not None:
            if len(parents) != n or any(len(p) != k for p in parents):
                raise EEError(EE_EINVAL, "parents must match the drafts")
            p, pp = _i32arr(np.concatenate([np.asarray(x, dtype=np.int32).reshape(-1) for x in parents]))
        _check(ee_verify_batch(self.ctx, n, sp, dp, k, pp, acc.ctypes.data_as(_pi32), nxt.ctypes.data_as(_pi32),
                               nodes.ctypes.data_as(_pi32) if parents is not None else None), self.ctx)
        self._last_rows = n * (k + 1)
        out = []
        for b in range(n):
            a = int(acc[b])
            out.append((a, int(nxt[b]), nodes[b * k:b * k + a].copy() if parents is not None else None))
        return out

    def verify_sample(self, seq: int, draft, eps, u, q=None, temperature: float = 1.0, residual: bool = True):
        """Stochastic verification (Eq. 4).  ``q``: None (greedy draft) or a
        [K, vocab] float32 array of draft distributions (uploaded to the
        device here); ``eps`` (K) and ``u`` (K + 1) are uniform draws.
        Returns (accept_len, next_token)."""
        d, dp = _i32arr(draft)
        k = len(d)
        e = np.ascontiguousarray(np.asarray(eps, dtype=np.float32).reshape(-1))
        uu = np.ascontiguousarray(np.asarray(u, dtype=np.float32).reshape(-1))
        if len(e) != k or len(uu) != k + 1:
            raise EEError(EE_EINVAL, "eps needs K values and u K + 1")
        qdev = None
        if q is not None:
            qa = np.ascontiguousarray(np.asarray(q, dtype=np.float32))
            if qa.shape != (k, self.shape.vocab):
                raise EEError(EE_EINVAL, "q must be [K, vocab]")
            qdev = torch.from_numpy(qa).to(self.device)
            torch.cuda.synchronize(self.device)
        a, nxt = ctypes.c_int32(), ctypes.c_int32()
        _check(ee_verify_sample(self.ctx, seq, dp if k else None, k, qdev.data_ptr() if qdev is not None else None,
                                e.ctypes.data_as(_pf32), uu.ctypes.data_as(_pf32), float(temperature),
                                int(bool(residual)), ctypes.byref(a), ctypes.byref(nxt)), self.ctx)
        self._last_rows = k + 1
        return a.value, nxt.value

    def verify_topk(self, seqs, drafts, top_k: int, dynamic: bool = True):
        """Entropy-aware (``dynamic``) or fixed top-k verification of linear
        drafts, one per sequence, all of the same length.  Returns
        [(accept_len, next_token, thresholds)] in the order of ``seqs``, where
        thresholds[i] is the tau applied to draft token i."""
        n = len(seqs)
        k = len(drafts[0]) if n else 0
        if len(drafts) != n or any(len(d) != k for d in drafts):
            raise EEError(EE_EINVAL, "one draft per sequence, all of the same length")
        sq, sp = _i32arr(seqs)
        d, dp = _i32arr(np.concatenate([np.asarray(x, dtype=np.int32).reshape(-1) for x in drafts])
                        if n else np.zeros(0, np.int32))
        acc = np.zeros(max(n, 1), dtype=np.int32)
        nxt = np.zeros(max(n, 1), dtype=np.int32)
        thr = np.zeros(max(n * k, 1), dtype=np.int32)
        _check(ee_verify_topk(self.ctx, n, sp, dp, k, int(top_k), int(bool(dynamic)), acc.ctypes.data_as(_pi32),
                              nxt.ctypes.data_as(_pi32), thr.ctypes.data_as(_pi32)), self.ctx)
        self._last_rows = n * (k + 1)
        return [(int(acc[b]), int(nxt[b]), thr[b * k:(b + 1) * k].copy()) for b in range(n)]

    def rollback(self, seq: int, new_len: int, pending: int):
        _check(ee_kv_rollback(self.ctx, seq, new_len, pending), self.ctx)

    def seq_state(self, seq: int):
        n, p = ctypes.c_int32(), ctypes.c_int32()
        _check(ee_seq_state(self.ctx, seq, ctypes.byref(n), ctypes.byref(p)), self.ctx)
        return n.value, p.value

    def logits(self) -> np.ndarray:
        rows = self._last_rows
        out = np.empty((rows, self.shape.vocab), dtype=np.float32)
        _check(ee_get_logits(self.ctx, out.ctypes.data_as(ctypes.POINTER(ctypes.c_float)), rows), self.ctx)
        return out

    def read_kv(self, seq: int, layer: int):
        n, _ = self.seq_state(seq)
        s = self.shape
        dt = np.uint16 if s.dtype == "bf16" else np.float32
        k = np.empty((n, s.n_kv_heads, s.head_dim), dtype=dt)
        v = np.empty_like(k)
        _check(ee_read_kv(self.ctx, seq, layer, k.ctypes.data, v.ctypes.data), self.ctx)
        return k, v

    def load_kv(self, seq: int, k, v, pending: int):
        """Install a committed cache in the empty sequence `seq`: k and v are
        [n_layers, n, n_kv_heads, head_dim] in the model dtype (bf16 bit
        patterns as uint16, or float32); `pending` starts the next block."""
        s = self.shape
        dt = np.uint16 if s.dtype == "bf16" else np.float32
        k = np.ascontiguousarray(k, dtype=dt)
        v = np.ascontiguousarray(v, dtype=dt)
        if k.shape != v.shape or k.ndim != 4 or k.shape[0] != s.n_layers or k.shape[2:] != (s.n_kv_heads, s.head_dim):
            raise EEError(EE_EINVAL, "k and v must be [n_layers, n, n_kv_heads, head_dim]")
        _check(ee_load_kv(self.ctx, seq, k.shape[1], int(pending), k.ctypes.data, v.ctypes.data), self.ctx)

    def capture(self, rows: int | None):
        """Start (rows: the row count of the blocks to capture) or end (None)
        recording every rounding site's values (ee_capture) into a device
        buffer of this engine; ``captured()`` reads the last block's."""
        if rows is None:     # the buffer stays readable until the next capture
            _check(ee_capture(self.ctx, None, 0), self.ctx)
            return
        nb = ee_capture_bytes(ctypes.byref(self.cfg), int(rows))
        if not nb:
            raise EEError(EE_EINVAL, "invalid capture row count")
        self._cap = torch.empty(nb, dtype=torch.uint8, device=self.device)
        self._cap_rows = int(rows)
        _check(ee_capture(self.ctx, self._cap.data_ptr(), nb), self.ctx)

    def captured(self):
        """{(site, layer): array} of the last captured block, in the model
        dtype (bf16 bit patterns as uint16): x_attn, o, x_ffn, z [rows, cols]
        and q [rows, n_heads, head_dim], k, v [rows, n_kv_heads, head_dim]
        per layer; x_final [rows, d_model] at layer n_layers."""
        s, R = self.shape, self._cap_rows
        torch.cuda.synchronize(self.device)
        raw = self._cap.cpu().numpy()
        dt, esz, ks = (np.uint16, 2, 32) if s.dtype == "bf16" else (np.float32, 4, 16)
        R16 = (R + 15) // 16 * 16
        off = 0

        def take(n):
            nonlocal off
            a = raw[off:off + n * esz].view(dt)
            off += n * esz
            return a

        def packed(cols):
            # fragments [R16/16][cols/KS][4 lane groups][16 lanes][KS/4 elements]
            a = take(R16 * cols).reshape(R16 // 16, cols // ks, 4, 16, ks // 4)
            return a.transpose(0, 3, 1, 2, 4).reshape(R16, cols)[:R]

        out = {}
        qd, kd = s.n_heads * s.head_dim, s.n_kv_heads * s.head_dim
        for l in range(s.n_layers):
            out[("x_attn", l)] = packed(s.d_model)
            out[("q", l)] = take(R * qd).reshape(R, s.n_heads, s.head_dim)
            out[("k", l)] = take(R * kd).reshape(R, s.n_kv_heads, s.head_dim)
            out[("v", l)] = take(R * kd).reshape(R, s.n_kv_heads, s.head_dim)
            out[("o", l)] = packed(qd)
            out[("x_ffn", l)] = packed(s.d_model)
            out[("z", l)] = packed(s.ffn)
        out[("x_final", s.n_layers)] = packed(s.d_model)
        assert off == len(raw)
        return out

    def use_graphs(self, on: bool):
        """Replay captured HIP graphs per block shape and attention split count
        (default) or launch eagerly."""
        _check(ee_use_graphs(self.ctx, int(bool(on))), self.ctx)

    def profile(self, classes=()):
        """Bracket launches of the named kernel classes with HIP events."""
        mask = 0
        for c in classes:
            mask |= 1 << PROF_CLASSES.index(c)
        _check(ee_profile(self.ctx, mask), self.ctx)

    def profile_read(self, reset: bool = True):
        """{class: (total ms, launches)} accumulated since the last reset."""
        ms = (ctypes.c_double * len(PROF_CLASSES))()
        n = (ctypes.c_int64 * len(PROF_CLASSES))()
        _check(ee_profile_read(self.ctx, ms, n, int(reset)), self.ctx)
        return {c: (ms[i], n[i]) for i, c in enumerate(PROF_CLASSES)}

    def time_gemm(self, cls: str, rows: int, reps: int = 3) -> float:
        """Microseconds per launch of one projection's GEMM, launched for every
        layer in turn, back to back (ee_time_gemm)."""
        us = ctypes.c_double()
        _check(ee_time_gemm(self.ctx, PROF_CLASSES.index(cls), rows, reps, ctypes.byref(us)), self.ctx)
        return us.value

    def time_stream_read(self, buf: torch.Tensor, reps: int = 10) -> float:
        """Microseconds per pass of a plain streaming read of the device
        tensor ``buf`` (ee_time_stream_read)."""
        us = ctypes.c_double()
        nb = buf.numel() * buf.element_size() // 16 * 16
        _check(ee_time_stream_read(self.ctx, buf.data_ptr(), nb, int(reps), ctypes.byref(us)), self.ctx)
        return us.value

    def close(self):
        if getattr(self, "ctx", None):
            _check(ee_destroy(self.ctx))
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class EditSession:
    """An edit session over a target engine's sequence and, optionally, a
    draft engine's sequence holding the same prompt (ee_edit_begin /
    ee_edit_step).  ``output`` is the emitted token stream so far."""

    def __init__(self, target: Engine, seq: int, original, draft: Engine | None = None, draft_seq: int = 0,
                 k_reuse: int = 32, gamma: int = 7, top_k: int = 0, dynamic: bool = True,
                 min_match: int = 3, max_match: int = 8, capacity: int = 1 << 16):
        self.target, self.seq, self.draft, self.draft_seq = target, seq, draft, draft_seq
        self.original, self._op = _i32arr(original)
        self.params = EEEditParams(k_reuse, gamma, top_k, int(bool(dynamic)), min_match, max_match)
        self.state = EEEditState()
        _check(ee_edit_begin(target.ctx, seq, draft.ctx if draft else None, draft_seq,
                             ctypes.byref(self.state)), target.ctx)
        self._out = np.zeros(capacity, dtype=np.int32)
        self._out[0] = target.seq_state(seq)[1]
        self.n = 1

    @property
    def output(self):
        return self._out[:self.n].tolist()

    def step(self):
        """One Reuse or Generate step; returns (phase, new tokens)."""
        nn = ctypes.c_int32()
        _check(ee_edit_step(self.target.ctx, self.seq, self.draft.ctx if self.draft else None, self.draft_seq,
                            self._op, len(self.original), ctypes.byref(self.params), ctypes.byref(self.state),
                            self._out.ctypes.data_as(_pi32), self.n, len(self._out), ctypes.byref(nn)),
               self.target.ctx)
        new = self._out[self.n:self.n + nn.value].tolist()
        self.n += nn.value
        return self.state.last_phase, new
