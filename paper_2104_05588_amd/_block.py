"""ctypes binding of the transformer block's operators of libdaso.so (declared in include/daso_block.h): the norm and
rotation of queries and keys, attention over packed sequences, and the norm and clipping of averaged gradients.

As in _train: tensors are checked and their addresses and the current HIP stream cross the C ABI, outputs that are
not given and workspaces come from torch's allocator on the stream that the call runs on, and nothing is recorded by
autograd: the *_backward functions return the gradients."""
from __future__ import annotations

import ctypes
import math
from typing import Optional, Sequence, Tuple

import torch

from . import _lib as L
from . import _train as T

DASO_ROTARY_INTERLEAVED = 1
DASO_ATTENTION_CAUSAL, DASO_ATTENTION_ZERO_Q, DASO_ATTENTION_ZERO_K, DASO_ATTENTION_ZERO_V = 1, 2, 4, 8
DASO_MAX_HEAD_DIM = 128
DASO_MAX_HEADS = 1024
DASO_MAX_TOKENS = 1 << 24
DASO_MAX_SEQUENCES = 1 << 20
EXPORTED_BLOCK = ("daso_head_norm_rotary", "daso_head_norm_rotary_backward_workspace", "daso_head_norm_rotary_backward",
                  "daso_attention", "daso_attention_backward_workspace", "daso_attention_backward",
                  "daso_clip_gradients_workspace", "daso_clip_gradients")

_vp, _i32, _i64, _u32, _f32, _size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32, ctypes.c_float, ctypes.c_size_t


class daso_heads(ctypes.Structure):
    _fields_ = [("data", _vp), ("token_stride", _i64), ("head_stride", _i64)]


class daso_rotary_args(ctypes.Structure):
    _fields_ = [("tokens", _i64), ("heads", _i32), ("kv_heads", _i32), ("dim", _i32), ("rotated", _i32), ("type", _i32),
                ("eps", _f32), ("flags", _u32), ("reserved", _u32), ("positions", _vp), ("frequencies", _vp),
                ("q_weight", _vp), ("k_weight", _vp), ("q", daso_heads), ("k", daso_heads), ("q_out", daso_heads),
                ("k_out", daso_heads), ("dq_out", daso_heads), ("dk_out", daso_heads), ("dq", daso_heads),
                ("dk", daso_heads), ("dq_weight", _vp), ("dk_weight", _vp), ("workspace", _vp), ("workspace_bytes", _size)]


class daso_attention_args(ctypes.Structure):
    _fields_ = [("tokens", _i64), ("heads", _i32), ("kv_heads", _i32), ("dim", _i32), ("type", _i32), ("sequences", _i32),
                ("flags", _u32), ("scale", _f32), ("reserved", _u32), ("offsets", _vp), ("q", daso_heads), ("k", daso_heads),
                ("v", daso_heads), ("out", daso_heads), ("lse", _vp), ("dout", daso_heads), ("dq", daso_heads),
                ("dk", daso_heads), ("dv", daso_heads), ("workspace", _vp), ("workspace_bytes", _size)]


class daso_span(ctypes.Structure):
    _fields_ = [("start", _i64), ("n", _i64)]


class daso_clip_args(ctypes.Structure):
    _fields_ = [("n", _i64), ("g", _i32), ("ntensors", _i32), ("grads", ctypes.POINTER(_vp)),
                ("tensors", ctypes.POINTER(daso_span)), ("out", _vp), ("norm", _vp), ("norms", _vp), ("max_norm", _f32),
                ("eps", _f32), ("workspace", _vp), ("workspace_bytes", _size)]


_typed = False


def _load() -> ctypes.CDLL:
    global _typed
    lib = T._load()
    if not _typed:
        for name, struct in (("daso_head_norm_rotary", daso_rotary_args), ("daso_head_norm_rotary_backward", daso_rotary_args),
                             ("daso_attention", daso_attention_args), ("daso_attention_backward", daso_attention_args),
                             ("daso_clip_gradients", daso_clip_args)):
            getattr(lib, name).argtypes = [ctypes.POINTER(struct), _vp]
        for name, struct in (("daso_head_norm_rotary_backward_workspace", daso_rotary_args),
                             ("daso_attention_backward_workspace", daso_attention_args),
                             ("daso_clip_gradients_workspace", daso_clip_args)):
            getattr(lib, name).argtypes = [ctypes.POINTER(struct), ctypes.POINTER(_size)]
        for name in EXPORTED_BLOCK:
            getattr(lib, name).restype = ctypes.c_int
        _typed = True
    return lib


# ------------------------------------------------------------- marshalling
def _heads(t: torch.Tensor, shape: Tuple[int, int, int], dtypes, what: str) -> daso_heads:
    """Address and strides of tokens x heads rows whose elements are contiguous."""
    if t.dtype not in dtypes or not t.is_cuda or t.get_device() != torch.cuda.current_device():
        T._device_tensor(t, dtypes, what)
    if t.shape != shape:
        raise ValueError(f"{what} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    token, head, each = t.stride()
    if each != 1 and shape[2] > 1:
        raise ValueError(f"the rows of {what} must be contiguous")
    return daso_heads(t.data_ptr(), token, head)


def _shape_of(x: torch.Tensor, what: str) -> Tuple[int, int, int]:
    if x.dim() != 3:
        raise ValueError(f"{what} must be [tokens, heads, elements], got {x.dim()} dimensions")
    return tuple(x.shape)


# ------------------------------------------------------- norm and rotation
def rotary_frequencies(rotated: int, base: float = 10000.0, device="cuda") -> torch.Tensor:
    """The usual frequencies, base^(-2 j / rotated) radians a position for each of rotated / 2 pairs (float64)."""
    if rotated < 0 or rotated % 2:
        raise ValueError("the rotated elements are pairs")
    return float(base) ** (torch.arange(0, rotated, 2, dtype=torch.float64, device=device) / -max(rotated, 1))


def _rotary_args(q, k, positions, frequencies, q_weight, k_weight, eps, interleaved) -> daso_rotary_args:
    n, heads, dim = _shape_of(q, "q")
    kn, kv, kdim = _shape_of(k, "k")
    if kn != n or kdim != dim:
        raise ValueError(f"q has {n} tokens of {dim} elements a head and k {kn} of {kdim}")
    a = daso_rotary_args()
    a.tokens, a.heads, a.kv_heads, a.dim = n, heads, kv, dim
    a.eps, a.flags = float(eps), DASO_ROTARY_INTERLEAVED if interleaved else 0
    a.q, a.k = _heads(q, q.shape, T._FLOATS, "q"), _heads(k, k.shape, (q.dtype,), "k")
    a.type = T._TYPES[q.dtype]
    a.positions = T._flat(positions, n, (torch.int64,), "positions")
    a.rotated = 2 * frequencies.numel()
    a.frequencies = T._flat(frequencies, frequencies.numel(), (torch.float64,), "frequencies")
    a.q_weight, a.k_weight = T._flat(q_weight, dim, T._F32, "q_weight"), T._flat(k_weight, dim, T._F32, "k_weight")
    return a


def head_norm_rotary(q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor, frequencies: torch.Tensor,
                     q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                     interleaved: bool = False, out_q: Optional[torch.Tensor] = None, out_k: Optional[torch.Tensor] = None,
                     stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The root-mean-square norm of each head of q [tokens, heads, dim] and k [tokens, kv_heads, dim] (bf16 or fp32, a
    head's elements contiguous, dim a multiple of 8 up to 128), and its rotation by the token's position (int64 [tokens])
    times the frequencies (float64, a multiple of 4 of them; see rotary_frequencies): of the pairs (j, j + rotated / 2), or
    neighbours if `interleaved`.  The weights are fp32 [dim].  out_q and out_k may be q and k, with the same strides.  Not recorded by
    autograd, whatever the inputs require: head_norm_rotary_backward gives the gradients."""
    a = _rotary_args(q, k, positions, frequencies, q_weight, k_weight, eps, interleaved)
    with T._on(stream):
        out_q = torch.empty(q.shape, dtype=q.dtype, device=q.device) if out_q is None else out_q
        out_k = torch.empty(k.shape, dtype=q.dtype, device=q.device) if out_k is None else out_k
        a.q_out, a.k_out = _heads(out_q, q.shape, (q.dtype,), "out_q"), _heads(out_k, k.shape, (q.dtype,), "out_k")
        L._check(_load().daso_head_norm_rotary(ctypes.byref(a), L._stream_handle(stream)), "daso_head_norm_rotary")
    return out_q, out_k


def head_norm_rotary_backward(dq_out: torch.Tensor, dk_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor,
                              positions: torch.Tensor, frequencies: torch.Tensor, q_weight: Optional[torch.Tensor] = None,
                              k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, interleaved: bool = False,
                              dq: Optional[torch.Tensor] = None, dk: Optional[torch.Tensor] = None,
                              dq_weight: Optional[torch.Tensor] = None, dk_weight: Optional[torch.Tensor] = None,
                              stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]:
    """dq, dk, dq_weight and dk_weight from the gradients dq_out and dk_out of what head_norm_rotary gave for q and k.  dq
    and dk may be dq_out and dk_out; the weights' gradients are fp32 [dim], may be views of a flat gradient buffer, and are computed in any
    case: without weights, for ones."""
    a = _rotary_args(q, k, positions, frequencies, q_weight, k_weight, eps, interleaved)
    dim = a.dim
    a.dq_out, a.dk_out = _heads(dq_out, q.shape, (q.dtype,), "dq_out"), _heads(dk_out, k.shape, (q.dtype,), "dk_out")
    with T._on(stream):
        dq = torch.empty(q.shape, dtype=q.dtype, device=q.device) if dq is None else dq
        dk = torch.empty(k.shape, dtype=q.dtype, device=q.device) if dk is None else dk
        dq_weight = torch.empty(dim, dtype=torch.float32, device=q.device) if dq_weight is None else dq_weight
        dk_weight = torch.empty(dim, dtype=torch.float32, device=q.device) if dk_weight is None else dk_weight
        a.dq, a.dk = _heads(dq, q.shape, (q.dtype,), "dq"), _heads(dk, k.shape, (q.dtype,), "dk")
        a.dq_weight, a.dk_weight = T._flat(dq_weight, dim, T._F32, "dq_weight"), T._flat(dk_weight, dim, T._F32, "dk_weight")
        ws = _workspace("daso_head_norm_rotary_backward_workspace", a)  # noqa: F841 (held until the call is queued)
        L._check(_load().daso_head_norm_rotary_backward(ctypes.byref(a), L._stream_handle(stream)), "daso_head_norm_rotary_backward")
    return dq, dk, dq_weight, dk_weight


def _workspace(name: str, args) -> Optional[torch.Tensor]:
    _load()
    return T._workspace(name, args)


# --------------------------------------------------------------- attention
def _attention_args(q, k, v, offsets, causal, scale) -> daso_attention_args:
    n, heads, dim = _shape_of(q, "q")
    kn, kv, kdim = _shape_of(k, "k")
    if kn != n or kdim != dim:
        raise ValueError(f"q has {n} tokens of {dim} elements a head and k {kn} of {kdim}")
    a = daso_attention_args()
    a.tokens, a.heads, a.kv_heads, a.dim = n, heads, kv, dim
    a.q, a.k, a.v = _heads(q, q.shape, T._FLOATS, "q"), _heads(k, k.shape, (q.dtype,), "k"), _heads(v, k.shape, (q.dtype,), "v")
    a.type = T._TYPES[q.dtype]
    a.flags = DASO_ATTENTION_CAUSAL if causal else 0
    a.scale = 1.0 / math.sqrt(max(dim, 1)) if scale is None else float(scale)
    if offsets is None:
        a.sequences = 1
    else:
        if offsets.numel() < 1:
            raise ValueError("offsets are one more than the sequences")
        a.sequences = offsets.numel() - 1
        a.offsets = T._flat(offsets, offsets.numel(), (torch.int64,), "offsets")
    return a


def packed_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, offsets: Optional[torch.Tensor] = None,
                     causal: bool = True, scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                     lse: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Attention of each token of q [tokens, heads, dim] to those of its sequence (up to itself if `causal`) in k and v
    [tokens, kv_heads, dim], whose heads are shared by heads / kv_heads neighbouring query heads: out, of q's shape, and the
    log-sum-exp of the scores, fp32 [heads, tokens].  bf16 or fp32, a head's elements contiguous, dim a multiple of 8 up to
    128.  offsets (int64, on the device) holds the first token of each sequence and, last, where they end; without it
    all tokens are one sequence.  Pairs of offsets that fall, pass the tokens or begin before the end of an earlier one are empty
    sequences.  Rows of tokens in no sequence, as those behind the last, are left as they are; in an out made here they are zeros;
    lse's follow out's.  Meant for sequences of dozens of tokens and more, some thousands at most: short ones cost as much as ones of 128
    tokens, and beyond that the time grows with the square of their number.
    scale is 1 / sqrt(dim) unless given.  Not recorded by autograd, whatever the inputs require: packed_attention_backward gives the
    gradients."""
    a = _attention_args(q, k, v, offsets, causal, scale)
    with T._on(stream):
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
            a.flags |= DASO_ATTENTION_ZERO_Q
        lse = torch.empty((a.heads, a.tokens), dtype=torch.float32, device=q.device) if lse is None else lse
        a.out = _heads(out, q.shape, (q.dtype,), "out")
        a.lse = T._flat(lse, a.heads * a.tokens, T._F32, "lse")
        L._check(_load().daso_attention(ctypes.byref(a), L._stream_handle(stream)), "daso_attention")
    return out, lse


def packed_attention_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                              lse: torch.Tensor, offsets: Optional[torch.Tensor] = None, causal: bool = True,
                              scale: Optional[float] = None, dq: Optional[torch.Tensor] = None,
                              dk: Optional[torch.Tensor] = None, dv: Optional[torch.Tensor] = None,
                              stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """dq, dk and dv from the gradient dout of what packed_attention gave (out and lse) for the same arguments.  They may be
    given, for instance as parts of one gradient of a joint projection: then the rows of tokens in no sequence are left as
    they are, else they are zeros."""
    a = _attention_args(q, k, v, offsets, causal, scale)
    a.out, a.dout = _heads(out, q.shape, (q.dtype,), "out"), _heads(dout, q.shape, (q.dtype,), "dout")
    a.lse = T._flat(lse, a.heads * a.tokens, T._F32, "lse")
    with T._on(stream):
        if dq is None:
            dq = torch.empty(q.shape, dtype=q.dtype, device=q.device)
            a.flags |= DASO_ATTENTION_ZERO_Q
        if dk is None:
            dk = torch.empty(k.shape, dtype=q.dtype, device=q.device)
            a.flags |= DASO_ATTENTION_ZERO_K
        if dv is None:
            dv = torch.empty(k.shape, dtype=q.dtype, device=q.device)
            a.flags |= DASO_ATTENTION_ZERO_V
        a.dq, a.dk, a.dv = _heads(dq, q.shape, (q.dtype,), "dq"), _heads(dk, k.shape, (q.dtype,), "dk"), _heads(dv, k.shape, (q.dtype,), "dv")
        ws = _workspace("daso_attention_backward_workspace", a)  # noqa: F841
        L._check(_load().daso_attention_backward(ctypes.byref(a), L._stream_handle(stream)), "daso_attention_backward")
    return dq, dk, dv


# ---------------------------------------------------------------- clipping
def _clip(grads, max_norm, tensors, out, eps, stream) -> Tuple[torch.Tensor, torch.Tensor]:
    if not len(grads):
        raise ValueError("clipping needs a gradient buffer")
    n = grads[0].numel()
    a = daso_clip_args()
    at = L._ptr_array(grads, T._F32, n, "grads")
    a.n, a.g, a.grads = n, len(grads), at
    count = 1
    if tensors is not None:
        count = len(tensors)
        spans = (daso_span * max(count, 1))()
        for span, (start, k) in zip(spans, tensors):
            span.start, span.n = start, k
        if count == 0:  # no tensors: not the whole buffer, but nothing
            a.ntensors = 1
        else:
            a.ntensors = count
        a.tensors = spans
    a.out = L._ptr(out, T._F32, n, "out")
    a.max_norm, a.eps = float(max_norm), float(eps)
    with T._on(stream):
        norm = torch.empty((), dtype=torch.float32, device=grads[0].device)
        norms = torch.empty(count, dtype=torch.float32, device=grads[0].device)
        a.norm, a.norms = norm.data_ptr(), norms.data_ptr() if count else None
        ws = _workspace("daso_clip_gradients_workspace", a)  # noqa: F841
        L._check(_load().daso_clip_gradients(ctypes.byref(a), L._stream_handle(stream)), "daso_clip_gradients")
    return norm, norms


def gradient_norm(grads: Sequence[torch.Tensor], tensors: Optional[Sequence[Tuple[int, int]]] = None,
                  stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The norm of the mean of the replicas' flat fp32 gradient buffers over all elements of the tensors, (start, elements)
    in ascending order (without them, of the buffer), and each tensor's own norm: fp32 [] and [tensors]."""
    return _clip(grads, math.inf, tensors, None, 0.0, stream)


def clip_gradients(grads: Sequence[torch.Tensor], max_norm: float, tensors: Optional[Sequence[Tuple[int, int]]] = None,
                   out: Optional[torch.Tensor] = None, eps: float = 1e-6, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The mean of the replicas' flat fp32 gradient buffers, scaled down to max_norm where its norm over all tensors is larger:
    out = mean * min(1, max_norm / (norm + eps)), and what gradient_norm returns.  max_norm and eps are taken as fp32.  out is the first buffer unless given, and
    may be any of them; a step then takes it as the gradient of one replica.  Elements outside the tensors stay as
    they are."""
    return _clip(grads, max_norm, tensors, grads[0] if out is None and len(grads) else out, eps, stream)
