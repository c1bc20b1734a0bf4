"""ctypes binding of the training operators of libdaso.so (declared in include/daso_train.h):
layer norm, the cross entropy of an output projection, and orthogonalised updates.

As in _lib: tensors are checked and their addresses and the current HIP stream cross the C ABI;
every step of the computation runs in the library's kernels.  Outputs that are not
given, and workspaces, come from torch's allocator, on the stream that the call runs on.

Nothing here is recorded by autograd: results of tensors that require a gradient have no history, and the gradients are what the
*_backward functions return."""
from __future__ import annotations

import contextlib
import ctypes
import math
from typing import Optional, Sequence, Tuple

import torch

from . import _lib as L

DASO_TYPE_F32, DASO_TYPE_BF16 = 0, 1
DASO_MUON_NESTEROV = 1
DASO_MAX_NORM_D = 65536
DASO_MAX_SIDE = 1 << 20
DASO_MAX_SCHULZ_STEPS = 16
EXPORTED_TRAIN = ("daso_layer_norm", "daso_layer_norm_backward_workspace", "daso_layer_norm_backward",
                  "daso_linear_cross_entropy_workspace", "daso_linear_cross_entropy",
                  "daso_linear_cross_entropy_backward", "daso_orthogonalize_workspace", "daso_orthogonalize",
                  "daso_muon_workspace", "daso_muon_step")

MUON_COEFFICIENTS = (3.4445, -4.7750, 2.0315)  # the quintic in common use; five steps

_TYPES = {torch.float32: DASO_TYPE_F32, torch.bfloat16: DASO_TYPE_BF16}
_vp, _i32, _i64, _f32, _size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t


class daso_layer_norm_args(ctypes.Structure):
    _fields_ = [("rows", _i64), ("d", _i64), ("type", _i32), ("eps", _f32), ("x", _vp), ("x_stride", _i64),
                ("weight", _vp), ("bias", _vp), ("y", _vp), ("y_stride", _i64), ("mean", _vp), ("rstd", _vp)]


class daso_layer_norm_backward_args(ctypes.Structure):
    _fields_ = [("rows", _i64), ("d", _i64), ("type", _i32), ("reserved", _i32), ("dy", _vp), ("dy_stride", _i64),
                ("x", _vp), ("x_stride", _i64), ("weight", _vp), ("mean", _vp), ("rstd", _vp), ("dx", _vp),
                ("dx_stride", _i64), ("dweight", _vp), ("dbias", _vp), ("workspace", _vp), ("workspace_bytes", _size)]


class daso_loss_args(ctypes.Structure):
    _fields_ = [("tokens", _i64), ("vocab", _i64), ("d", _i64), ("type", _i32), ("dweight_type", _i32),
                ("hidden", _vp), ("hidden_stride", _i64), ("weight", _vp), ("weight_stride", _i64), ("targets", _vp),
                ("ignore_index", _i64), ("loss", _vp), ("lse", _vp), ("dloss", _vp), ("dhidden", _vp),
                ("dhidden_stride", _i64), ("dweight", _vp), ("dweight_stride", _i64), ("workspace", _vp),
                ("workspace_bytes", _size)]


class daso_orthogonalize_args(ctypes.Structure):
    _fields_ = [("batch", _i64), ("rows", _i64), ("cols", _i64), ("type", _i32), ("out_type", _i32), ("src", _vp),
                ("src_batch_stride", _i64), ("src_stride", _i64), ("out", _vp), ("out_batch_stride", _i64),
                ("out_stride", _i64), ("steps", _i32), ("eps", _f32), ("coefficients", ctypes.POINTER(_f32)),
                ("workspace", _vp), ("workspace_bytes", _size)]


class daso_matrix(ctypes.Structure):
    _fields_ = [("start", _i64), ("rows", _i32), ("cols", _i32), ("scale", _f32), ("reserved", ctypes.c_uint32)]


class daso_muon_args(ctypes.Structure):
    _fields_ = [("n", _i64), ("g", _i32), ("nmatrices", _i32), ("grads", ctypes.POINTER(_vp)), ("params", _vp),
                ("momentum", _vp), ("wire", _vp), ("matrices", ctypes.POINTER(daso_matrix)), ("lr", _f32), ("mu", _f32),
                ("weight_decay", _f32), ("eps", _f32), ("coefficients", ctypes.POINTER(_f32)), ("steps", _i32),
                ("flags", ctypes.c_uint32), ("workspace", _vp), ("workspace_bytes", _size)]


_typed = False


def _load() -> ctypes.CDLL:
    global _typed
    lib = L.load()
    if not _typed:
        sized = ctypes.POINTER(_size)
        for name, struct in (("daso_layer_norm", daso_layer_norm_args),
                             ("daso_layer_norm_backward", daso_layer_norm_backward_args),
                             ("daso_linear_cross_entropy", daso_loss_args),
                             ("daso_linear_cross_entropy_backward", daso_loss_args),
                             ("daso_orthogonalize", daso_orthogonalize_args), ("daso_muon_step", daso_muon_args)):
            getattr(lib, name).argtypes = [ctypes.POINTER(struct), _vp]
        lib.daso_layer_norm_backward_workspace.argtypes = [ctypes.POINTER(daso_layer_norm_backward_args), sized]
        lib.daso_linear_cross_entropy_workspace.argtypes = [ctypes.POINTER(daso_loss_args), ctypes.c_int, sized]
        lib.daso_orthogonalize_workspace.argtypes = [ctypes.POINTER(daso_orthogonalize_args), sized]
        lib.daso_muon_workspace.argtypes = [ctypes.POINTER(daso_muon_args), sized]
        for name in EXPORTED_TRAIN:
            getattr(lib, name).restype = ctypes.c_int
        _typed = True
    return lib


# ------------------------------------------------------------- marshalling
def _device_tensor(t: torch.Tensor, dtypes, what: str) -> torch.Tensor:
    # (get_device costs a third of device.index, and is -1 off the device)
    if t.is_cuda and t.dtype in dtypes and t.get_device() == torch.cuda.current_device():
        return t
    if not t.is_cuda:
        raise ValueError(f"{what} must be a device tensor")
    if t.device.index != torch.cuda.current_device():
        raise ValueError(f"{what} is on {t.device}, not on the current device cuda:{torch.cuda.current_device()}")
    raise ValueError(f"{what} must have dtype in {tuple(dtypes)}, got {t.dtype}")


def _rows(t: torch.Tensor, shape: Tuple[int, int], dtypes, what: str) -> Tuple[int, int]:
    """Address and row stride of a matrix whose rows are contiguous."""
    _device_tensor(t, dtypes, what)
    if t.shape != shape:
        raise ValueError(f"{what} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    rows, cols = shape
    row, col = t.stride()
    if (cols > 1 and col != 1) or (rows > 1 and row < cols):
        raise ValueError(f"the rows of {what} must be contiguous and must not overlap")
    return t.data_ptr(), row if rows > 1 else max(cols, 1)


def _flat(t: Optional[torch.Tensor], n: int, dtypes, what: str) -> Optional[int]:
    if t is None:
        return None
    if (t.numel() != n or not t.is_contiguous() or not t.is_cuda or t.dtype not in dtypes
            or t.get_device() != torch.cuda.current_device()):
        _device_tensor(t, dtypes, what)
        raise ValueError(f"{what} must be contiguous with {n} elements")
    return t.data_ptr()


def _on(stream: Optional[torch.cuda.Stream]):
    """What is allocated for a call belongs to the stream that the call runs on, which is one of the current device:
    torch.cuda.stream would make another one current, under tensors of this one."""
    if stream is None:
        return _HERE
    if stream.device_index != torch.cuda.current_device():
        raise ValueError(f"the stream is of cuda:{stream.device_index}, not of the current device cuda:{torch.cuda.current_device()}")
    return torch.cuda.stream(stream)


_HERE = contextlib.nullcontext()


def _workspace(name: str, args, *more) -> Optional[torch.Tensor]:
    need = _size()
    L._check(getattr(_load(), name)(ctypes.byref(args), *more, ctypes.byref(need)), name)
    if need.value == 0:
        return None
    ws = torch.empty(need.value, dtype=torch.uint8, device="cuda")
    args.workspace, args.workspace_bytes = ws.data_ptr(), need.value
    return ws


_F32 = (torch.float32,)
_FLOATS = (torch.float32, torch.bfloat16)


def _matrix_of(x: torch.Tensor, what: str) -> Tuple[int, int]:
    if x.dim() != 2:
        raise ValueError(f"{what} must be a matrix, got {x.dim()} dimensions")
    return x.shape[0], x.shape[1]


# --------------------------------------------------------------- layer norm
def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
               eps: float = 1e-5, out: Optional[torch.Tensor] = None,
               stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """y, mean and rstd of the layer norm of each row of x [rows, d] (bf16 or fp32, rows
    contiguous); weight and bias are fp32 [d]; mean and rstd fp32 [rows].  `out` may be x."""
    rows, d = _matrix_of(x, "x")
    x_at, x_stride = _rows(x, (rows, d), _FLOATS, "x")
    weight_at, bias_at = _flat(weight, d, _F32, "weight"), _flat(bias, d, _F32, "bias")
    with _on(stream):
        if out is None:
            y = x.new_empty((rows, d))
            y_at, y_stride = y.data_ptr(), max(d, 1)
        else:
            y = out
            y_at, y_stride = _rows(y, (rows, d), (x.dtype,), "out")
        mean = x.new_empty(rows, dtype=torch.float32)
        rstd = torch.empty_like(mean)
        if d == 0:  # the call is a no-op; a row of no elements has the statistics 0 / 0
            mean.fill_(math.nan)
            rstd.fill_(math.nan)
        a = daso_layer_norm_args(rows, d, _TYPES[x.dtype], eps, x_at, x_stride, weight_at, bias_at, y_at, y_stride,
                                 mean.data_ptr(), rstd.data_ptr())
        L._check(_load().daso_layer_norm(ctypes.byref(a), L._stream_handle(stream)), "daso_layer_norm")
    return y, mean, rstd


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: Optional[torch.Tensor], mean: torch.Tensor,
                        rstd: torch.Tensor, bias: bool = True, dx: Optional[torch.Tensor] = None,
                        dweight: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None,
                        stream=None) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
    """dx, dweight and dbias (None without `bias`) from dy and what the forward pass gave.
    dx has x's type and may be dy; dweight and dbias are fp32 [d], and may be views of a flat
    gradient buffer."""
    rows, d = _matrix_of(x, "x")
    a = daso_layer_norm_backward_args()
    a.rows, a.d = rows, d
    a.x, a.x_stride = _rows(x, (rows, d), _FLOATS, "x")
    a.type = _TYPES[x.dtype]
    a.dy, a.dy_stride = _rows(dy, (rows, d), (x.dtype,), "dy")
    a.weight = _flat(weight, d, _F32, "weight")
    a.mean, a.rstd = _flat(mean, rows, _F32, "mean"), _flat(rstd, rows, _F32, "rstd")
    with _on(stream):
        dx = torch.empty((rows, d), dtype=x.dtype, device=x.device) if dx is None else dx
        dweight = torch.empty(d, dtype=torch.float32, device=x.device) if dweight is None else dweight
        if bias and dbias is None:
            dbias = torch.empty(d, dtype=torch.float32, device=x.device)
        a.dx, a.dx_stride = _rows(dx, (rows, d), (x.dtype,), "dx")
        a.dweight, a.dbias = _flat(dweight, d, _F32, "dweight"), _flat(dbias, d, _F32, "dbias")
        ws = _workspace("daso_layer_norm_backward_workspace", a)  # noqa: F841 (held until the call is queued)
        L._check(_load().daso_layer_norm_backward(ctypes.byref(a), L._stream_handle(stream)), "daso_layer_norm_backward")
    return dx, dweight, dbias


# ----------------------------------------------------------------- the loss
def _loss_args(hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, ignore_index: int) -> daso_loss_args:
    n, d = _matrix_of(hidden, "hidden")
    vocab, wd = _matrix_of(weight, "weight")
    if wd != d:
        raise ValueError(f"hidden has {d} features and weight {wd}")
    a = daso_loss_args()
    a.tokens, a.vocab, a.d = n, vocab, d
    a.hidden, a.hidden_stride = _rows(hidden, (n, d), _FLOATS, "hidden")
    a.weight, a.weight_stride = _rows(weight, (vocab, d), (hidden.dtype,), "weight")
    a.type = a.dweight_type = _TYPES[hidden.dtype]
    a.targets = _flat(targets, n, (torch.int64,), "targets")
    a.ignore_index = int(ignore_index)
    return a


def linear_cross_entropy(hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, ignore_index: int = -100,
                         stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Each token's cross entropy of the logits hidden weight^T, and their log-sum-exp
    (fp32 [tokens] both), without the logits in memory.  hidden [tokens, d] and weight
    [vocab, d] are both bf16 or both fp32; targets int64 [tokens], whose ignore_index gives 0."""
    a = _loss_args(hidden, weight, targets, ignore_index)
    with _on(stream):
        loss = torch.empty(a.tokens, dtype=torch.float32, device=hidden.device)
        lse = torch.empty(a.tokens, dtype=torch.float32, device=hidden.device)
        a.loss, a.lse = loss.data_ptr(), lse.data_ptr()
        ws = _workspace("daso_linear_cross_entropy_workspace", a, 0)  # noqa: F841
        L._check(_load().daso_linear_cross_entropy(ctypes.byref(a), L._stream_handle(stream)), "daso_linear_cross_entropy")
    return loss, lse


def linear_cross_entropy_backward(dloss: torch.Tensor, hidden: torch.Tensor, weight: torch.Tensor,
                                  targets: torch.Tensor, lse: torch.Tensor, ignore_index: int = -100,
                                  dhidden: Optional[torch.Tensor] = None, dweight: Optional[torch.Tensor] = None,
                                  stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """dhidden [tokens, d] (hidden's type) and dweight [vocab, d] from the gradient dloss
    (fp32 [tokens]) of each token's loss.  dweight may be given as fp32 or bf16, for
    instance a view of a flat fp32 gradient buffer; else it has weight's type."""
    a = _loss_args(hidden, weight, targets, ignore_index)
    n, d, vocab = a.tokens, a.d, a.vocab
    a.dloss, a.lse = _flat(dloss, n, _F32, "dloss"), _flat(lse, n, _F32, "lse")
    with _on(stream):
        dhidden = torch.empty((n, d), dtype=hidden.dtype, device=hidden.device) if dhidden is None else dhidden
        dweight = torch.empty((vocab, d), dtype=weight.dtype, device=hidden.device) if dweight is None else dweight
        a.dhidden, a.dhidden_stride = _rows(dhidden, (n, d), (hidden.dtype,), "dhidden")
        a.dweight, a.dweight_stride = _rows(dweight, (vocab, d), _FLOATS, "dweight")
        a.dweight_type = _TYPES[dweight.dtype]
        ws = _workspace("daso_linear_cross_entropy_workspace", a, 1)  # noqa: F841
        L._check(_load().daso_linear_cross_entropy_backward(ctypes.byref(a), L._stream_handle(stream)),
                 "daso_linear_cross_entropy_backward")
    return dhidden, dweight


# ------------------------------------------------------- orthogonalised updates
def _coefficients(steps: int, coefficients: Sequence) -> ctypes.Array:
    """3 * steps floats: one (a, b, c) for all steps, or one a step."""
    if not 1 <= int(steps) <= DASO_MAX_SCHULZ_STEPS:
        raise ValueError(f"steps must be in 1..{DASO_MAX_SCHULZ_STEPS}")
    rows = list(coefficients)
    if len(rows) == 3 and not hasattr(rows[0], "__len__"):
        rows = [rows] * int(steps)
    if len(rows) != int(steps) or any(len(r) != 3 for r in rows):
        raise ValueError("coefficients are one (a, b, c), or one for each step")
    return (_f32 * (3 * int(steps)))(*[float(v) for r in rows for v in r])


def orthogonalize(src: torch.Tensor, steps: int = 5, coefficients: Sequence = MUON_COEFFICIENTS, eps: float = 1e-7,
                  out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Newton-Schulz orthogonalisation of src ([rows, cols], or a batch of them; bf16 or
    fp32).  The result has src's type, or that of `out` (which may be src); an fp32 result takes
    three times the products of a bf16 one."""
    if src.dim() not in (2, 3):
        raise ValueError(f"src must have 2 or 3 dimensions, got {src.dim()}")
    _device_tensor(src, _FLOATS, "src")
    with _on(stream):
        result = torch.empty(src.shape, dtype=src.dtype, device=src.device) if out is None else out
        _device_tensor(result, _FLOATS, "out")
        if result.shape != src.shape:
            raise ValueError(f"out must have shape {tuple(src.shape)}, got {tuple(result.shape)}")
        a = daso_orthogonalize_args()
        s, o = (src, result) if src.dim() == 3 else (src[None], result[None])
        a.batch, a.rows, a.cols = s.shape
        for t, what in ((s, "src"), (o, "out")):
            if t.numel() and ((a.cols > 1 and t.stride(2) != 1) or (a.rows > 1 and t.stride(1) < a.cols)):
                raise ValueError(f"the rows of {what} must be contiguous and must not overlap")
        a.type, a.out_type = _TYPES[s.dtype], _TYPES[o.dtype]
        a.src, a.out = s.data_ptr(), o.data_ptr()
        a.src_stride = s.stride(1) if a.rows > 1 else max(a.cols, 1)
        a.out_stride = o.stride(1) if a.rows > 1 else max(a.cols, 1)
        a.src_batch_stride = s.stride(0) if a.batch > 1 else 0
        a.out_batch_stride = o.stride(0) if a.batch > 1 else 0
        c = _coefficients(steps, coefficients)
        a.steps, a.eps, a.coefficients = int(steps), float(eps), c
        ws = _workspace("daso_orthogonalize_workspace", a)  # noqa: F841
        L._check(_load().daso_orthogonalize(ctypes.byref(a), L._stream_handle(stream)), "daso_orthogonalize")
    return result


def muon_scale(rows: int, cols: int, adjust: Optional[str] = "spectral") -> float:
    """The factor of a matrix's update: "spectral" sqrt(max(1, rows / cols)), "rms"
    0.2 sqrt(max(rows, cols)) (the size of an Adam update), None 1."""
    if adjust is None:
        return 1.0
    if adjust == "spectral":
        return math.sqrt(max(1.0, rows / cols))
    if adjust == "rms":
        return 0.2 * math.sqrt(max(rows, cols))
    raise ValueError("adjust is 'spectral', 'rms' or None")


class MuonStep:
    """A prepared daso_muon_step: argument checks, marshalling and the workspace happen once
    here, so that each call costs one C call.  grads are g fp32 flat buffers, params and
    momentum fp32 (updated in place), matrices the (start, rows, cols) that are stepped; wire
    receives their bf16 form.  The tensors must stay alive (and keep their storage)
    while the object is used, and so must the object while a graph that a call was captured into is replayed;
    calls on it must not overlap.  They may run on any stream: the first on a stream waits there for what the stream of
    construction has queued (not in a capture, before which that work has to be done)."""

    def __init__(self, grads: Sequence[torch.Tensor], params: torch.Tensor, momentum: torch.Tensor,
                 matrices: Sequence[Tuple[int, int, int]], lr: float, mu: float = 0.95, weight_decay: float = 0.0,
                 nesterov: bool = True, steps: int = 5, coefficients: Sequence = MUON_COEFFICIENTS, eps: float = 1e-7,
                 adjust: Optional[str] = "spectral", wire: Optional[torch.Tensor] = None, stream=None):
        n = params.numel()
        self._keep = (list(grads), params, momentum, wire)
        self._grads = L._ptr_array(grads, _F32, n, "grads")
        self._matrices = (daso_matrix * max(len(matrices), 1))()
        factors = {}
        for m, (start, rows, cols) in zip(self._matrices, matrices):
            if (rows, cols) not in factors:
                factors[rows, cols] = muon_scale(rows, cols, adjust) if rows > 0 and cols > 0 else 1.0
            m.start, m.rows, m.cols, m.scale = int(start), int(rows), int(cols), factors[rows, cols]
        self._coefficients = _coefficients(steps, coefficients)
        a = daso_muon_args()
        a.n, a.g, a.nmatrices = n, len(grads), len(matrices)
        a.grads, a.matrices = self._grads, self._matrices
        a.params = L._ptr(params, _F32, n, "params")
        a.momentum = L._ptr(momentum, _F32, n, "momentum")
        a.wire = L._ptr(wire, L._BF16, n, "wire")
        a.lr, a.mu, a.weight_decay, a.eps = float(lr), float(mu), float(weight_decay), float(eps)
        a.coefficients, a.steps = self._coefficients, int(steps)
        a.flags = DASO_MUON_NESTEROV if nesterov else 0
        with _on(stream):
            self._workspace = _workspace("daso_muon_workspace", a)
        self.args = a
        self._byref = ctypes.byref(a)
        self._device = torch.cuda.current_device()
        self._made_on = L._stream_handle(stream).value
        self._streams = {self._made_on}  # on which the workspace is in order
        self._fn = _load().daso_muon_step

    def __call__(self, stream=None) -> None:
        if torch.cuda.current_device() != self._device:
            raise ValueError(f"prepared on cuda:{self._device}, called with cuda:{torch.cuda.current_device()} "
                             "current")
        handle = L._stream_handle(stream)
        if handle.value not in self._streams and self._workspace is not None:
            self._bring_workspace(torch.cuda.current_stream() if stream is None else stream)
        L._check(self._fn(self._byref, handle), "daso_muon_step")

    def _bring_workspace(self, to: torch.cuda.Stream) -> None:
        """The workspace is of the stream of construction: memory that the work queued there may still use, and that
        goes back to it when the object does.  `to` waits for the one, and the allocator for `to` before the other."""
        with _on(to):
            capturing = torch.cuda.is_current_stream_capturing()
        self._workspace.record_stream(to)
        if capturing:
            return
        to.wait_stream(torch.cuda.ExternalStream(self._made_on) if self._made_on else torch.cuda.default_stream())
        self._streams.add(to.cuda_stream or None)


def muon_step(grads, params, momentum, matrices, lr, mu=0.95, weight_decay=0.0, nesterov=True, steps=5,
              coefficients=MUON_COEFFICIENTS, eps=1e-7, adjust="spectral", wire=None, stream=None) -> None:
    """One local step with an orthogonalised update for the matrices of flat buffers (see
    include/daso_train.h), in place on params and momentum; writes wire when given."""
    MuonStep(grads, params, momentum, matrices, lr, mu, weight_decay, nesterov, steps, coefficients, eps, adjust, wire,
             stream)(stream)
