"""Python binding of the operators of the workers' models: argument marshalling only.

Layer norm, dropout from a counter-based generator, the join between two branches of a transformer block (bias, dropout,
residual add and layer norm in one pass) and the softmax cross-entropy, each with its gradient: what the forward and
backward pass that fills the rows of `Compams.compams_step`'s g needs around its matrix products.  With products of their own:
a gated feed-forward block, the gradients behind its projections, and the cross-entropy of an output layer whose logits are
never stored.  And the norm of every worker's gradient, cut to a largest one.  Same names as the C ABI (include/compams.h,
where every formula stands).

Activations are matrices (2-D tensors, rows contiguous, any distance between them) of n * rows rows: n workers, one
after another.  Weights are float32 vectors, such as views of theta; their gradients are n x cols float32 tensors whose
rows may be any distance apart, such as `g[:, first:first + cols]`, which puts them where the step reads them.

Every output may be given by name, and is then written in place and returned; what is not given is allocated.  Nothing
is recorded for autograd.  Work is enqueued on the current stream of the tensors' device.
"""
import ctypes
import functools
import struct
from typing import Optional

import torch

from .binding import _check, _on_stream, lib

F32, F16, BF16, I32, I64 = 0, 1, 2, 3, 4
_TYPE = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
_TARGET_TYPE = {torch.int32: I32, torch.int64: I64}


class compams_drop(ctypes.Structure):
    _fields_ = [("p", ctypes.c_double), ("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64),
                ("step", ctypes.c_void_p)]


class compams_norm(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("type", ctypes.c_int32),
                ("stream_type", ctypes.c_int32), ("eps", ctypes.c_float), ("drop", compams_drop),
                ("gamma", ctypes.c_void_p), ("beta", ctypes.c_void_p), ("bias", ctypes.c_void_p),
                ("x", ctypes.c_void_p), ("ld_x", ctypes.c_int64),
                ("residual", ctypes.c_void_p), ("ld_residual", ctypes.c_int64),
                ("h", ctypes.c_void_p), ("ld_h", ctypes.c_int64), ("y", ctypes.c_void_p), ("ld_y", ctypes.c_int64),
                ("mean", ctypes.c_void_p), ("rstd", ctypes.c_void_p),
                ("dy", ctypes.c_void_p), ("ld_dy", ctypes.c_int64), ("dh", ctypes.c_void_p), ("ld_dh", ctypes.c_int64),
                ("dx", ctypes.c_void_p), ("ld_dx", ctypes.c_int64),
                ("dresidual", ctypes.c_void_p), ("ld_dresidual", ctypes.c_int64),
                ("dgamma", ctypes.c_void_p), ("ld_dgamma", ctypes.c_int64),
                ("dbeta", ctypes.c_void_p), ("ld_dbeta", ctypes.c_int64),
                ("dbias", ctypes.c_void_p), ("ld_dbias", ctypes.c_int64), ("accumulate", ctypes.c_int32),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class compams_loss(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("rows", ctypes.c_int64), ("vocab", ctypes.c_int64), ("type", ctypes.c_int32),
                ("target_type", ctypes.c_int32), ("logits", ctypes.c_void_p), ("ld_logits", ctypes.c_int64),
                ("targets", ctypes.c_void_p), ("ignore_index", ctypes.c_int64), ("grad_scale", ctypes.c_float),
                ("mean_loss", ctypes.c_void_p), ("losses", ctypes.c_void_p),
                ("dlogits", ctypes.c_void_p), ("ld_dlogits", ctypes.c_int64),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class compams_gated(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("hidden", ctypes.c_int64),
                ("type", ctypes.c_int32), ("activation", ctypes.c_int32),
                ("x", ctypes.c_void_p), ("ld_x", ctypes.c_int64),
                ("gate_weight", ctypes.c_void_p), ("ld_gate_weight", ctypes.c_int64),
                ("up_weight", ctypes.c_void_p), ("ld_up_weight", ctypes.c_int64),
                ("gate_bias", ctypes.c_void_p), ("up_bias", ctypes.c_void_p),
                ("m", ctypes.c_void_p), ("ld_m", ctypes.c_int64), ("gate", ctypes.c_void_p), ("ld_gate", ctypes.c_int64),
                ("up", ctypes.c_void_p), ("ld_up", ctypes.c_int64), ("dm", ctypes.c_void_p), ("ld_dm", ctypes.c_int64),
                ("dgate", ctypes.c_void_p), ("ld_dgate", ctypes.c_int64), ("dup", ctypes.c_void_p), ("ld_dup", ctypes.c_int64),
                ("dgate_bias", ctypes.c_void_p), ("ld_dgate_bias", ctypes.c_int64),
                ("dup_bias", ctypes.c_void_p), ("ld_dup_bias", ctypes.c_int64), ("accumulate", ctypes.c_int32),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class compams_projections(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("hidden", ctypes.c_int64),
                ("type", ctypes.c_int32), ("dgate", ctypes.c_void_p), ("ld_dgate", ctypes.c_int64),
                ("dup", ctypes.c_void_p), ("ld_dup", ctypes.c_int64), ("x", ctypes.c_void_p), ("ld_x", ctypes.c_int64),
                ("gate_weight", ctypes.c_void_p), ("ld_gate_weight", ctypes.c_int64),
                ("up_weight", ctypes.c_void_p), ("ld_up_weight", ctypes.c_int64),
                ("dx", ctypes.c_void_p), ("ld_dx", ctypes.c_int64),
                ("dgate_weight", ctypes.c_void_p), ("ld_dgate_weight", ctypes.c_int64), ("stride_dgate_weight", ctypes.c_int64),
                ("dup_weight", ctypes.c_void_p), ("ld_dup_weight", ctypes.c_int64), ("stride_dup_weight", ctypes.c_int64),
                ("accumulate", ctypes.c_int32), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class compams_linear_loss(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("vocab", ctypes.c_int64),
                ("type", ctypes.c_int32), ("target_type", ctypes.c_int32), ("x", ctypes.c_void_p), ("ld_x", ctypes.c_int64),
                ("weight", ctypes.c_void_p), ("ld_weight", ctypes.c_int64), ("targets", ctypes.c_void_p),
                ("ignore_index", ctypes.c_int64), ("grad_scale", ctypes.c_float),
                ("mean_loss", ctypes.c_void_p), ("losses", ctypes.c_void_p), ("dx", ctypes.c_void_p), ("ld_dx", ctypes.c_int64),
                ("dweight", ctypes.c_void_p), ("ld_dweight", ctypes.c_int64), ("stride_dweight", ctypes.c_int64),
                ("accumulate", ctypes.c_int32), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class compams_clip_tensor(ctypes.Structure):
    _fields_ = [("from", ctypes.c_void_p), ("ld_from", ctypes.c_int64), ("to", ctypes.c_void_p), ("ld_to", ctypes.c_int64),
                ("count", ctypes.c_int64), ("from_type", ctypes.c_int32), ("to_type", ctypes.c_int32)]


class compams_clip(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("tensors", ctypes.c_int32), ("tensor", ctypes.c_void_p),
                ("max_norm", ctypes.c_float), ("scale", ctypes.c_float),
                ("norms", ctypes.c_void_p), ("factors", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


# The calls below lay the structures out with one pack each: a ctypes structure takes 50 ns for every field, and the
# smallest calls are as long as their marshalling.  (The C compiler's own padding; a null pointer is 0.)
_DROP = struct.Struct("@dQQP")
_NORM = struct.Struct("@iqqiif dQQP PPP PqPqPqPq PP PqPqPqPq PqPqPqi PN")
_LOSS = struct.Struct("@iqqii Pq Pqf PP Pq PN")
_GATED = struct.Struct("@iqqqii PqPqPq PP PqPqPq Pq PqPq PqPq i PN")
_PROJECTIONS = struct.Struct("@iqqqi PqPq Pq PqPq Pq PqqPqq i PN")
_LINEAR_LOSS = struct.Struct("@iqqqii PqPq Pqf PP Pq Pqq i PN")
_CLIP_TENSOR = struct.Struct("@PqPqqii")
_CLIP = struct.Struct("@iiPffPPPN")
ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2, "relu": 3, "sigmoid": 4}
_NO_DROP = (0.0, 0, 0, 0)
_LOW64 = (1 << 64) - 1


def _type(dtype: torch.dtype, what: str) -> int:
    t = _TYPE.get(dtype)
    if t is None:
        raise ValueError(f"{what} must be float32, float16 or bfloat16, got {dtype}")
    return t


def _matrix(t: Optional[torch.Tensor], what: str, shape, dtype: torch.dtype, device: torch.device):
    """(pointer, row stride) of a matrix that has to have this shape, type and device; (0, 0) for None."""
    if t is None:
        return 0, 0
    if t.dtype is dtype and t.shape == shape and t.device == device:
        apart, beside = t.stride()
        total, cols = shape
        if beside == 1 or cols == 1:
            return t.data_ptr(), apart if total > 1 else cols
        raise ValueError(f"the entries of a row of {what} must be contiguous, got strides {t.stride()}")
    raise ValueError(f"{what} must be {dtype} {tuple(shape)} on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")


def _vector(t: Optional[torch.Tensor], what: str, shape, device: torch.device, dtype=torch.float32):
    """Pointer of a contiguous vector of this shape; 0 for None."""
    if t is None:
        return 0
    if t.dtype is dtype and t.shape == shape and t.device == device and t.is_contiguous():
        return t.data_ptr()
    raise ValueError(f"{what} must be contiguous {dtype} {shape} on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")


def _shape(x: torch.Tensor, what: str, n: int = 1):
    """(total rows, rows of a worker, columns) of a matrix of n workers' rows."""
    if x.dim() != 2:
        raise ValueError(f"{what} must be a matrix, got shape {tuple(x.shape)}")
    total, cols = x.shape
    if n < 1 or total % n:
        raise ValueError(f"{what} has {total} rows: not the same number for each of {n} workers")
    return total, total // n, cols


def _drop(p: float, seed: int, offset: int, step: Optional[torch.Tensor], device: torch.device):
    return p, seed & _LOW64, offset & _LOW64, _vector(step, "step", (1,), device, torch.int64)


def _workspace(workspace: Optional[torch.Tensor], need: int, device: torch.device):
    """(tensor to keep, pointer, bytes) of the caller's workspace, or of one that is allocated."""
    if workspace is None:
        if need == 0:
            return None, 0, 0
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    elif workspace.device != device or not workspace.is_contiguous():
        raise ValueError(f"workspace must be contiguous on {device}")
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def compams_dropout(x: torch.Tensor, p: float, seed: int, offset: int = 0, *, residual: Optional[torch.Tensor] = None,
                    y: Optional[torch.Tensor] = None, dtype: Optional[torch.dtype] = None,
                    step: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dropout(x), or residual + dropout(x).  The backward pass is the same call on the gradient, without a residual.
    dtype: y's type where it is not given and there is no residual (default x's).  step: int64[1] that is added to
    offset when the kernel runs."""
    total, rows, cols = _shape(x, "x")
    dev = x.device
    if y is None:
        y = torch.empty((total, cols), dtype=dtype or (x if residual is None else residual).dtype, device=dev)
    px, lx = _matrix(x, "x", x.shape, x.dtype, dev)
    pr, lr = _matrix(residual, "residual", x.shape, y.dtype, dev)
    py, ly = _matrix(y, "y", x.shape, y.dtype, dev)
    _check(_on_stream(dev, lib().compams_dropout, 1, rows, cols, _type(x.dtype, "x"), _type(y.dtype, "y"), px, lx, pr, lr,
                      py, ly, _DROP.pack(*_drop(p, seed, offset, step, dev))), "compams_dropout")
    return y


def _forward(call, what, x, residual, h, y, gamma, beta, bias, mean, rstd, eps, drop, shape, dev):
    total, cols = shape
    stream_dtype, dtype = h.dtype, y.dtype
    px, lx = _matrix(x, "x", shape, dtype, dev)
    pr, lr = _matrix(residual, "residual", shape, stream_dtype, dev)
    ph, lh = _matrix(h, "h" if x is not None else "x", shape, stream_dtype, dev)
    py, ly = _matrix(y, "y", shape, dtype, dev)
    of_cols, of_rows = (cols,), (total,)
    a = _NORM.pack(1, total, cols, _type(dtype, "y"), _type(stream_dtype, "the stream"), eps, *drop,
                   _vector(gamma, "gamma", of_cols, dev), _vector(beta, "beta", of_cols, dev),
                   _vector(bias, "bias", of_cols, dev), px, lx, pr, lr, ph, lh, py, ly,
                   _vector(mean, "mean", of_rows, dev), _vector(rstd, "rstd", of_rows, dev),
                   0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0)
    _check(_on_stream(dev, call, a), what)


def compams_layer_norm_forward(x: torch.Tensor, gamma: Optional[torch.Tensor], beta: Optional[torch.Tensor],
                               eps: float = 1e-5, *, y: Optional[torch.Tensor] = None,
                               mean: Optional[torch.Tensor] = None, rstd: Optional[torch.Tensor] = None,
                               dtype: Optional[torch.dtype] = None):
    """(y, mean, rstd).  dtype: y's type where it is not given (default x's); x may be float32 beside a narrower y."""
    total, _, cols = _shape(x, "x")
    dev = x.device
    if y is None:
        y = torch.empty((total, cols), dtype=dtype or x.dtype, device=dev)
    if mean is None:
        mean = torch.empty(total, dtype=torch.float32, device=dev)
    if rstd is None:
        rstd = torch.empty(total, dtype=torch.float32, device=dev)
    _forward(lib().compams_layer_norm_forward, "compams_layer_norm_forward", None, None, x, y, gamma, beta, None, mean, rstd,
             eps, _NO_DROP, x.shape, dev)
    return y, mean, rstd


def compams_dropout_add_norm_forward(x: torch.Tensor, residual: Optional[torch.Tensor], gamma: Optional[torch.Tensor],
                                     beta: Optional[torch.Tensor], p: float, seed: int, offset: int = 0,
                                     eps: float = 1e-5, *, bias: Optional[torch.Tensor] = None,
                                     h: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None,
                                     mean: Optional[torch.Tensor] = None, rstd: Optional[torch.Tensor] = None,
                                     step: Optional[torch.Tensor] = None):
    """(h, y, mean, rstd) with h = residual + dropout(x + bias) and y the layer norm of h.  x and y have one type, residual
    and h another, which is the same or float32 (without either, x's)."""
    total, _, cols = _shape(x, "x")
    dev = x.device
    if h is None:
        h = torch.empty((total, cols), dtype=(x if residual is None else residual).dtype, device=dev)
    if y is None:
        y = torch.empty((total, cols), dtype=x.dtype, device=dev)
    if mean is None:
        mean = torch.empty(total, dtype=torch.float32, device=dev)
    if rstd is None:
        rstd = torch.empty(total, dtype=torch.float32, device=dev)
    _forward(lib().compams_dropout_add_norm_forward, "compams_dropout_add_norm_forward", x, residual, h, y, gamma, beta, bias,
             mean, rstd, eps, _drop(p, seed, offset, step, dev), x.shape, dev)
    return h, y, mean, rstd


def _backward(call, what, dy, dh, h, mean, rstd, gamma, dx, dresidual, dgamma, dbeta, dbias, drop, n, rows, accumulate,
              workspace, shape, dev):
    total, cols = shape
    dtype, stream_dtype, of_weights = dy.dtype, h.dtype, (n, cols)
    py, ly = _matrix(dy, "dy", shape, dtype, dev)
    pg, lg = _matrix(dh, "dh", shape, stream_dtype, dev)
    ph, lh = _matrix(h, "h", shape, stream_dtype, dev)
    px, lx = _matrix(dx, "dx", shape, dtype, dev)
    pr, lr = _matrix(dresidual, "the stream's gradient", shape, stream_dtype, dev)
    p0, l0 = _matrix(dgamma, "dgamma", of_weights, torch.float32, dev)
    p1, l1 = _matrix(dbeta, "dbeta", of_weights, torch.float32, dev)
    p2, l2 = _matrix(dbias, "dbias", of_weights, torch.float32, dev)
    of_cols, of_rows = (cols,), (total,)
    a = (n, rows, cols, _type(dtype, "dy"), _type(stream_dtype, "h"), 0.0, *drop, _vector(gamma, "gamma", of_cols, dev),
         0, 0, 0, 0, 0, 0, ph, lh, 0, 0, _vector(mean, "mean", of_rows, dev), _vector(rstd, "rstd", of_rows, dev),
         py, ly, pg, lg, px, lx, pr, lr, p0, l0, p1, l1, p2, l2, 1 if accumulate else 0)
    need = lib().compams_norm_workspace_size(_NORM.pack(*a, 0, 0))
    workspace, at, size = _workspace(workspace, need, dev)
    _check(_on_stream(dev, call, _NORM.pack(*a, at, size)), what)


def compams_layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                                gamma: Optional[torch.Tensor], n: int = 1, *, dx: Optional[torch.Tensor] = None,
                                dgamma: Optional[torch.Tensor] = None, dbeta: Optional[torch.Tensor] = None,
                                accumulate: bool = False, workspace: Optional[torch.Tensor] = None):
    """(dx, dgamma, dbeta): the gradient of x, and of the weights for each of the n workers that the rows belong to.
    accumulate: dgamma and dbeta are added to what is there (they have to be given then)."""
    total, rows, cols = _shape(dy, "dy", n)
    dev = dy.device
    if dx is None:
        dx = torch.empty((total, cols), dtype=x.dtype, device=dev)
    dgamma, dbeta = _gradients(accumulate, n, cols, dev, dgamma, dbeta)
    _backward(lib().compams_layer_norm_backward, "compams_layer_norm_backward", dy, None, x, mean, rstd, gamma, None, dx,
              dgamma, dbeta, None, _NO_DROP, n, rows, accumulate, workspace, dy.shape, dev)
    return dx, dgamma, dbeta


def compams_dropout_add_norm_backward(dy: torch.Tensor, dh: Optional[torch.Tensor], h: torch.Tensor, mean: torch.Tensor,
                                      rstd: torch.Tensor, gamma: Optional[torch.Tensor], p: float, seed: int,
                                      offset: int = 0, n: int = 1, *, dx: Optional[torch.Tensor] = None,
                                      dresidual: Optional[torch.Tensor] = None, dgamma: Optional[torch.Tensor] = None,
                                      dbeta: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None,
                                      accumulate: bool = False, workspace: Optional[torch.Tensor] = None,
                                      step: Optional[torch.Tensor] = None):
    """(dx, dresidual, dgamma, dbeta, dbias) from the gradients of y and of h (dh: None where nothing else reads h).
    p, seed, offset and step are the forward call's."""
    total, rows, cols = _shape(dy, "dy", n)
    dev = dy.device
    if dx is None:
        dx = torch.empty((total, cols), dtype=dy.dtype, device=dev)
    if dresidual is None:
        dresidual = torch.empty((total, cols), dtype=h.dtype, device=dev)
    dgamma, dbeta, dbias = _gradients(accumulate, n, cols, dev, dgamma, dbeta, dbias)
    _backward(lib().compams_dropout_add_norm_backward, "compams_dropout_add_norm_backward", dy, dh, h, mean, rstd, gamma, dx,
              dresidual, dgamma, dbeta, dbias, _drop(p, seed, offset, step, dev), n, rows, accumulate, workspace, dy.shape, dev)
    return dx, dresidual, dgamma, dbeta, dbias


def _gradients(accumulate, n, cols, dev, *given):
    if accumulate and any(t is None for t in given):
        raise ValueError("accumulate needs the gradients that are added to")
    return [torch.empty((n, cols), dtype=torch.float32, device=dev) if t is None else t for t in given]


def compams_cross_entropy(logits: torch.Tensor, targets: torch.Tensor, n: int = 1, ignore_index: int = -100,
                          grad_scale: float = 1.0, *, mean_loss: Optional[torch.Tensor] = None,
                          losses: Optional[torch.Tensor] = None, dlogits: Optional[torch.Tensor] = None,
                          gradient: bool = True, workspace: Optional[torch.Tensor] = None):
    """(mean_loss, losses, dlogits): every worker's mean loss, every row's, and grad_scale times the gradient of the
    workers' mean losses (None with gradient=False; may be written over the logits)."""
    total, rows, vocab = _shape(logits, "logits", n)
    dev = logits.device
    if mean_loss is None:
        mean_loss = torch.empty(n, dtype=torch.float32, device=dev)
    if losses is None:
        losses = torch.empty(total, dtype=torch.float32, device=dev)
    if not gradient:
        if dlogits is not None:
            raise ValueError("dlogits is given, but no gradient asked for")
    elif dlogits is None:
        dlogits = torch.empty((total, vocab), dtype=logits.dtype, device=dev)
    target_type = _TARGET_TYPE.get(targets.dtype)
    if target_type is None:
        raise ValueError(f"targets must be int32 or int64, got {targets.dtype}")
    pl, ll = _matrix(logits, "logits", logits.shape, logits.dtype, dev)
    pd, ld = _matrix(dlogits, "dlogits", logits.shape, logits.dtype, dev)
    a = (n, rows, vocab, _type(logits.dtype, "logits"), target_type, pl, ll,
         _vector(targets, "targets", (total,), dev, targets.dtype), ignore_index, grad_scale,
         _vector(mean_loss, "mean_loss", (n,), dev), _vector(losses, "losses", (total,), dev), pd, ld)
    need = lib().compams_loss_workspace_size(_LOSS.pack(*a, 0, 0))
    workspace, at, size = _workspace(workspace, need, dev)
    _check(_on_stream(dev, lib().compams_cross_entropy, _LOSS.pack(*a, at, size)), "compams_cross_entropy")
    return mean_loss, losses, dlogits


def _activation(name: str) -> int:
    a = ACTIVATIONS.get(name)
    if a is None:
        raise ValueError(f"unknown activation {name!r}: one of {', '.join(ACTIVATIONS)}")
    return a


def _weight_gradient(t: Optional[torch.Tensor], what: str, shape, device: torch.device):
    """(pointer, row stride, worker stride) of a weight's gradients, a matrix for every worker; (0, 0, 0) for None."""
    if t is None:
        return 0, 0, 0
    if t.dtype is torch.float32 and t.shape == shape and t.device == device:
        n, outputs, cols = shape
        worker, row, beside = t.stride()
        if beside == 1 or cols == 1:
            return t.data_ptr(), row if outputs > 1 else cols, worker if n > 1 else 0
        raise ValueError(f"the entries of a row of {what} must be contiguous, got strides {t.stride()}")
    raise ValueError(f"{what} must be {torch.float32} {tuple(shape)} on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")


def _room(size, pack, a, workspace, device):
    """The structure with the workspace that its call asks for, and what has to live until the call is made."""
    need = size(pack(*a, 0, 0))
    workspace, at, given = _workspace(workspace, need, device)
    return pack(*a, at, given), workspace


def compams_gated_forward(x: torch.Tensor, gate_weight: torch.Tensor, up_weight: torch.Tensor, activation: str = "silu", *,
                          gate_bias: Optional[torch.Tensor] = None, up_bias: Optional[torch.Tensor] = None,
                          m: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                          up: Optional[torch.Tensor] = None, keep: bool = True, workspace: Optional[torch.Tensor] = None):
    """(m, gate, up) with gate = x gate_weight' + gate_bias, up = x up_weight' + up_bias and m = act(gate) up, formed before
    the two are rounded.  keep=False: m alone (gate and up are None), for answers without a backward pass."""
    total, _, cols = _shape(x, "x")
    dev, dtype = x.device, x.dtype
    hidden = _shape(gate_weight, "gate_weight")[0]
    shape, of_weight, of_bias = (total, hidden), (hidden, cols), (hidden,)
    if m is None:
        m = torch.empty(shape, dtype=dtype, device=dev)
    if not keep:
        if gate is not None or up is not None:
            raise ValueError("gate or up is given, but not to be kept")
    else:
        if gate is None:
            gate = torch.empty(shape, dtype=dtype, device=dev)
        if up is None:
            up = torch.empty(shape, dtype=dtype, device=dev)
    a = (1, total, cols, hidden, _type(dtype, "x"), _activation(activation), *_matrix(x, "x", x.shape, dtype, dev),
         *_matrix(gate_weight, "gate_weight", of_weight, dtype, dev), *_matrix(up_weight, "up_weight", of_weight, dtype, dev),
         _vector(gate_bias, "gate_bias", of_bias, dev), _vector(up_bias, "up_bias", of_bias, dev),
         *_matrix(m, "m", shape, dtype, dev), *_matrix(gate, "gate", shape, dtype, dev), *_matrix(up, "up", shape, dtype, dev),
         0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0)
    a, workspace = _room(lib().compams_gated_forward_workspace_size, _GATED.pack, a, workspace, dev)
    _check(_on_stream(dev, lib().compams_gated_forward, a), "compams_gated_forward")
    return m, gate, up


def compams_gated_backward(dm: torch.Tensor, gate: torch.Tensor, up: torch.Tensor, n: int = 1, activation: str = "silu", *,
                           dgate: Optional[torch.Tensor] = None, dup: Optional[torch.Tensor] = None,
                           dgate_bias: Optional[torch.Tensor] = None, dup_bias: Optional[torch.Tensor] = None,
                           bias: bool = True, accumulate: bool = False, workspace: Optional[torch.Tensor] = None):
    """(dgate, dup, dgate_bias, dup_bias): the gradients of the two projections (dgate and dup may be written over dm, gate or
    up) and of the two biases for each of the n workers (None with bias=False).  accumulate: the biases' gradients are added
    to what is there (they have to be given then)."""
    total, rows, hidden = _shape(dm, "dm", n)
    dev, dtype, shape, of_bias = dm.device, dm.dtype, dm.shape, (n, hidden)
    if dgate is None:
        dgate = torch.empty((total, hidden), dtype=dtype, device=dev)
    if dup is None:
        dup = torch.empty((total, hidden), dtype=dtype, device=dev)
    if bias:
        dgate_bias, dup_bias = _gradients(accumulate, n, hidden, dev, dgate_bias, dup_bias)
    elif dgate_bias is not None or dup_bias is not None:
        raise ValueError("a bias's gradient is given, but not asked for")
    a = (n, rows, 0, hidden, _type(dtype, "dm"), _activation(activation), 0, 0, 0, 0, 0, 0, 0, 0, 0, 0,
         *_matrix(gate, "gate", shape, dtype, dev), *_matrix(up, "up", shape, dtype, dev), *_matrix(dm, "dm", shape, dtype, dev),
         *_matrix(dgate, "dgate", shape, dtype, dev), *_matrix(dup, "dup", shape, dtype, dev),
         *_matrix(dgate_bias, "dgate_bias", of_bias, torch.float32, dev),
         *_matrix(dup_bias, "dup_bias", of_bias, torch.float32, dev), 1 if accumulate else 0)
    a, workspace = _room(lib().compams_gated_backward_workspace_size, _GATED.pack, a, workspace, dev)
    _check(_on_stream(dev, lib().compams_gated_backward, a), "compams_gated_backward")
    return dgate, dup, dgate_bias, dup_bias


def compams_projections_backward(dgate: torch.Tensor, dup: Optional[torch.Tensor], x: Optional[torch.Tensor],
                                 gate_weight: Optional[torch.Tensor], up_weight: Optional[torch.Tensor], n: int = 1, *,
                                 dx: Optional[torch.Tensor] = None, dgate_weight: Optional[torch.Tensor] = None,
                                 dup_weight: Optional[torch.Tensor] = None, accumulate: bool = False,
                                 workspace: Optional[torch.Tensor] = None):
    """(dx, dgate_weight, dup_weight): the gradient of what two projections read, and of their weights for each of the n
    workers.  One projection: dup and up_weight None (and dup_weight, which is None then too).  Without x no weight's gradient
    is formed, without gate_weight no dx.  accumulate: the weights' gradients are added to what is there (they have to be
    given then)."""
    total, rows, hidden = _shape(dgate, "dgate", n)
    dev, dtype, shape = dgate.device, dgate.dtype, dgate.shape
    if x is None and gate_weight is None:
        raise ValueError("neither x nor gate_weight is given: there is no gradient to form")
    cols = _shape(x, "x")[2] if x is not None else _shape(gate_weight, "gate_weight")[2]
    if dup is None and (up_weight is not None or dup_weight is not None):
        raise ValueError("up_weight or dup_weight is given, but no dup")
    if gate_weight is None:
        if dx is not None or up_weight is not None:
            raise ValueError("dx or up_weight is given, but no gate_weight")
    elif dx is None:
        dx = torch.empty((total, cols), dtype=dtype, device=dev)
    if x is None:
        if dgate_weight is not None or dup_weight is not None:
            raise ValueError("a weight's gradient is given, but no x")
    elif accumulate and (dgate_weight is None or (dup is not None and dup_weight is None)):
        raise ValueError("accumulate needs the gradients that are added to")
    else:
        if dgate_weight is None:
            dgate_weight = torch.empty((n, hidden, cols), dtype=torch.float32, device=dev)
        if dup is not None and dup_weight is None:
            dup_weight = torch.empty((n, hidden, cols), dtype=torch.float32, device=dev)
    of_x, of_weight, of_gradient = (total, cols), (hidden, cols), (n, hidden, cols)
    a = (n, rows, cols, hidden, _type(dtype, "dgate"), *_matrix(dgate, "dgate", shape, dtype, dev),
         *_matrix(dup, "dup", shape, dtype, dev), *_matrix(x, "x", of_x, dtype, dev),
         *_matrix(gate_weight, "gate_weight", of_weight, dtype, dev), *_matrix(up_weight, "up_weight", of_weight, dtype, dev),
         *_matrix(dx, "dx", of_x, dtype, dev), *_weight_gradient(dgate_weight, "dgate_weight", of_gradient, dev),
         *_weight_gradient(dup_weight, "dup_weight", of_gradient, dev), 1 if accumulate else 0)
    a, workspace = _room(lib().compams_projections_workspace_size, _PROJECTIONS.pack, a, workspace, dev)
    _check(_on_stream(dev, lib().compams_projections_backward, a), "compams_projections_backward")
    return dx, dgate_weight, dup_weight


def compams_linear_cross_entropy(x: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, n: int = 1,
                                 ignore_index: int = -100, grad_scale: float = 1.0, *,
                                 mean_loss: Optional[torch.Tensor] = None, losses: Optional[torch.Tensor] = None,
                                 dx: Optional[torch.Tensor] = None, dweight: Optional[torch.Tensor] = None,
                                 gradient: bool = True, accumulate: bool = False, workspace: Optional[torch.Tensor] = None):
    """(mean_loss, losses, dx, dweight) of the logits x weight', which are never stored: every worker's mean loss, every
    row's, and grad_scale times the gradients of the workers' mean losses (None with gradient=False), of the weight for
    each of the n workers.  accumulate: dweight is added to what is there (it has to be given then)."""
    total, rows, cols = _shape(x, "x", n)
    dev, dtype = x.device, x.dtype
    vocab = _shape(weight, "weight")[0]
    if mean_loss is None:
        mean_loss = torch.empty(n, dtype=torch.float32, device=dev)
    if losses is None:
        losses = torch.empty(total, dtype=torch.float32, device=dev)
    if not gradient:
        if dx is not None or dweight is not None:
            raise ValueError("dx or dweight is given, but no gradient asked for")
    else:
        if accumulate and dweight is None:
            raise ValueError("accumulate needs the gradients that are added to")
        if dx is None:
            dx = torch.empty((total, cols), dtype=dtype, device=dev)
        if dweight is None:
            dweight = torch.empty((n, vocab, cols), dtype=torch.float32, device=dev)
    target_type = _TARGET_TYPE.get(targets.dtype)
    if target_type is None:
        raise ValueError(f"targets must be int32 or int64, got {targets.dtype}")
    a = (n, rows, cols, vocab, _type(dtype, "x"), target_type, *_matrix(x, "x", x.shape, dtype, dev),
         *_matrix(weight, "weight", (vocab, cols), dtype, dev), _vector(targets, "targets", (total,), dev, targets.dtype),
         ignore_index, grad_scale, _vector(mean_loss, "mean_loss", (n,), dev), _vector(losses, "losses", (total,), dev),
         *_matrix(dx, "dx", x.shape, dtype, dev), *_weight_gradient(dweight, "dweight", (n, vocab, cols), dev),
         1 if accumulate else 0)
    a, workspace = _room(lib().compams_linear_loss_workspace_size, _LINEAR_LOSS.pack, a, workspace, dev)
    _check(_on_stream(dev, lib().compams_linear_cross_entropy, a), "compams_linear_cross_entropy")
    return mean_loss, losses, dx, dweight


@functools.lru_cache(maxsize=64)
def _clip_table(count: int):
    return struct.Struct("@" + _CLIP_TENSOR.format[1:] * count)


def compams_clip_gradients(gradients, max_norm: float, n: int = 1, *, scale: float = 1.0, out=None,
                           norms: Optional[torch.Tensor] = None, factors: Optional[torch.Tensor] = None,
                           workspace: Optional[torch.Tensor] = None):
    """(out, norms, factors): scale times the norm of each worker's gradient, and factors[i] = scale min(1, max_norm /
    norms[i]) times it (0 and zeros where it is not finite: the worker takes no part).
    gradients: a matrix of n rows, or a list of them (a tensor's gradients of all workers each), in any mixture of types.
    out: the same shapes, each float32 or of its gradient's type, such as views of the step's g; None: in place.
    max_norm: math.inf cuts nothing.  scale: takes a loss's scale back.  (Both are fp32 numbers and rounded to one.)"""
    alone = isinstance(gradients, torch.Tensor)
    given = [gradients] if alone else list(gradients)
    to = given if out is None else [out] if isinstance(out, torch.Tensor) else list(out)
    if len(to) != len(given):
        raise ValueError(f"out has {len(to)} tensors for {len(given)} gradients")
    if not given:
        raise ValueError("no gradients are given")
    dev = given[0].device
    if norms is None:
        norms = torch.empty(n, dtype=torch.float32, device=dev)
    if factors is None:
        factors = torch.empty(n, dtype=torch.float32, device=dev)
    table, where = [], norms.get_device()
    for t, o in zip(given, to):    # (an answer of many tensors waits for this loop: a microsecond a tensor)
        shape, kind = t.shape, _TYPE.get(t.dtype)
        if len(shape) != 2 or shape[0] != n:
            raise ValueError(f"a gradient must be a matrix of {n} rows, got shape {tuple(shape)}")
        apart, beside = t.stride()
        count = shape[1]
        if kind is None or t.get_device() != where or (beside != 1 and count > 1):
            _matrix(t, "a gradient", shape, t.dtype, dev)
            _type(t.dtype, "a gradient")
        p = t.data_ptr()
        if o is t:
            table += (p, apart, p, apart, count, kind, kind)
            continue
        kind_to = _TYPE.get(o.dtype)
        apart_to, beside = o.stride() if o.dim() == 2 else (0, 0)
        if kind_to is None or o.shape != shape or o.get_device() != where or (beside != 1 and count > 1):
            _matrix(o, "out", shape, o.dtype, dev)
            _type(o.dtype, "out")
        table += (p, apart, o.data_ptr(), apart_to, count, kind, kind_to)
    table = _clip_table(len(given)).pack(*table)
    keep = ctypes.c_char_p(table)
    a = (n, len(given), ctypes.cast(keep, ctypes.c_void_p).value, max_norm, scale, _vector(norms, "norms", (n,), dev),
         _vector(factors, "factors", (n,), dev))
    a, workspace = _room(lib().compams_clip_workspace_size, _CLIP.pack, a, workspace, dev)
    _check(_on_stream(dev, lib().compams_clip_gradients, a), "compams_clip_gradients")
    return gradients if out is None else out, norms, factors
