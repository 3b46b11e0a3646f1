"""Python binding of the operators of the workers' models: argument marshalling only.

Layer norm, dropout from a counter-based generator, the join between two branches of a transformer block (bias, dropout,
residual add and layer norm in one pass) and the softmax cross-entropy, each with its gradient: what the forward and
backward pass that fills the rows of `Compams.compams_step`'s g needs around its matrix products.  Same names as the C ABI
(include/compams.h, where every formula stands).

Activations are matrices (2-D tensors, rows contiguous, any distance between them) of n * rows rows: n workers, one
after another.  Weights are float32 vectors, such as views of theta; their gradients are n x cols float32 tensors whose
rows may be any distance apart, such as `g[:, first:first + cols]`, which puts them where the step reads them.

Every output may be given by name, and is then written in place and returned; what is not given is allocated.  Nothing
is recorded for autograd.  Work is enqueued on the current stream of the tensors' device.
"""
import ctypes
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


# The calls below lay the structures out with one pack each: a ctypes structure takes 50 ns for every field, and the
# smallest calls are as long as their marshalling.  (The C compiler's own padding; a null pointer is 0.)
_DROP = struct.Struct("@dQQP")
_NORM = struct.Struct("@iqqiif dQQP PPP PqPqPqPq PP PqPqPqPq PqPqPqi PN")
_LOSS = struct.Struct("@iqqii Pq Pqf PP Pq PN")
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
