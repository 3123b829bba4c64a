"""Operators on torch tensors in device memory (binding of include/ccdpp_ops.h).

Softmax cross entropy of rows (users' factors, hidden states) against a whole
table (items' factors, a vocabulary) without keeping the logits, its gradients,
and the global norm of gradient tensors with their clipping.  Every computation
happens in libccdpp.so; torch gives device memory and the current stream, on
which the work is enqueued.  Nothing waits for the device.  A tensor that was
made on another stream must have been waited for by the caller's, as with any
torch operator.  Refused arguments raise ValueError or TypeError here, or
CCDPPError (EINVAL) where the library finds them.
"""
from __future__ import annotations

import ctypes
import functools

import torch

from . import ccdpp as _c

F32, BF16, F16 = range(3)
_DTYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
LOSS, GRAD, TRAIN = range(3)


class Softmax(ctypes.Structure):
    """ccdpp_softmax_t."""
    _fields_ = [("t", ctypes.c_int64), ("v", ctypes.c_int64), ("d", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("x", ctypes.c_void_p), ("ldx", ctypes.c_int64), ("table", ctypes.c_void_p), ("ldt", ctypes.c_int64),
                ("target", ctypes.c_void_p), ("target_bits", ctypes.c_int32), ("scale", ctypes.c_float),
                ("offset", ctypes.c_void_p)]


@functools.lru_cache(maxsize=None)
def _lib():
    L = _c.lib()
    P, i64, i32, f32, S = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float, ctypes.POINTER(Softmax)
    sig = {
        "ccdpp_softmax_workspace": [S, i32, ctypes.POINTER(i64)],
        "ccdpp_softmax_loss": [S, P, P, P, i64, P],
        "ccdpp_softmax_loss_grad": [S, P, P, P, i64, P, i64, P, i64, P],
        "ccdpp_softmax_loss_train": [S, P, P, P, P, i64, P, i64, P, i64, P],
        "ccdpp_grad_norm_workspace": [ctypes.POINTER(i64)],
        "ccdpp_grad_norm": [i32, P, P, P, P, P, i64, P],
        "ccdpp_clip_grads": [i32, P, P, P, P, f32, f32, P, P, i64, P],
    }
    for name, args in sig.items():
        f = getattr(L, name)
        f.argtypes, f.restype = args, ctypes.c_int
    L.ccdpp_ops_last_error.argtypes, L.ccdpp_ops_last_error.restype = [], ctypes.c_char_p
    return L


def _check(rc):
    if rc < 0:
        raise _c.CCDPPError(rc, _lib().ccdpp_ops_last_error().decode())


class _On:
    """Makes the tensors' device current while a call runs, where it is not."""

    def __init__(self, device):
        self._guard = None if device.index == torch.cuda.current_device() else torch.cuda.device(device)

    def __enter__(self):
        if self._guard:
            self._guard.__enter__()

    def __exit__(self, *exc):
        if self._guard:
            self._guard.__exit__(*exc)


def _matrix(a, name):
    if not isinstance(a, torch.Tensor) or a.dim() != 2:
        raise TypeError(f"{name} must be a matrix (a two-dimensional tensor)")
    if not a.is_cuda:
        raise ValueError(f"{name} must be in device memory")
    if a.dtype not in _DTYPES:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, not {a.dtype}")
    rows, d = a.shape
    if d > 1 and a.stride(1) != 1:
        raise ValueError(f"{name}'s rows must be contiguous")
    return a.stride(0) if rows > 1 else max(d, 1)


def _vector(a, name, n, dtypes, device):
    if not isinstance(a, torch.Tensor) or a.dtype not in dtypes:
        raise TypeError(f"{name} must be a tensor of {' or '.join(str(t)[6:] for t in dtypes)}")
    if a.shape != (n,) or not a.is_contiguous():
        raise ValueError(f"{name} must be contiguous, with {n} values")
    if a.device != device:
        raise ValueError(f"{name} must be on {device}")
    return a.data_ptr()


def _problem(x, table, target, scale, offset):
    ldx, ldt = _matrix(x, "x"), _matrix(table, "table")
    if x.dtype != table.dtype or x.device != table.device:
        raise ValueError("x and table must have the same type and device")
    if x.shape[1] != table.shape[1]:
        raise ValueError(f"x has {x.shape[1]} columns and table {table.shape[1]}")
    y = _vector(target, "target", x.shape[0], (torch.int64, torch.int32), x.device)
    o = None if offset is None else _vector(offset, "offset", table.shape[0], (torch.float32,), x.device)
    return Softmax(x.shape[0], table.shape[0], x.shape[1], _DTYPES[x.dtype], x.data_ptr(), ldx, table.data_ptr(), ldt,
                   y, 64 if target.dtype == torch.int64 else 32, scale, o)


def _workspace(p, call, device):
    n = ctypes.c_int64()
    _check(_lib().ccdpp_softmax_workspace(ctypes.byref(p), call, ctypes.byref(n)))
    return torch.empty(n.value, dtype=torch.uint8, device=device)


def _stream(device):
    return torch.cuda.current_stream(device).cuda_stream


def _out(a, like, name):
    if a is None:
        return torch.empty(like.shape, dtype=like.dtype, device=like.device)
    if _matrix(a, name) < 0 or a.shape != like.shape or a.dtype != like.dtype or a.device != like.device:
        raise ValueError(f"{name} must have the shape, type and device of what it is the gradient of")
    return a


def _gradient_buffers(x, table, dx, dtable, need):
    """(dx, its pointer, its row stride, dtable, ...) for the gradients that are asked for."""
    for n in need:
        if n not in ("x", "table"):
            raise ValueError(f"need is made of 'x' and 'table', not {n!r}")
    got = []
    for name, like, a in (("x", x, dx), ("table", table, dtable)):
        a = _out(a, like, "d" + name) if name in need else None
        got += [a, None if a is None else a.data_ptr(), 0 if a is None else _matrix(a, "d" + name)]
    return got


def softmax_loss(x, table, target, *, scale=1.0, offset=None):
    """(loss, lse), float32 per row: lse[i] = log sum_v exp(scale x_i.table_v + offset_v), loss[i] = lse[i] - the
    target's logit.  x: t x d, table: v x d (float32, bfloat16 or float16; rows may lie apart), target: int32 or int64.
    A negative target marks an ignored row (loss 0); one past the table makes the row's loss NaN.  offset: float32 per
    item or None; -inf (or anything below -1e38) excludes an item, and a target that is excluded has loss +inf."""
    p = _problem(x, table, target, scale, offset)
    with _On(x.device):
        loss = torch.empty(p.t, dtype=torch.float32, device=x.device)
        lse = torch.empty_like(loss)
        ws = _workspace(p, LOSS, x.device)
        _check(_lib().ccdpp_softmax_loss(ctypes.byref(p), loss.data_ptr(), lse.data_ptr(), ws.data_ptr(), ws.numel(),
                                         _stream(x.device)))
    return loss, lse


def softmax_loss_grad(x, table, target, lse, *, grad=None, scale=1.0, offset=None, dx=None, dtable=None, need=("x", "table")):
    """(dx, dtable): gradients of sum_i grad[i] loss[i], from the lse of softmax_loss.  grad: float32 per row, or None
    for ones.  dx and dtable may be given to write to.  A gradient that is not in `need` is not computed (None).
    Ignored rows, rows whose target is excluded and excluded items take no part, whatever they hold."""
    p = _problem(x, table, target, scale, offset)
    l = _vector(lse, "lse", p.t, (torch.float32,), x.device)
    g = None if grad is None else _vector(grad, "grad", p.t, (torch.float32,), x.device)
    with _On(x.device):
        dx, pdx, lddx, dtable, pde, ldde = _gradient_buffers(x, table, dx, dtable, need)
        ws = _workspace(p, GRAD, x.device)
        _check(_lib().ccdpp_softmax_loss_grad(ctypes.byref(p), l, g, pdx, lddx, pde, ldde, ws.data_ptr(), ws.numel(),
                                              _stream(x.device)))
    return dx, dtable


def softmax_loss_train(x, table, target, *, grad=None, scale=1.0, offset=None, dx=None, dtable=None, need=("x", "table")):
    """(loss, lse, dx, dtable): softmax_loss and softmax_loss_grad in one call, for rows whose weights `grad` are known
    beforehand (1 / the number of rows that count, for a mean)."""
    p = _problem(x, table, target, scale, offset)
    g = None if grad is None else _vector(grad, "grad", p.t, (torch.float32,), x.device)
    with _On(x.device):
        loss = torch.empty(p.t, dtype=torch.float32, device=x.device)
        lse = torch.empty_like(loss)
        dx, pdx, lddx, dtable, pde, ldde = _gradient_buffers(x, table, dx, dtable, need)
        ws = _workspace(p, TRAIN, x.device)
        _check(_lib().ccdpp_softmax_loss_train(ctypes.byref(p), loss.data_ptr(), lse.data_ptr(), g, pdx, lddx, pde, ldde,
                                               ws.data_ptr(), ws.numel(), _stream(x.device)))
    return loss, lse, dx, dtable


def _dense(a):
    """Whether a's values fill one piece of memory, in whatever order of its dimensions."""
    n = 1
    for size, stride in sorted(((s, st) for s, st in zip(a.shape, a.stride()) if s > 1), key=lambda q: q[1]):
        if stride != n:
            return False
        n *= size
    return True


def _tensors(tensors, out):
    tensors = list(tensors)
    n = len(tensors)
    device = tensors[0].device if n and isinstance(tensors[0], torch.Tensor) else None
    kinds, sizes, flat = [], [], True
    for a in tensors:
        kind = _DTYPES.get(a.dtype) if isinstance(a, torch.Tensor) else None
        if kind is None:
            raise TypeError("gradients must be float32, bfloat16 or float16 tensors")
        if not a.is_cuda or a.device != device:
            raise ValueError("gradients must be in the memory of one device")
        if not a.is_contiguous():
            flat = False
            if not _dense(a):
                raise ValueError("gradients must fill one piece of memory each")
        kinds.append(kind)
        sizes.append(a.numel())
    P = ctypes.c_void_p * n
    ins = outs = P(*[a.data_ptr() for a in tensors])
    if out is not None:
        out = list(out)
        if len(out) != n:
            raise ValueError("out must have one tensor for each gradient")
        for a, o in zip(tensors, out):
            if o.shape != a.shape or o.dtype != a.dtype or o.device != device or not (
                    o.is_contiguous() if flat else o.stride() == a.stride() or a.numel() < 2):
                raise ValueError("out must be like the gradients in shape, strides, type and device")
        outs = P(*[o.data_ptr() for o in out])
    return (device or torch.device("cuda", torch.cuda.current_device()), n, ins, outs, (ctypes.c_int64 * n)(*sizes),
            (ctypes.c_int32 * n)(*kinds))


@functools.lru_cache(maxsize=None)
def _norm_workspace_bytes():
    n = ctypes.c_int64()
    _check(_lib().ccdpp_grad_norm_workspace(ctypes.byref(n)))
    return n.value


def grad_norm(tensors):
    """The 2-norm of all values of the tensors together: a float32 scalar in device memory."""
    device, n, ptrs, _, sizes, dtypes = _tensors(tensors, None)
    with _On(device):
        norm = torch.empty((), dtype=torch.float32, device=device)
        ws = torch.empty(_norm_workspace_bytes(), dtype=torch.uint8, device=device)
        _check(_lib().ccdpp_grad_norm(n, ptrs, sizes, dtypes, norm.data_ptr(), ws.data_ptr(), ws.numel(), _stream(device)))
    return norm


def clip_grads(tensors, max_norm, *, eps=1e-6, out=None):
    """Multiplies all tensors with min(1, max_norm / (norm + eps)), in place or into `out`; returns their norm before
    that (a float32 scalar in device memory).  A norm that is NaN makes every value NaN, an infinite one the finite
    values 0."""
    device, n, ptrs, outs, sizes, dtypes = _tensors(tensors, out)
    with _On(device):
        norm = torch.empty((), dtype=torch.float32, device=device)
        ws = torch.empty(_norm_workspace_bytes(), dtype=torch.uint8, device=device)
        _check(_lib().ccdpp_clip_grads(n, ptrs, outs, sizes, dtypes, max_norm, eps,
                                       norm.data_ptr(), ws.data_ptr(), ws.numel(), _stream(device)))
    return norm
