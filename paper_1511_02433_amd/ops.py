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


# Tells autograd that tensors of the caller's have other values now, as torch's own operators in place do.
_written = torch.autograd.graph.increment_version


def _check(rc):
    if rc < 0:
        raise _c.CCDPPError(rc, _lib().ccdpp_ops_last_error().decode())


class _On:
    """Makes a device current while a call runs, where it is not."""
    __slots__ = ("guard",)

    def __init__(self, index):
        self.guard = None if index == torch.cuda.current_device() else torch.cuda.device(index)

    def __enter__(self):
        if self.guard:
            self.guard.__enter__()

    def __exit__(self, *exc):
        if self.guard:
            self.guard.__exit__(*exc)


def _matrix(a, name):
    """The row stride of a matrix of device memory."""
    if not isinstance(a, torch.Tensor) or a.dim() != 2:
        raise TypeError(f"{name} must be a matrix (a two-dimensional tensor)")
    if a.get_device() < 0:
        raise ValueError(f"{name} must be in device memory")
    if a.dtype not in _DTYPES:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, not {a.dtype}")
    rows, d = a.shape
    ld, step = a.stride()
    if step != 1 and d > 1:
        raise ValueError(f"{name}'s rows must be contiguous")
    return ld if rows > 1 else max(d, 1)


def _vector(a, name, n, dtypes, index):
    if not isinstance(a, torch.Tensor) or a.dtype not in dtypes:
        raise TypeError(f"{name} must be a tensor of {' or '.join(str(t)[6:] for t in dtypes)}")
    if a.dim() != 1 or a.numel() != n or not a.is_contiguous():
        raise ValueError(f"{name} must be contiguous, with {n} values")
    if a.get_device() != index:
        raise ValueError(f"{name} must be on device {index}")
    return a.data_ptr()


_INTS, _FLOATS = (torch.int64, torch.int32), (torch.float32,)


def _problem(x, table, target, scale, offset):
    ldx, ldt = _matrix(x, "x"), _matrix(table, "table")
    index, dtype = x.get_device(), x.dtype
    if dtype != table.dtype or index != table.get_device():
        raise ValueError("x and table must have the same type and device")
    (t, d), (v, e) = x.shape, table.shape
    if d != e:
        raise ValueError(f"x has {d} columns and table {e}")
    y = _vector(target, "target", t, _INTS, index)
    o = None if offset is None else _vector(offset, "offset", v, _FLOATS, index)
    return Softmax(t, v, d, _DTYPES[dtype], x.data_ptr(), ldx, table.data_ptr(), ldt, y,
                   64 if target.dtype == torch.int64 else 32, scale, o), index


def _workspace(p, call, device):
    n = ctypes.c_int64()
    _check(_lib().ccdpp_softmax_workspace(ctypes.byref(p), call, ctypes.byref(n)))
    return torch.empty(n.value, dtype=torch.uint8, device=device), n


# PyTorch's current stream of a device, as the handle alone (1.9 us with the stream object).
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _out(a, like, name):
    if _matrix(a, name) < 0 or a.shape != like.shape or a.dtype != like.dtype or a.get_device() != like.get_device():
        raise ValueError(f"{name} must have the shape, type and device of what it is the gradient of")
    return a


def _gradient_buffers(x, table, dx, dtable, need):
    """(dx, its pointer, its row stride, dtable, ...) for the gradients that are asked for."""
    if not set(need) <= {"x", "table"}:
        raise ValueError(f"need is made of 'x' and 'table', not {need!r}")
    got = []
    for name, like, a in (("x", x, dx), ("table", table, dtable)):
        if name not in need:
            got += [None, None, 0]
        elif a is None:
            a = torch.empty(like.shape, dtype=like.dtype, device=like.device)
            got += [a, a.data_ptr(), max(like.shape[1], 1)]
        else:
            a = _out(a, like, "d" + name)
            got += [a, a.data_ptr(), _matrix(a, "d" + name)]
    return got


def softmax_loss(x, table, target, *, scale=1.0, offset=None):
    """(loss, lse), float32 per row: lse[i] = log sum_v exp(scale x_i.table_v + offset_v), loss[i] = lse[i] - the
    target's logit.  x: t x d, table: v x d (float32, bfloat16 or float16; rows may lie apart), target: int32 or int64.
    A negative target marks an ignored row (loss 0); one past the table makes the row's loss NaN.  offset: float32 per
    item or None; -inf (or anything below -1e38) excludes an item, and a target that is excluded has loss +inf.  No graph is
    recorded, whatever x and table require: softmax_loss_grad and softmax_loss_train give the gradients."""
    p, index = _problem(x, table, target, scale, offset)
    device = x.device
    with _On(index):
        loss = torch.empty(p.t, dtype=torch.float32, device=device)
        lse = torch.empty(p.t, dtype=torch.float32, device=device)
        ws, n = _workspace(p, LOSS, device)
        _check(_lib().ccdpp_softmax_loss(ctypes.byref(p), loss.data_ptr(), lse.data_ptr(), ws.data_ptr(), n, _stream(index)))
    return loss, lse


def softmax_loss_grad(x, table, target, lse, *, grad=None, scale=1.0, offset=None, dx=None, dtable=None, need=("x", "table")):
    """(dx, dtable): gradients of sum_i grad[i] loss[i], from the lse of softmax_loss.  grad: float32 per row, or None
    for ones.  dx and dtable may be given to write to.  A gradient that is not in `need` is not computed (None).
    Ignored rows, rows whose target is excluded and excluded items take no part, whatever they hold."""
    p, index = _problem(x, table, target, scale, offset)
    l = _vector(lse, "lse", p.t, _FLOATS, index)
    g = None if grad is None else _vector(grad, "grad", p.t, _FLOATS, index)
    given = [a for a in (dx, dtable) if a is not None]
    with _On(index):
        dx, pdx, lddx, dtable, pde, ldde = _gradient_buffers(x, table, dx, dtable, need)
        ws, n = _workspace(p, GRAD, x.device)
        _check(_lib().ccdpp_softmax_loss_grad(ctypes.byref(p), l, g, pdx, lddx, pde, ldde, ws.data_ptr(), n, _stream(index)))
    if given:
        _written(given)
    return dx, dtable


def softmax_loss_train(x, table, target, *, grad=None, scale=1.0, offset=None, dx=None, dtable=None, need=("x", "table")):
    """(loss, lse, dx, dtable): softmax_loss and softmax_loss_grad in one call, for rows whose weights `grad` are known
    beforehand (1 / the number of rows that count, for a mean)."""
    p, index = _problem(x, table, target, scale, offset)
    g = None if grad is None else _vector(grad, "grad", p.t, _FLOATS, index)
    device = x.device
    given = [a for a in (dx, dtable) if a is not None]
    with _On(index):
        loss = torch.empty(p.t, dtype=torch.float32, device=device)
        lse = torch.empty(p.t, dtype=torch.float32, device=device)
        dx, pdx, lddx, dtable, pde, ldde = _gradient_buffers(x, table, dx, dtable, need)
        ws, n = _workspace(p, TRAIN, device)
        _check(_lib().ccdpp_softmax_loss_train(ctypes.byref(p), loss.data_ptr(), lse.data_ptr(), g, pdx, lddx, pde, ldde,
                                               ws.data_ptr(), n, _stream(index)))
    if given:
        _written(given)
    return loss, lse, dx, dtable


def _dense(a):
    """Whether a's values fill one piece of memory, in whatever order of its dimensions."""
    n = 1
    for size, stride in sorted(((s, st) for s, st in zip(a.shape, a.stride()) if s > 1), key=lambda q: q[1]):
        if stride != n:
            return False
        n *= size
    return True


def _each(method, tensors):
    return list(map(method, tensors))


def _tensors(tensors, out):
    """(device index, n, the library's tables of) the gradients and what they are clipped into; `tensors` is a list."""
    n = len(tensors)
    T = torch.Tensor
    where = set(_each(T.get_device, tensors))  # (a TypeError for what is no tensor)
    dtypes = [a.dtype for a in tensors]
    kinds = [_DTYPES.get(t) for t in dtypes]
    if None in kinds:
        raise TypeError("gradients must be float32, bfloat16 or float16 tensors")
    if len(where) > 1 or -1 in where:
        raise ValueError("gradients must be in the memory of one device")
    flat = all(map(T.is_contiguous, tensors))
    if not flat and not all(map(_dense, tensors)):
        raise ValueError("gradients must fill one piece of memory each")
    sizes = _each(T.numel, tensors)
    P = ctypes.c_void_p * n
    ins = outs = P(*_each(T.data_ptr, tensors))
    if out is not None:
        if len(out) != n:
            raise ValueError("out must have one tensor for each gradient")
        if (not set(_each(T.get_device, out)) <= where or [o.dtype for o in out] != dtypes or _each(T.numel, out) != sizes
                or _each(T.dim, out) != _each(T.dim, tensors)
                or not (all(map(T.is_contiguous, out)) if flat else all(
                    o.shape == a.shape and (o.stride() == a.stride() or a.numel() < 2) for a, o in zip(tensors, out)))):
            raise ValueError("out must be like the gradients in shape, strides, type and device")
        outs = P(*_each(T.data_ptr, out))
    return (where.pop() if where else torch.cuda.current_device(), n, ins, outs, (ctypes.c_int64 * n)(*sizes),
            (ctypes.c_int32 * n)(*kinds))


@functools.lru_cache(maxsize=None)
def _norm_workspace_bytes():
    n = ctypes.c_int64()
    _check(_lib().ccdpp_grad_norm_workspace(ctypes.byref(n)))
    return n.value


def grad_norm(tensors):
    """The 2-norm of all values of the tensors together: a float32 scalar in device memory."""
    index, n, ptrs, _, sizes, dtypes = _tensors(list(tensors), None)
    with _On(index):
        device = torch.device("cuda", index)
        norm = torch.empty((), dtype=torch.float32, device=device)
        ws = torch.empty(_norm_workspace_bytes(), dtype=torch.uint8, device=device)
        _check(_lib().ccdpp_grad_norm(n, ptrs, sizes, dtypes, norm.data_ptr(), ws.data_ptr(), ws.numel(), _stream(index)))
    return norm


def clip_grads(tensors, max_norm, *, eps=1e-6, out=None):
    """Multiplies all tensors with min(1, max_norm / (norm + eps)), in place or into `out`; returns their norm before
    that (a float32 scalar in device memory).  A norm that is NaN makes every value NaN, an infinite one the finite
    values 0 (unless max_norm is infinite, too).  A tensor is there once: one that shares memory with another would be
    read by one block while another clips it."""
    tensors, out = list(tensors), None if out is None else list(out)
    index, n, ptrs, outs, sizes, dtypes = _tensors(tensors, out)
    with _On(index):
        device = torch.device("cuda", index)
        norm = torch.empty((), dtype=torch.float32, device=device)
        ws = torch.empty(_norm_workspace_bytes(), dtype=torch.uint8, device=device)
        _check(_lib().ccdpp_clip_grads(n, ptrs, outs, sizes, dtypes, max_norm, eps, norm.data_ptr(), ws.data_ptr(), ws.numel(),
                                       _stream(index)))
    _written(tensors if out is None else out)
    return norm
