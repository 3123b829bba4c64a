"""Operators on sequences of choices, on torch tensors in device memory (binding of include/ccdpp_seq.h).

A gated linear recurrence over packed sequences of rows (the factors of the items that users took, one after another)
with its gradients and its form for one more row, the selection of beams with the reordering of their states, and
dropout whose mask is drawn from a counter.  Its place is before and after ops.softmax_loss: the recurrence's rows,
with dropout in training, are the rows that choose among all items; beams answer with several items in sequence.
As in ops, everything is computed in libccdpp.so on torch's current stream, nothing waits for the device, no graph is
recorded for autograd, and refused arguments raise ValueError or TypeError here, or CCDPPError (EINVAL) where the library
finds them.
"""
from __future__ import annotations

import ctypes
import functools
from operator import index as _whole

import torch

from . import ccdpp as _c
from .ops import _DTYPES, _FLOATS, _INTS, _On, _check, _matrix, _stream, _vector, _written

FORWARD, GRAD = range(2)
MODES = {"given": 0, "sigmoid": 1}


class Scan(ctypes.Structure):
    """ccdpp_scan_t."""
    _fields_ = [("n", ctypes.c_int64), ("s", ctypes.c_int64), ("d", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("mode", ctypes.c_int32), ("starts_bits", ctypes.c_int32), ("x", ctypes.c_void_p), ("ldx", ctypes.c_int64),
                ("gate", ctypes.c_void_p), ("ldg", ctypes.c_int64), ("starts", ctypes.c_void_p), ("initial", ctypes.c_void_p)]


class Beam(ctypes.Structure):
    """ccdpp_beam_t."""
    _fields_ = [("groups", ctypes.c_int64), ("v", ctypes.c_int64), ("beams", ctypes.c_int32), ("k", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32), ("logits", ctypes.c_void_p), ("ld", ctypes.c_int64),
                ("score", ctypes.c_void_p), ("offset", ctypes.c_void_p), ("done", ctypes.c_void_p), ("end", ctypes.c_int64)]


@functools.lru_cache(maxsize=None)
def _lib():
    L = _c.lib()
    P, i64, i32, f64, u64 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_double, ctypes.c_uint64
    S, B, N = ctypes.POINTER(Scan), ctypes.POINTER(Beam), ctypes.POINTER(i64)
    sig = {
        "ccdpp_scan_workspace": [S, i32, N],
        "ccdpp_scan_kept": [S, N],
        "ccdpp_gated_scan": [S, P, i64, P, P, P, i64, P],
        "ccdpp_gated_scan_grad": [S, P, i64, P, P, P, i64, P, i64, P, P, i64, P],
        "ccdpp_gated_scan_step": [i64, i32, i32, i32, P, i64, P, i64, P, i64, P, i64, P],
        "ccdpp_beam_workspace": [B, N],
        "ccdpp_beam_select": [B, P, P, P, P, P, i64, P],
        "ccdpp_beam_reorder": [i64, i32, i32, P, i32, P, P, P, P, P],
        "ccdpp_dropout": [i64, i64, i32, P, i64, P, i64, P, i64, f64, u64, P, i64, P],
    }
    for name, args in sig.items():
        f = getattr(L, name)
        f.argtypes, f.restype = args, ctypes.c_int
    L.ccdpp_ops_last_error.argtypes, L.ccdpp_ops_last_error.restype = [], ctypes.c_char_p
    return L


def _mode(mode):
    if mode not in MODES:
        raise ValueError(f"mode is 'sigmoid' or 'given', not {mode!r}")
    return MODES[mode]


def _alike(a, name, x):
    """The row stride of a matrix that has x's shape, type and device."""
    ld = _matrix(a, name)
    if a.shape != x.shape or a.dtype != x.dtype or a.get_device() != x.get_device():
        raise ValueError(f"{name} must have the shape, type and device of x")
    return ld


def _states(a, name, s, d, index):
    """The pointer of s contiguous rows of d states."""
    if not isinstance(a, torch.Tensor) or a.dtype != torch.float32:
        raise TypeError(f"{name} must be a tensor of float32")
    if a.shape != (s, d) or not a.is_contiguous():
        raise ValueError(f"{name} must be contiguous, {s} x {d}")
    if a.get_device() != index:
        raise ValueError(f"{name} must be on device {index}")
    return a.data_ptr()


def _given(a, name, x):
    """What is written to, given or new, and its row stride."""
    if a is None:
        return torch.empty_like(x) if x.is_contiguous() else torch.empty(x.shape, dtype=x.dtype, device=x.device), max(x.shape[1], 1)
    return a, _alike(a, name, x)


def _sequences(x, gate, starts, initial, mode):
    ldx = _matrix(x, "x")
    ldg, index = _alike(gate, "gate", x), x.get_device()
    n, d = x.shape
    if d > 65536:
        raise ValueError("d must be in [1, 65536]")
    s = (starts.numel() if isinstance(starts, torch.Tensor) else 0) - 1
    if s < 0:
        raise ValueError("starts must be a vector with at least one value")
    at = _vector(starts, "starts", s + 1, _INTS, index)
    first = None if initial is None else _states(initial, "initial", s, d, index)
    return Scan(n, s, d, _DTYPES[x.dtype], _mode(mode), 64 if starts.dtype == torch.int64 else 32, x.data_ptr(), ldx,
                gate.data_ptr(), ldg, at, first), index


# Sizes of workspaces go by the problems' sizes: asked for once (a call of the library takes a microsecond or two).
@functools.lru_cache(maxsize=4096)
def _scan_bytes(n, s, d, dtype, mode, call):
    """Bytes of the workspace of a call, or (None) rows of kept states."""
    p, got = Scan(n, s, d, dtype, mode, 64, None, d, None, d, None, None), ctypes.c_int64()
    if call is None:
        _check(_lib().ccdpp_scan_kept(ctypes.byref(p), ctypes.byref(got)))
        return got.value // (4 * d)
    _check(_lib().ccdpp_scan_workspace(ctypes.byref(p), call, ctypes.byref(got)))
    return got.value


def _kept_rows(p):
    return _scan_bytes(p.n, p.s, p.d, p.dtype, p.mode, None)


def _scan_workspace(p, call, device):
    n = _scan_bytes(p.n, p.s, p.d, p.dtype, p.mode, call)
    return torch.empty(n, dtype=torch.uint8, device=device), n


def gated_scan(x, gate, *, starts, initial=None, mode="sigmoid", keep=False, y=None):
    """(y, last), or (y, last, kept) with `keep`: h_t = a_t h_(t-1) + u_t along each sequence of rows, every column by itself.
    mode 'sigmoid': a = sigmoid(gate), u = (1 - a) x; 'given': a = gate, u = x (decays above 1 as long as products of any that follow
    one another stay within float32's range).  x, gate: n x d (float32, bfloat16 or float16;
    rows may lie apart).  starts: s + 1 ascending int32 or int64 values: sequence q has rows starts[q] to starts[q + 1] - 1; rows
    outside of all are not read and 0 in y.  initial: float32, s x d, the states before the sequences' first rows, or None for
    zeros.  y has x's type (or may be given to write to); last: float32, s x d, the states behind the last rows; kept: what
    gated_scan_grad needs."""
    p, index = _sequences(x, gate, starts, initial, mode)
    device, out = x.device, y
    with _On(index):
        y, ldy = _given(y, "y", x)
        last = torch.empty((p.s, p.d), dtype=torch.float32, device=device)
        kept, at = None, None
        if keep:
            kept = torch.empty(_kept_rows(p), p.d, dtype=torch.float32, device=device)
            at = kept.data_ptr()
        ws, n = _scan_workspace(p, FORWARD, device)
        _check(_lib().ccdpp_gated_scan(ctypes.byref(p), y.data_ptr(), ldy, last.data_ptr(), at, ws.data_ptr(), n, _stream(index)))
    if out is not None:
        _written([out])
    return (y, last, kept) if keep else (y, last)


def gated_scan_grad(x, gate, dy, kept, *, starts, initial=None, mode="sigmoid", dlast=None, dx=None, dgate=None):
    """(dx, dgate, dinitial): gradients of sum(dy y) + sum(dlast last), from what gated_scan kept for the same arguments.  dlast:
    float32, s x d, or None for zeros; dinitial is None where initial is.  dx and dgate may be given to write to."""
    p, index = _sequences(x, gate, starts, initial, mode)
    lddy = _alike(dy, "dy", x)
    k = _states(kept, "kept", _kept_rows(p), p.d, index)
    dl = None if dlast is None else _states(dlast, "dlast", p.s, p.d, index)
    given = [a for a in (dx, dgate) if a is not None]
    with _On(index):
        dx, lddx = _given(dx, "dx", x)
        dgate, lddg = _given(dgate, "dgate", x)
        dinitial = None if initial is None else torch.empty((p.s, p.d), dtype=torch.float32, device=x.device)
        ws, n = _scan_workspace(p, GRAD, x.device)
        _check(_lib().ccdpp_gated_scan_grad(ctypes.byref(p), dy.data_ptr(), lddy, dl, k, dx.data_ptr(), lddx, dgate.data_ptr(), lddg,
                                            None if dinitial is None else dinitial.data_ptr(), ws.data_ptr(), n, _stream(index)))
    if given:
        _written(given)
    return dx, dgate, dinitial


def gated_scan_step(x, gate, state, *, mode="sigmoid", y=None):
    """One more row of n sequences: state = a state + u in place (float32, n x d), and y = state in x's type."""
    ldx = _matrix(x, "x")
    ldg, index = _alike(gate, "gate", x), x.get_device()
    lds = _matrix(state, "state")
    if x.shape[1] > 65536:
        raise ValueError("d must be in [1, 65536]")
    if state.dtype != torch.float32 or state.shape != x.shape or state.get_device() != index:
        raise ValueError("state must be float32, with the shape and device of x")
    out = y
    with _On(index):
        y, ldy = _given(y, "y", x)
        _check(_lib().ccdpp_gated_scan_step(x.shape[0], x.shape[1], _DTYPES[x.dtype], _mode(mode), x.data_ptr(), ldx, gate.data_ptr(), ldg,
                                            state.data_ptr(), lds, y.data_ptr(), ldy, _stream(index)))
    _written([state] if out is None else [state, out])
    return y


def _count(a, name):
    a = _whole(a)
    if not 1 <= a <= 64:
        raise ValueError(f"{name} must be in [1, 64], not {a}")
    return a


@functools.lru_cache(maxsize=4096)
def _beam_bytes(g, v, b, k, dtype):
    p, got = Beam(g, v, b, k, dtype, 0, None, v, None, None, None, -1), ctypes.c_int64()
    _check(_lib().ccdpp_beam_workspace(ctypes.byref(p), ctypes.byref(got)))
    return got.value


def beam_select(logits, score, k, *, offset=None, done=None, end=None):
    """(score, parent, item, done): the k best continuations of each group of beams, in descending order.  score: float32, g x b;
    logits: (g b) x v, the beams' rows one group after another (float32, bfloat16 or float16; rows may lie apart).  Beam b
    continued by item i has the score score_b + z_i - log sum exp z, z = logits + offset (in 32 bits; the log sum within 2^-17); of equal
    ones the lowest beam goes first, and of a beam the greatest z, then the lowest item.  offset: float32 per item; -inf (or below -1e38) excludes it.  A beam with score -inf is none.  done:
    bool, g x b: such a beam is at its end and goes on as itself, with the item `end`.  parent (the beam within the group) and item:
    int64, g x k, and score; -1, -1 and -inf where there are fewer than k.  done is None where `end` is."""
    ld = _matrix(logits, "logits")
    index = logits.get_device()
    if not isinstance(score, torch.Tensor) or score.dim() != 2:
        raise TypeError("score must be a matrix (a two-dimensional tensor)")
    g, b = score.shape
    _count(b, "beams")
    k = _count(k, "k")
    rows, v = logits.shape
    if rows != g * b:
        raise ValueError(f"logits must have a row for each of the {g} x {b} beams, not {rows}")
    s = _states(score, "score", g, b, index)
    o = None if offset is None else _vector(offset, "offset", v, _FLOATS, index)
    f = None
    if done is not None:
        if end is None:
            raise ValueError("done needs the item that ends a beam")
        if not isinstance(done, torch.Tensor) or done.dtype != torch.bool:
            raise TypeError("done must be a tensor of bool")
        if done.shape != score.shape or not done.is_contiguous() or done.get_device() != index:
            raise ValueError("done must be contiguous, with the shape and device of score")
        f = done.data_ptr()
    if end is not None:
        end = _whole(end)
        if not 0 <= end < v:
            raise ValueError(f"end must be an item, in [0, {v})")
    p = Beam(g, v, b, k, _DTYPES[logits.dtype], 0, logits.data_ptr(), ld, s, o, f, -1 if end is None else end)
    L, device = _lib(), logits.device
    with _On(index):
        n = _beam_bytes(g, v, b, k, p.dtype)
        ws = torch.empty(n, dtype=torch.uint8, device=device)
        out = torch.empty_like(score) if k == b else torch.empty((g, k), dtype=torch.float32, device=device)
        parent, item = torch.empty((2, g, k), dtype=torch.int64, device=device).unbind()
        ended = None if end is None else torch.empty((g, k), dtype=torch.bool, device=device)
        _check(L.ccdpp_beam_select(ctypes.byref(p), out.data_ptr(), parent.data_ptr(), item.data_ptr(), None if ended is None else ended.data_ptr(),
                                   ws.data_ptr(), n, _stream(index)))
    return out, parent, item, ended


def beam_reorder(parent, states, *, beams, out=None):
    """The states that the continuations of beam_select start from: for each tensor (its first dimension g x beams, each of its
    rows contiguous, any type) one whose rows (g, j) are rows (g, parent[g, j]); zeros where parent is none of the group's beams.
    `out`: contiguous tensors to write to, none of them a part of `states`."""
    if not isinstance(parent, torch.Tensor) or parent.dtype != torch.int64 or parent.dim() != 2:
        raise TypeError("parent must be a matrix of int64")
    g, k = parent.shape
    index, states = parent.get_device(), list(states)
    beams, k = _count(beams, "beams"), _count(k, "k")
    if index < 0 or not parent.is_contiguous():
        raise ValueError("parent must be contiguous, in device memory")
    n = len(states)
    if out is not None:
        out = list(out)
        if len(out) != n:
            raise ValueError("out must have one tensor for each state")
    rows, to = g * beams, g * k
    with _On(index):
        strides, sizes, got = [], [], []
        for i, a in enumerate(states):
            if not isinstance(a, torch.Tensor) or a.dim() < 1:
                raise TypeError("states must be tensors with a row for each beam")
            if a.get_device() != index or a.shape[0] != rows:
                raise ValueError(f"states must have {rows} rows, on the device of parent")
            if a.is_conj() or a.is_neg():  # views whose memory holds other values than they stand for
                a = states[i] = a.resolve_conj().resolve_neg()
            row = a.nbytes // max(rows, 1)
            sizes.append(row)
            if a.is_contiguous():
                strides.append(row)
                if out is None:
                    got.append(torch.empty_like(a) if to == rows else a.new_empty((to, *a.shape[1:])))
            else:
                apart = a.stride(0) * a.element_size()
                if not a[0].is_contiguous() or apart < row:
                    raise ValueError("rows of states must be contiguous")
                strides.append(apart)
                if out is None:
                    got.append(a.new_empty((to, *a.shape[1:])))
        if out is not None:
            got = out
            for a, o in zip(states, out):
                if (not isinstance(o, torch.Tensor) or o.shape != (to, *a.shape[1:]) or o.dtype != a.dtype or o.get_device() != index
                        or not o.is_contiguous() or o.is_conj() or o.is_neg()):
                    raise ValueError("out must be contiguous (no conjugate), with the states' type and row shape, and a row for each continuation")
        P, N = ctypes.c_void_p * n, ctypes.c_int64 * n
        _check(_lib().ccdpp_beam_reorder(g, beams, k, parent.data_ptr(), n, P(*[a.data_ptr() for a in states]), N(*strides),
                                         P(*[o.data_ptr() for o in got]), N(*sizes), _stream(index)))
    if out is not None:
        _written(out)
    return got


def dropout(x, p, seed, *, first_row=0, residual=None, out=None):
    """[residual +] x * [r >= p] / (1 - p), with r from a counter (row, column) and the seed: the same call gives the same mask, so
    the gradient of x is dropout(dy, p, seed, first_row=first_row).  x, residual: n x d (float32, bfloat16 or float16; rows may lie
    apart).  seed: an integer of 64 bits, or an int64 tensor of one value in device memory, read when the work runs (a captured
    graph draws another mask when it changes).  first_row: the number of x's first row among all rows that share the seed.  `out` may
    be x or residual."""
    ldx, index = _matrix(x, "x"), x.get_device()
    ldr = 0 if residual is None else _alike(residual, "residual", x)
    at = None
    if isinstance(seed, torch.Tensor):
        if seed.dtype != torch.int64 or seed.numel() != 1 or seed.get_device() != index:
            raise ValueError("a seed in device memory must be one int64 value on the device of x")
        at, seed = seed.data_ptr(), 0
    else:
        seed = _whole(seed)
        if not -2 ** 63 <= seed < 2 ** 64:
            raise ValueError("seed must fit 64 bits")
    try:
        p = ctypes.c_double(p)  # (what is no number is a TypeError)
    except OverflowError:
        raise ValueError("p must be in [0, 1]") from None
    first_row = _whole(first_row)
    if not 0 <= first_row < 2 ** 63:
        raise ValueError("first_row must be in [0, 2^63)")
    with _On(index):
        y, ldy = _given(out, "out", x)
        _check(_lib().ccdpp_dropout(x.shape[0], x.shape[1], _DTYPES[x.dtype], x.data_ptr(), ldx, None if residual is None else residual.data_ptr(), ldr,
                                    y.data_ptr(), ldy, p, seed & 0xFFFFFFFFFFFFFFFF, at, first_row, _stream(index)))
    if out is not None:
        _written([out])
    return y
