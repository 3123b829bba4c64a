"""The C ABI of the operators on sequences without a GPU: every function of include/ccdpp_seq.h is exported and bound, and bad
arguments are refused on the host, before any HIP call, with a message."""
import ctypes
import math
import os
import re

import pytest

torch = pytest.importorskip("torch")

import paper_1511_02433_amd.ccdpp as C
from paper_1511_02433_amd import seq

HEADER = os.path.join(os.path.dirname(C.HEADER), "ccdpp_seq.h")
B, E = ctypes.byref, C.CCDPP_EINVAL


def _lib_or_skip():
    try:
        return seq._lib()
    except RuntimeError as e:  # not built in this checkout
        pytest.skip(str(e))


def said(L, msg):
    return msg in L.ccdpp_ops_last_error().decode()


def test_every_declared_function_is_exported_and_bound():
    L = _lib_or_skip()
    with open(HEADER) as f:
        names = sorted(set(re.findall(r"^int (ccdpp_[a-z_]+)\s*\(", f.read(), re.M)))
    assert len(names) == 9
    for n in names:
        assert getattr(L, n).argtypes is not None, n


def scan(**kw):
    f = dict(n=4, s=2, d=8, dtype=0, mode=1, starts_bits=64, x=256, ldx=8, gate=256, ldg=8, starts=256, initial=None)
    f.update(kw)
    return seq.Scan(*[f[n] for n, _ in seq.Scan._fields_])


SIZES = [(dict(n=-1), "n and s"), (dict(n=1 << 31), "n and s"), (dict(s=-1), "n and s"), (dict(s=1 << 31), "n and s"), (dict(d=0), "d must"),
         (dict(d=65537), "d must"), (dict(dtype=3), "dtype"), (dict(dtype=-1), "dtype"), (dict(mode=2), "mode"), (dict(starts_bits=16), "starts_bits"),
         (dict(ldx=7), "ldx"), (dict(ldg=7), "ldg")]
POINTERS = [(dict(x=None), "non-NULL"), (dict(gate=None), "non-NULL"), (dict(starts=None), "non-NULL"), (dict(x=258), "aligned"), (dict(gate=258), "aligned"),
            (dict(starts=260), "aligned"), (dict(starts=258, starts_bits=32), "aligned"), (dict(initial=258), "aligned"), (dict(x=257, dtype=1), "aligned")]


@pytest.mark.parametrize("kw, msg", SIZES + POINTERS)
def test_scan_refuses_bad_problems(kw, msg):
    L = _lib_or_skip()
    p, n = scan(**kw), ctypes.c_int64()
    if (kw, msg) in SIZES:
        for rc in (L.ccdpp_scan_workspace(B(p), 0, B(n)), L.ccdpp_scan_kept(B(p), B(n))):
            assert rc == E and said(L, msg)
    else:  # sizes need no pointer
        assert L.ccdpp_scan_workspace(B(p), 1, B(n)) == 0 and L.ccdpp_scan_kept(B(p), B(n)) == 0
    assert L.ccdpp_gated_scan(B(p), 256, 8, 256, 256, 256, 1 << 40, None) == E and said(L, msg)
    assert L.ccdpp_gated_scan_grad(B(p), 256, 8, 256, 256, 256, 8, 256, 8, 256, 256, 1 << 40, None) == E and said(L, msg)


def test_scan_refuses_bad_calls():
    L = _lib_or_skip()
    n = ctypes.c_int64()
    assert L.ccdpp_scan_workspace(None, 0, B(n)) == E and L.ccdpp_scan_workspace(B(scan()), 0, None) == E
    assert L.ccdpp_scan_workspace(B(scan()), 2, B(n)) == E and said(L, "call")
    assert L.ccdpp_scan_kept(B(scan()), None) == E
    need = {}
    for call in (0, 1):
        assert L.ccdpp_scan_workspace(B(scan()), call, B(n)) == 0
        need[call] = n.value
    for args, msg in (((None, 8, 256, 256, 256, 1 << 40), "y must"), ((256, 7, 256, 256, 256, 1 << 40), "ldy"), ((258, 8, 256, 256, 256, 1 << 40), "aligned"),
                      ((512, 8, 258, 256, 256, 1 << 40), "aligned"), ((512, 8, 256, 264, 256, 1 << 40), "aligned"), ((512, 8, 256, 256, None, 1 << 40), "workspace"),
                      ((512, 8, 256, 256, 264, 1 << 40), "workspace"), ((512, 8, 256, 256, 256, need[0] - 1), "workspace")):
        assert L.ccdpp_gated_scan(B(scan()), *args, None) == E and said(L, msg), args
    good = [768, 8, 256, 256, 1024, 8, 1280, 8, 256, 256, 1 << 40]
    for at, value, msg in ((0, None, "non-NULL"), (1, 7, "lddy"), (2, 258, "aligned"), (3, None, "non-NULL"), (3, 264, "aligned"), (4, None, "non-NULL"), (4, 258, "aligned"),
                           (5, 7, "lddx"), (6, None, "non-NULL"), (7, 7, "lddg"), (8, 258, "aligned"), (9, None, "workspace"), (10, need[1] - 1, "workspace")):
        args = list(good)
        args[at] = value
        assert L.ccdpp_gated_scan_grad(B(scan()), *args, None) == E and said(L, msg), (at, value)
    good = [4, 8, 0, 1, 256, 8, 256, 8, 256, 8, 256, 8]
    for at, value, msg in ((0, -1, "n and s"), (1, 0, "d must"), (2, 5, "dtype"), (3, 9, "mode"), (4, None, "non-NULL"), (4, 258, "aligned"), (5, 7, "ldx"), (6, None, "non-NULL"),
                           (8, None, "non-NULL"), (8, 258, "aligned"), (9, 7, "lds"), (10, None, "non-NULL"), (11, 7, "ldy")):
        args = list(good)
        args[at] = value
        assert L.ccdpp_gated_scan_step(*args, None) == E and said(L, msg), (at, value)


def test_outputs_that_are_inputs_are_refused():
    """The same pointer; other overlaps are the caller's to avoid.  (Dropout and the step may write in place.)"""
    L = _lib_or_skip()
    p = scan(x=256, gate=512, starts=1024)
    W = (2048, 1 << 40, None)
    for y in (256, 512):
        assert L.ccdpp_gated_scan(B(p), y, 8, 4096, None, *W) == E and said(L, "must not be an input")
    for dx, dg in ((256, 8192), (512, 8192), (4096, 8192), (8192, 256), (8192, 512), (8192, 4096), (8192, 8192)):
        assert L.ccdpp_gated_scan_grad(B(p), 4096, 8, None, 16384, dx, 8, dg, 8, None, *W) == E and said(L, "must not be an input"), (dx, dg)
    one, sz = (ctypes.c_void_p * 1)(256), (ctypes.c_int64 * 1)(8)
    assert L.ccdpp_beam_reorder(2, 3, 4, 256, 1, one, sz, one, sz, None) == E and said(L, "must not be an input")


def test_kept_states_and_workspaces_are_small():
    L = _lib_or_skip()
    n = ctypes.c_int64()
    for rows, s, d in ((0, 0, 1), (1, 1, 1), (17, 3, 65536), (1_000_209, 6041, 40), (32_768, 16, 4096), (65_537, 1, 100), ((1 << 31) - 1, (1 << 31) - 1, 8)):
        for dtype in (0, 1, 2):
            p = scan(n=rows, s=s, d=d, ldx=d, ldg=d, dtype=dtype)
            assert L.ccdpp_scan_kept(B(p), B(n)) == 0 and n.value == (rows + 7) // 8 * 4 * d
            for call in (0, 1):
                # a few numbers a row, and the states of the shares of rows
                assert L.ccdpp_scan_workspace(B(p), call, B(n)) == 0 and 0 <= n.value <= 8 * rows + 64 * d * 4096 + (1 << 20)


def beam(**kw):
    f = dict(groups=2, v=10, beams=3, k=4, dtype=0, reserved=0, logits=256, ld=10, score=256, offset=None, done=None, end=-1)
    f.update(kw)
    return seq.Beam(*[f[n] for n, _ in seq.Beam._fields_])


@pytest.mark.parametrize("kw, msg", [(dict(groups=-1), "groups"), (dict(groups=1 << 24), "groups"), (dict(beams=0), "beams and k"), (dict(beams=65), "beams and k"), (dict(k=0), "beams and k"),
                                     (dict(k=65), "beams and k"), (dict(v=0), "v must"), (dict(v=1 << 28, ld=1 << 28), "v must"), (dict(dtype=4), "dtype"), (dict(ld=9), "ld must"),
                                     (dict(end=10), "end"), (dict(end=-2), "end"), (dict(done=256), "done"), (dict(reserved=1), "reserved")])
def test_beam_refuses_bad_problems(kw, msg):
    L = _lib_or_skip()
    p, n = beam(**kw), ctypes.c_int64()
    assert L.ccdpp_beam_workspace(B(p), B(n)) == E and said(L, msg)
    assert L.ccdpp_beam_select(B(p), 256, 256, 256, None, 256, 1 << 40, None) == E and said(L, msg)


def test_beam_refuses_bad_calls():
    L = _lib_or_skip()
    n = ctypes.c_int64()
    assert L.ccdpp_beam_workspace(None, B(n)) == E and L.ccdpp_beam_workspace(B(beam()), None) == E
    assert L.ccdpp_beam_workspace(B(beam()), B(n)) == 0
    for kw, args, msg in ((dict(logits=None), (256, 256, 256, None, 256, 1 << 40), "non-NULL"), (dict(score=None), (256, 256, 256, None, 256, 1 << 40), "non-NULL"),
                          (dict(), (None, 256, 256, None, 256, 1 << 40), "non-NULL"), (dict(), (256, None, 256, None, 256, 1 << 40), "non-NULL"),
                          (dict(), (256, 256, None, None, 256, 1 << 40), "non-NULL"), (dict(logits=258), (256, 256, 256, None, 256, 1 << 40), "aligned"),
                          (dict(offset=258), (256, 256, 256, None, 256, 1 << 40), "aligned"), (dict(), (258, 256, 256, None, 256, 1 << 40), "aligned"),
                          (dict(), (256, 260, 256, None, 256, 1 << 40), "aligned"), (dict(), (256, 256, 260, None, 256, 1 << 40), "aligned"),
                          (dict(), (256, 256, 256, None, None, 1 << 40), "workspace"), (dict(), (256, 256, 256, None, 264, 1 << 40), "workspace"),
                          (dict(), (256, 256, 256, None, 256, n.value - 1), "workspace")):
        assert L.ccdpp_beam_select(B(beam(**kw)), *args, None) == E and said(L, msg), (kw, args)
    one, two, sz = (ctypes.c_void_p * 1)(256), (ctypes.c_void_p * 1)(512), (ctypes.c_int64 * 1)(8)
    good = [2, 3, 4, 256, 1, one, sz, two, sz]
    for at, value, msg in ((0, -1, "groups"), (1, 0, "beams"), (1, 65, "beams"), (2, 0, "beams"), (2, 65, "beams"), (3, None, "parent"), (3, 260, "parent"), (4, -1, "n must"),
                           (5, None, "tables"), (6, None, "tables"), (7, None, "tables"), (8, None, "tables"), (5, (ctypes.c_void_p * 1)(None), "NULL"),
                           (7, (ctypes.c_void_p * 1)(None), "NULL"), (6, (ctypes.c_int64 * 1)(7), "row_bytes"), (8, (ctypes.c_int64 * 1)(-1), "row_bytes")):
        args = list(good)
        args[at] = value
        assert L.ccdpp_beam_reorder(*args, None) == E and said(L, msg), (at, value)


def test_dropout_refuses_bad_calls():
    L = _lib_or_skip()
    good = [4, 8, 0, 256, 8, 512, 8, 1024, 8, 0.1, 7, None, 0]
    for at, value, msg in ((0, -1, "n must"), (0, 1 << 31, "n must"), (1, 0, "n must"), (1, 1 << 31, "n must"), (2, 3, "dtype"), (3, None, "non-NULL"), (3, 258, "aligned"),
                           (4, 7, "strides"), (5, 514, "aligned"), (6, 7, "strides"), (7, None, "non-NULL"), (7, 1026, "aligned"), (8, 7, "strides"), (9, -0.1, "p must"),
                           (9, 1.1, "p must"), (9, math.nan, "p must"), (11, 260, "aligned"), (12, -1, "first_row"), (12, (1 << 63) - 2, "first_row")):
        args = list(good)
        args[at] = value
        assert L.ccdpp_dropout(*args, None) == E and said(L, msg), (at, value)
    assert L.ccdpp_dropout(4, 8, 0, 256, 8, None, 0, 256, 9, 0.1, 7, None, 0, None) == E and said(L, "in place")
    assert L.ccdpp_dropout(4, 8, 0, 256, 8, 512, 8, 512, 9, 0.1, 7, None, 0, None) == E and said(L, "in place")


def test_without_a_device_calls_report_edevice():
    L = _lib_or_skip()
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    D = C.CCDPP_EDEVICE
    assert L.ccdpp_gated_scan(B(scan()), 512, 8, 256, 256, 256, 1 << 40, None) == D
    assert L.ccdpp_gated_scan_grad(B(scan()), 768, 8, 256, 256, 1024, 8, 1280, 8, 256, 256, 1 << 40, None) == D
    assert L.ccdpp_gated_scan_step(4, 8, 0, 1, 256, 8, 256, 8, 256, 8, 256, 8, None) == D
    assert L.ccdpp_beam_select(B(beam()), 256, 256, 256, None, 256, 1 << 40, None) == D
    one, two, sz = (ctypes.c_void_p * 1)(256), (ctypes.c_void_p * 1)(512), (ctypes.c_int64 * 1)(8)
    assert L.ccdpp_beam_reorder(2, 3, 4, 256, 1, one, sz, two, sz, None) == D
    assert L.ccdpp_dropout(4, 8, 0, 256, 8, None, 0, 1024, 8, 0.1, 7, None, 0, None) == D
    assert L.ccdpp_ops_last_error()


def test_the_binding_refuses():
    x, s = torch.ones(2, 3), torch.tensor([0, 2])
    with pytest.raises(ValueError):
        seq.gated_scan(x, x, starts=s)
    with pytest.raises(TypeError):
        seq.gated_scan(x[0], x, starts=s)
    with pytest.raises(ValueError):
        seq.gated_scan_step(x, x, x)
    with pytest.raises(ValueError):
        seq.beam_select(x, torch.zeros(1, 2), 2)
    with pytest.raises(TypeError):
        seq.beam_reorder(torch.zeros(1, 2), [x], beams=2)
    with pytest.raises(ValueError):
        seq.beam_reorder(torch.zeros(1, 2, dtype=torch.int64), [x], beams=2)
    with pytest.raises(ValueError):
        seq.dropout(x, 0.5, 1)
    with pytest.raises(ValueError):  # before the tensors' device is looked at
        seq._count(65, "k")
    with pytest.raises(TypeError):
        seq._count(2.0, "k")


def test_states_in_place_are_refused():
    """A sequence's first row, where its initial state is read, and its last one, where the last state is written, may be different blocks'."""
    L = _lib_or_skip()
    for initial in (4096, 8192):
        p = scan(x=256, gate=512, starts=1024, initial=initial)
        assert L.ccdpp_gated_scan(B(p), 2048, 8, initial, None, 16384, 1 << 40, None) == E and said(L, "last must not be initial")


@pytest.mark.parametrize("p, error", [("a", TypeError), ("0.1", TypeError), (None, TypeError), ([0.1], TypeError), (1j, TypeError),
                                      pytest.param(10 ** 400, ValueError, id="huge")])
def test_dropout_refuses_what_is_no_probability(p, error, monkeypatch):
    """With the errors that the module names, before the tensors' device is used."""
    monkeypatch.setattr(seq, "_matrix", lambda a, name: 3)
    with pytest.raises(error):
        seq.dropout(torch.ones(2, 3), p, 1)
