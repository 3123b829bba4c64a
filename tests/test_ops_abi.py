"""The operators' C ABI without a GPU: every function of include/ccdpp_ops.h is exported and bound, and bad arguments
are refused on the host, before any HIP call, with a message."""
import ctypes
import math
import os
import re

import pytest

torch = pytest.importorskip("torch")

import paper_1511_02433_amd.ccdpp as C
from paper_1511_02433_amd import ops

HEADER = os.path.join(os.path.dirname(C.HEADER), "ccdpp_ops.h")


def _lib_or_skip():
    try:
        return ops._lib()
    except RuntimeError as e:  # not built in this checkout
        pytest.skip(str(e))


def test_every_declared_function_is_exported_and_bound():
    L = _lib_or_skip()
    with open(HEADER) as f:
        names = sorted(set(re.findall(r"\b(ccdpp_[a-z_]+)\s*\(", f.read())))
    assert len(names) == 8
    for n in names:
        assert getattr(L, n).argtypes is not None, n


def _problem(**kw):
    f = dict(t=4, v=10, d=8, dtype=0, x=256, ldx=8, table=256, ldt=8, target=256, target_bits=64, scale=1.0, offset=None)
    f.update(kw)
    return ops.Softmax(*[f[n] for n, _ in ops.Softmax._fields_])


BAD = [(dict(t=-1), "t must"), (dict(t=1 << 26), "t must"), (dict(v=0), "v must"), (dict(v=1 << 28), "v must"),
       (dict(d=0), "d must"), (dict(d=65537), "d must"), (dict(dtype=3), "dtype"), (dict(dtype=-1), "dtype"),
       (dict(ldx=7), "ldx"), (dict(ldt=7), "ldt"), (dict(t=(1 << 25), v=(1 << 20)), "2^39"), (dict(target_bits=16), "target_bits"),
       (dict(scale=math.inf), "scale"), (dict(scale=math.nan), "scale")]


@pytest.mark.parametrize("kw, msg", BAD)
def test_softmax_refuses_bad_problems(kw, msg):
    L = _lib_or_skip()
    p, n = _problem(**kw), ctypes.c_int64()
    assert L.ccdpp_softmax_workspace(ctypes.byref(p), ops.LOSS, ctypes.byref(n)) == C.CCDPP_EINVAL
    assert msg in L.ccdpp_ops_last_error().decode()
    assert L.ccdpp_softmax_loss(ctypes.byref(p), 256, 256, 256, 1 << 40, None) == C.CCDPP_EINVAL
    assert L.ccdpp_softmax_loss_grad(ctypes.byref(p), 256, None, 256, 8, 256, 8, 256, 1 << 40, None) == C.CCDPP_EINVAL
    assert L.ccdpp_softmax_loss_train(ctypes.byref(p), 256, 256, None, 256, 8, 256, 8, 256, 1 << 40, None) == C.CCDPP_EINVAL


def test_softmax_refuses_null_pointers_and_workspaces():
    L = _lib_or_skip()
    n = ctypes.c_int64()
    B, E = ctypes.byref, C.CCDPP_EINVAL
    assert L.ccdpp_softmax_workspace(None, 0, B(n)) == E
    assert L.ccdpp_softmax_workspace(B(_problem()), 3, B(n)) == E and "call" in L.ccdpp_ops_last_error().decode()
    assert L.ccdpp_softmax_workspace(B(_problem()), 0, None) == E
    for kw in (dict(x=None), dict(table=None), dict(target=None)):
        assert L.ccdpp_softmax_loss(B(_problem(**kw)), 256, 256, 256, 1 << 40, None) == E
        assert "non-NULL" in L.ccdpp_ops_last_error().decode()
    assert L.ccdpp_softmax_loss(None, 256, 256, 256, 1 << 40, None) == E
    assert L.ccdpp_softmax_loss(B(_problem()), None, 256, 256, 1 << 40, None) == E
    assert L.ccdpp_softmax_loss_grad(B(_problem()), None, None, 256, 8, 256, 8, 256, 1 << 40, None) == E
    assert L.ccdpp_softmax_loss_grad(B(_problem()), 256, None, 256, 7, 256, 8, 256, 1 << 40, None) == E
    assert L.ccdpp_softmax_loss(B(_problem()), 256, 256, 256, 16, None) == E
    assert "too small" in L.ccdpp_ops_last_error().decode()
    assert L.ccdpp_softmax_loss(B(_problem()), 256, 256, None, 1 << 40, None) == E
    assert L.ccdpp_softmax_loss(B(_problem()), 256, 256, 264, 1 << 40, None) == E
    assert "aligned" in L.ccdpp_ops_last_error().decode()


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("t, v, d", [(0, 10, 8), (1, 17_770, 40), (16, 1 << 20, 4096), (17, 1000, 129), (128, 1 << 20, 4096),
                                     (129, 1 << 20, 4096), (8192, 131_072, 4096), (1 << 25, 16_000, 100), (1000, 1, 65536), (1, 1, 1)])
def test_workspace_sizes(t, v, d, dtype):
    """Positive, larger for more work, and far below the logits of large problems."""
    L = _lib_or_skip()
    p = _problem(t=t, v=v, d=d, dtype=dtype, ldx=d, ldt=d)
    got = []
    for call in (ops.LOSS, ops.GRAD, ops.TRAIN):
        n = ctypes.c_int64(-1)
        assert L.ccdpp_softmax_workspace(ctypes.byref(p), call, ctypes.byref(n)) == 0
        got.append(n.value)
    assert 0 <= got[0] <= got[2] and 0 <= got[1] <= got[2]
    operands = 8 * (t + v + 64) * (d + 32) * 4 * 3
    assert got[2] <= operands + 128 * 4 * (v + 64) + (3 << 30) + t * v // 16


def test_gradient_norm_refuses_bad_arguments():
    L = _lib_or_skip()
    n = ctypes.c_int64()
    assert L.ccdpp_grad_norm_workspace(None) == C.CCDPP_EINVAL
    assert L.ccdpp_grad_norm_workspace(ctypes.byref(n)) == 0 and n.value > 0
    ptrs, sizes, dtypes = (ctypes.c_void_p * 1)(256), (ctypes.c_int64 * 1)(4), (ctypes.c_int32 * 1)(0)

    def clip(count=1, ins=ptrs, outs=ptrs, sz=sizes, dt=dtypes, limit=1.0, eps=1e-6, norm=256, ws=256, nb=n.value):
        return L.ccdpp_clip_grads(count, ins, outs, sz, dt, limit, eps, norm, ws, nb, None)

    for kw, msg in ((dict(count=-1), "n must"), (dict(ins=None), "tables"), (dict(outs=None), "tables"), (dict(sz=None), "tables"),
                    (dict(dt=None), "tables"), (dict(norm=None), "norm"), (dict(limit=-1.0), "max_norm"),
                    (dict(limit=math.nan), "max_norm"), (dict(eps=-1.0), "max_norm"), (dict(eps=math.inf), "max_norm"),
                    (dict(ws=None), "workspace"), (dict(ws=260), "workspace"), (dict(nb=n.value - 1), "workspace"),
                    (dict(sz=(ctypes.c_int64 * 1)(-1)), "negative"), (dict(dt=(ctypes.c_int32 * 1)(7)), "dtypes"),
                    (dict(ins=(ctypes.c_void_p * 1)(None)), "NULL"), (dict(ins=(ctypes.c_void_p * 1)(258)), "aligned")):
        assert clip(**kw) == C.CCDPP_EINVAL, kw
        assert msg in L.ccdpp_ops_last_error().decode(), kw


def test_without_a_device_calls_report_edevice():
    L = _lib_or_skip()
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    p = _problem()
    assert L.ccdpp_softmax_loss(ctypes.byref(p), 256, 256, 256, 1 << 40, None) == C.CCDPP_EDEVICE
    assert L.ccdpp_ops_last_error()
    one = (ctypes.c_void_p * 1)(256)
    assert L.ccdpp_grad_norm(1, one, (ctypes.c_int64 * 1)(4), (ctypes.c_int32 * 1)(0), 256, 256, 1 << 20, None) == C.CCDPP_EDEVICE


def test_the_binding_refuses_host_tensors():
    x, e, y = torch.ones(2, 3), torch.ones(4, 3), torch.zeros(2, dtype=torch.int64)
    with pytest.raises(ValueError):
        ops.softmax_loss(x, e, y)
    with pytest.raises(ValueError):
        ops.grad_norm([x])
    with pytest.raises(TypeError):
        ops.softmax_loss(x[0], e, y)
    with pytest.raises(TypeError):
        ops.grad_norm([1.0])
