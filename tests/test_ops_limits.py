"""What the operators' workspaces hold, from the sizes alone (no GPU): bounded whatever the numbers of rows and items are; and which
pointers the calls refuse."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

import paper_1511_02433_amd.ccdpp as C
from paper_1511_02433_amd import ops

MIB = 1 << 20


def _lib_or_skip():
    try:
        return ops._lib()
    except RuntimeError as e:  # not built in this checkout
        pytest.skip(str(e))


def workspace(t, v, d, dtype, call):
    L = _lib_or_skip()
    p = ops.Softmax(t, v, d, dtype, 256, d, 256, d, 256, 64, 1.0, None)
    n = ctypes.c_int64(-1)
    assert L.ccdpp_softmax_workspace(ctypes.byref(p), call, ctypes.byref(n)) == 0
    return n.value


def up(a, b):
    return (a + b - 1) // b * b


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("t, v, d", [(129, 20_000, 200), (4096, 100_000, 300), (1 << 17, 2048, 200), (1 << 20, 17_770, 200), (1 << 21, 131_072, 256),
                                     (1 << 25, 16_000, 200), ((1 << 26) - 1, 8_000, 129), (129, (1 << 28) - 1, 129), (8192, 131_072, 4096)])
def test_wide_products(t, v, d, dtype):
    """The operands in fragment order (rows and columns in blocks of 32), twice for the gradients; 256 MiB of sums of the
    logits (or those of 256 rows); G and G^T of 512 MiB each with their items' powers; 1 GiB of kept logits in training; one
    32-bit dx; partial sums for the CUs that would have no block otherwise (128 MiB); a few numbers per row and item."""
    planes = 2 if dtype == 0 else 1
    rows = up(t, 32) + up(v, 32)
    packed = rows * up(d, 32) * 2 * planes
    numbers = 16 * rows + MIB
    sums = max(256 * MIB, 256 * 8 * up(v, 2048) // 256)
    grads = packed + 2 * 512 * MIB + 16 * MIB + 4 * up(d, 4) * t + 128 * MIB
    assert workspace(t, v, d, dtype, ops.LOSS) <= packed + numbers + sums
    assert workspace(t, v, d, dtype, ops.GRAD) <= packed + numbers + grads
    assert workspace(t, v, d, dtype, ops.TRAIN) <= packed + numbers + sums + grads + 1024 * MIB


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("t, v, d", [(1 << 22, 17_770, 40), (1 << 25, 16_000, 100), (1 << 20, 1000, 128)])
def test_few_factors(t, v, d, dtype):
    """Operands in blocks of 32 rows (x once with and once without its transpose), and no partial sums of a gradient whose
    blocks have one share each, as x has where rows are many; the table's in as many shares as blocks run at once."""
    planes = 2 if dtype == 0 else 1
    steps, blocks = (d + 15) // 16, (d + 31) // 32
    plain, turned = planes * steps + 1, planes * blocks * 2
    tt, vt = (t + 31) // 32, (v + 31) // 32
    packed = 1024 * (tt * (2 * plain + turned) + vt * (plain + turned))
    of_table = 768 * 2 * 128 * 32 * blocks * 4  # (at most two kept blocks of 128 a share)
    assert workspace(t, v, d, dtype, ops.TRAIN) <= packed + 8 * 8 * t + 4 * t + of_table + MIB


@pytest.mark.parametrize("dtype, value", [(0, 4), (1, 2), (2, 2)])
def test_pointers_that_are_not_aligned_to_their_type_are_refused(dtype, value):
    """By the calls, on the host; the workspace's size needs no pointer."""
    L, B, E = _lib_or_skip(), ctypes.byref, C.CCDPP_EINVAL
    fields = dict(t=4, v=10, d=8, dtype=dtype, x=256, ldx=8, table=256, ldt=8, target=256, target_bits=64, scale=1.0, offset=None)

    def problem(**kw):
        return ops.Softmax(*[{**fields, **kw}[n] for n, _ in ops.Softmax._fields_])

    for kw in (dict(x=256 + value // 2), dict(table=256 + value // 2), dict(target=260), dict(target=258, target_bits=32), dict(offset=258)):
        p, n = problem(**kw), ctypes.c_int64()
        assert L.ccdpp_softmax_workspace(B(p), ops.TRAIN, B(n)) == 0
        for rc in (L.ccdpp_softmax_loss(B(p), 256, 256, 256, 1 << 40, None), L.ccdpp_softmax_loss_grad(B(p), 256, None, 256, 8, 256, 8, 256, 1 << 40, None),
                   L.ccdpp_softmax_loss_train(B(p), 256, 256, None, 256, 8, 256, 8, 256, 1 << 40, None)):
            assert rc == E and "aligned to their types" in L.ccdpp_ops_last_error().decode(), kw
    p = problem()
    off = 256 + value // 2
    for args in ((258, 256, None, 256, 256), (256, 258, None, 256, 256), (256, 256, 258, 256, 256), (256, 256, None, off, 256), (256, 256, None, 256, off)):
        loss, lse, grad, dx, de = args
        assert L.ccdpp_softmax_loss_train(B(p), loss, lse, grad, dx, 8, de, 8, 256, 1 << 40, None) == E, args
        assert "aligned to their types" in L.ccdpp_ops_last_error().decode()
    assert L.ccdpp_softmax_loss_grad(B(p), 258, None, 256, 8, 256, 8, 256, 1 << 40, None) == E
    assert "aligned to their types" in L.ccdpp_ops_last_error().decode()
