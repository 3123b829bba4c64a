"""The log sum of long rows: within 2^-17 of the exact one, as include/ccdpp_seq.h has it, whatever order the row has."""
import ctypes
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


def best_of(row, score=0.0):
    """The best continuation's score and item where 768 beams have a share of their row each; all others are none, so theirs is not read."""
    from paper_1511_02433_amd import seq

    v, g, b = row.numel(), 12, 64
    scores = torch.full((g, b), -math.inf, device="cuda")
    scores[0, 0] = score
    p, n, L = seq.Beam(g, v, b, 1, seq._DTYPES[row.dtype], 0, row.data_ptr(), v, scores.data_ptr(), None, None, -1), ctypes.c_int64(), seq._lib()
    assert L.ccdpp_beam_workspace(ctypes.byref(p), ctypes.byref(n)) == 0
    ws = torch.empty(n.value, dtype=torch.uint8, device="cuda")
    out, parent, item = torch.empty(g, 1, device="cuda"), *torch.empty(2, g, 1, dtype=torch.int64, device="cuda").unbind()
    assert L.ccdpp_beam_select(ctypes.byref(p), out.data_ptr(), parent.data_ptr(), item.data_ptr(), None, ws.data_ptr(), n.value, seq._stream(0)) == 0
    torch.cuda.synchronize()
    assert parent[0, 0] == 0 and bool((parent[1:] == -1).all())
    return float(out[0, 0]), int(item[0, 0])


def log_sum(row):
    """Less the greatest value, in 64 bits."""
    top = float(row.max())
    return math.log(sum(float((part.double() - top).exp().sum()) for part in row.split(1 << 24)))


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("v, rise", [(2_000_003, 3.0), (1 << 26, 1.0), ((1 << 28) - 1, 4.0)])
@pytest.mark.parametrize("order", ["up", "down", "steps"])
def test_ordered_rows(order, v, rise, dtype):
    """Rows that rise a little from chunk to chunk ("steps": by 0.7 at a time), or fall."""
    row = torch.arange(v, dtype=torch.float32, device="cuda").mul_(rise / v)
    if order == "down":
        row = row.neg_()
    elif order == "steps":
        row = row.mul_(20 / rise).floor_().mul_(0.7)
    row = row.to(dtype)
    score, item = best_of(row)
    want = -log_sum(row)
    assert float(row[item]) == float(row.max()) and (item == 0 or float(row[item - 1]) < float(row[item]))
    assert abs(score - want) <= 2.0 ** -17 + 2.0 ** -24 * abs(want)
