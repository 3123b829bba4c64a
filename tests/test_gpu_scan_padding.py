"""Padded batches: rows that belong to no sequence are not read, cost less than others, and get zeros."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from seq_util import DT, backward, close, forward, to64

pytestmark = pytest.mark.gpu


def seq():
    from paper_1511_02433_amd import seq as o
    return o


@pytest.mark.parametrize("mode", ["sigmoid", "given"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("lead, rows, behind, d, s", [(5000, 40, 9000, 40, 3), (3, 8, 20_000, 100, 1), (12_345, 2001, 0, 7, 9), (0, 1, 7000, 513, 1), (4096, 1000, 4096, 64, 400),
                                                      (900, 16_384, 16_000, 4096, 2)])
def test_values(lead, rows, behind, d, s, dtype, mode):
    """Against 64 bits on some columns, with NaN in every row of no sequence."""
    rng = np.random.default_rng(lead + rows)
    starts = lead + np.sort(np.concatenate([[0], rng.integers(0, rows + 1, s - 1), [rows]])).astype(np.int64)
    n, gen = lead + rows + behind, torch.Generator(device="cuda").manual_seed(d)

    def make(f=lambda a: a):
        a = f(torch.randn(n, d, generator=gen, device="cuda")).to(DT[dtype])
        a[:lead] = float("nan")
        a[lead + rows:] = float("nan")
        return a

    x, dy, gate = make(), make(), make(lambda a: a * 2 + 2 if mode == "sigmoid" else torch.sigmoid(a * 2 + 2))
    first, dl = (torch.randn(s, d, generator=gen, device="cuda") for _ in range(2))
    at = torch.from_numpy(starts).cuda()
    y, last, kept = seq().gated_scan(x, gate, starts=at, initial=first, mode=mode, keep=True)
    dx, dg, di = seq().gated_scan_grad(x, gate, dy, kept, starts=at, initial=first, mode=mode, dlast=dl)
    for a in (y, dx, dg):
        assert not bool(a[:lead].any()) and not bool(a[lead + rows:].any())
    c = torch.unique(torch.tensor([0, 1, d // 2, d - 1]).clamp(max=d - 1)).cuda()
    inside = slice(lead, lead + rows)
    X, G, D = (to64(a[inside][:, c]) for a in (x, gate, dy))
    I, L, own = to64(first[:, c]), to64(dl[:, c]), starts - lead
    wy, wl, before, ey, el, eb = forward(X, G, own, I, mode)
    close(y[inside][:, c], wy, ey, "y")
    close(last[:, c], wl, el, "last")
    wx, wg, wi, ex, eg, ei = backward(X, G, D, L, own, before, eb, mode)
    close(dx[inside][:, c], wx, ex, "dx")
    close(dg[inside][:, c], wg, eg, "dgate")
    close(di[:, c], wi, ei, "dinitial")


def least_us(call):
    best = float("inf")
    for _ in range(8):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        call()
        a.record()
        for _ in range(3):
            call()
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b) * 1e3 / 3)
    return best


@pytest.mark.parametrize("n, d, dtype", [(65_536, 4096, "bf16"), (400_000, 512, "f32")])
def test_rows_of_no_sequence_cost_their_zeros_alone(n, d, dtype):
    """Values that are not read are seen in the time alone.  Forward a row reads two of its values and writes one, for the gradients it
    reads three and writes two: with nothing read a third and two fifths of the bytes are left, and three quarters of the time is allowed."""
    x, gate, dy = (torch.randn(n, d, device="cuda").to(DT[dtype]) for _ in range(3))
    y, dx, dg = (torch.empty_like(x) for _ in range(3))

    def times(rows):
        at = torch.arange(17, device="cuda") * rows // 16
        _, _, kept = seq().gated_scan(x, gate, starts=at, y=y, keep=True)
        return (least_us(lambda: seq().gated_scan(x, gate, starts=at, y=y)),
                least_us(lambda: seq().gated_scan_grad(x, gate, dy, kept, starts=at, dx=dx, dgate=dg)))

    full, padded = times(n), times(8)
    assert padded[0] < 0.75 * full[0] and padded[1] < 0.75 * full[1], (full, padded)
