"""What the recurrence's gradients refuse once a device is there."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


def test_gradients_of_states_in_place_are_refused():
    import paper_1511_02433_amd.ccdpp as C
    from paper_1511_02433_amd import seq

    L, n, d = seq._lib(), 6, 4
    x, gate, dy, dx, dgate = (torch.randn(n, d, device="cuda") for _ in range(5))
    starts, initial, dlast = torch.tensor([0, 2, 6], device="cuda"), torch.randn(2, d, device="cuda"), torch.randn(2, d, device="cuda")
    _, _, kept = seq.gated_scan(x, gate, starts=starts, initial=initial, keep=True)
    p = seq.Scan(n, 2, d, 0, 1, 64, x.data_ptr(), d, gate.data_ptr(), d, starts.data_ptr(), initial.data_ptr())
    ws, was = torch.empty(1 << 20, dtype=torch.uint8, device="cuda"), dlast.clone()
    rc = L.ccdpp_gated_scan_grad(ctypes.byref(p), dy.data_ptr(), d, dlast.data_ptr(), kept.data_ptr(), dx.data_ptr(), d, dgate.data_ptr(), d, dlast.data_ptr(),
                                 ws.data_ptr(), 1 << 20, seq._stream(0))
    assert rc == C.CCDPP_EINVAL and "dinitial must not be dlast" in L.ccdpp_ops_last_error().decode()
    torch.cuda.synchronize()
    assert torch.equal(dlast, was)
