"""The example that runs CCD++, the recurrence, dropout, the softmax loss, clipping and beams together: it runs, its gradients are those
of autograd in 64 bits, and its answers are items in descending order of their scores."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "next_items.py")
    spec = importlib.util.spec_from_file_location("next_items", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_it_runs():
    first, last, score, items = example().main(["--users", "800", "--items", "500", "--ratings", "30000", "--k", "16", "--steps", "12", "--batch", "64"])
    assert first == first and last == last
    assert items.shape == (4, 4, 3) and bool(((items >= 0) & (items < 500)).all())
    assert bool((score[:, :-1] >= score[:, 1:]).all()) and bool(torch.isfinite(score).all())


def test_its_gradients():
    """Without dropout, against autograd in 64 bits on the host; within 1e-4 of the largest (the softmax's terms have 22 bits)."""
    import numpy as np

    m = example()
    gen = torch.Generator().manual_seed(3)
    v, d = 90, 12
    H, G = torch.randn(v, d, generator=gen) * 0.5, torch.randn(v, d, generator=gen)
    offset = -torch.rand(v, generator=gen)
    rng = np.random.default_rng(3)
    sequences = [rng.integers(0, v, n) for n in (5, 1, 0, 40, 17)]
    loss, dH, dG = m.gradients(H.cuda(), G.cuda(), offset.cuda(), m.pack(sequences), 0.0, 1)
    H64, G64 = H.double().requires_grad_(), G.double().requires_grad_()
    total, steps = 0.0, 0
    for s in sequences:
        h = torch.zeros(d, dtype=torch.float64)
        for now, then in zip(s[:-1], s[1:]):
            a = torch.sigmoid(G64[now])
            h = a * h + (1 - a) * H64[now]
            z = H64 @ h + offset.double()
            total, steps = total + torch.logsumexp(z, 0) - z[then], steps + 1
    (total / steps).backward()
    assert abs(float(loss) - float(total.detach()) / steps) <= 1e-5 * float(total.detach()) / steps
    for got, want in ((dH, H64.grad), (dG, G64.grad)):
        assert float((got.cpu() - want).abs().max()) <= 1e-4 * float(want.abs().max())
