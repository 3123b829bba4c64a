"""What torch's autograd sees of the operators: tensors that they write to have another version, so that a backward pass
that needs their old values says so."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


def ops():
    from paper_1511_02433_amd import ops as o
    return o


def test_clipping_raises_the_version_of_what_it_writes():
    a, b = torch.randn(100, device="cuda"), torch.randn(7, 5, device="cuda")
    was = a._version, b._version
    out = [torch.empty_like(a), torch.empty_like(b)]
    ops().clip_grads([a, b], 1.0, out=out)
    assert (a._version, b._version) == was and out[0]._version == out[1]._version == 1
    ops().grad_norm([a, b])
    assert (a._version, b._version) == was
    ops().clip_grads((t for t in (a, b)), 1.0)
    assert (a._version, b._version) == (was[0] + 1, was[1] + 1)
    w = torch.randn(100, device="cuda", requires_grad=True)
    s = (a * w).sum()  # keeps a for the backward pass
    ops().clip_grads([a[10:20]], 1e-3)  # a part of it
    with pytest.raises(RuntimeError, match="inplace"):
        s.backward()
    with torch.inference_mode():
        g = torch.randn(10, device="cuda")
        ops().clip_grads([g], 1e-3)
    assert float(g.norm()) <= 1.1e-3


def test_given_gradients_have_another_version():
    x, e = torch.randn(4, 8, device="cuda"), torch.randn(10, 8, device="cuda")
    y = torch.randint(0, 10, (4,), device="cuda")
    dx, de = torch.empty_like(x), torch.empty_like(e)
    _, lse, got, _ = ops().softmax_loss_train(x, e, y, dx=dx)
    assert got is dx and (dx._version, de._version) == (1, 0)
    ops().softmax_loss_grad(x, e, y, lse, dx=dx, dtable=de)
    assert (dx._version, de._version) == (2, 1)
    assert (x._version, e._version, y._version, lse._version) == (0, 0, 0, 0)
