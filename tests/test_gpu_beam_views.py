"""States that are views whose memory holds other values than they stand for: conjugates, and what is negated when it is read."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


def test_reorder_takes_conjugate_and_negated_views():
    from paper_1511_02433_amd import seq

    gen = torch.Generator().manual_seed(1)
    z = torch.randn(6, 5, generator=gen, dtype=torch.complex64)
    wide = torch.randn(6, 9, generator=gen, dtype=torch.complex64)
    parent = torch.tensor([[2, 0, -1], [1, 1, 0]])
    row = torch.tensor([2, 0, 0, 4, 4, 3])

    def views(device):
        a, b = z.to(device), wide.to(device)
        return [a.conj(), b[:, 2:7].conj(), a[:, 0].conj().imag, a, a.conj().imag.contiguous()]

    host, dev = views("cpu"), views("cuda")
    assert dev[0].is_conj() and dev[1].is_conj() and dev[2].is_neg()
    want = [a[row].clone().resolve_conj().resolve_neg() for a in host]
    for a in want:
        a[2] = 0
    got = seq.beam_reorder(parent.cuda(), dev, beams=3)
    out = [torch.ones_like(a) for a in got]
    seq.beam_reorder(parent.cuda(), dev, beams=3, out=out)
    for a, b, c in zip(want, got, out):
        assert torch.equal(a, b.cpu()) and torch.equal(a, c.cpu())
    assert dev[0].is_conj()  # the caller's are as they were
    with pytest.raises(ValueError):
        seq.beam_reorder(parent.cuda(), [dev[3]], beams=3, out=[torch.zeros(6, 5, dtype=torch.complex64, device="cuda").conj()])
