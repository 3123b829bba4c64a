"""Clipping gradients that start anywhere and whose dimensions lie in another order, value by value against float64.

Tolerances as in test_gpu_grad_clip.py: the norm is rounded once, the factor's division and product round twice more in 32
bits; 16-bit results round once more."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TOL = {torch.float32: 4 * 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -10}


def ops():
    from paper_1511_02433_amd import ops as o
    return o


def layouts(dtype, many, seed=0):
    """(memory, tensors that are views of it): one starting past its first value, two with their dimensions in another order."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(DT[dtype])  # noqa: E731
    base = new(10_007 * many)
    return base, [base[1:-1], new(30, 50 * many).t(), new(4, 5, 6 * many).permute(2, 0, 1), new(3)[2:]]


def check(got, before, limit):
    norm = math.sqrt(sum(float((b.double() ** 2).sum()) for b in before))
    c = min(1.0, limit / (norm + 1e-6))
    for a, b in zip(got, before):
        w = b.double() * c
        slack = 2.0 ** -25 if a.dtype == torch.float16 else 0.0
        assert bool(((a.double() - w).abs() <= TOL[a.dtype] * w.abs() + slack).all())


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("many", [1, 40])  # one launch of one block; two launches
def test_in_place(dtype, many):
    base, ts = layouts(dtype, many)
    before, ends = [a.clone() for a in ts], (float(base[0]), float(base[-1]))
    limit = math.sqrt(sum(float((b.double() ** 2).sum()) for b in before)) / 2
    norm = ops().clip_grads(ts, limit)
    assert abs(float(norm) - 2 * limit) <= 2e-7 * 2 * limit
    check(ts, before, limit)
    assert (float(base[0]), float(base[-1])) == ends


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("many", [1, 40])
def test_into_others_of_the_same_strides(dtype, many):
    _, ts = layouts(dtype, many, seed=1)
    before = [a.clone() for a in ts]
    out = [torch.full_like(a, 7.0) for a in ts]
    assert [o.stride() for o in out] == [a.stride() for a in ts]
    ops().clip_grads(ts, 1.5, out=out)
    check(out, before, 1.5)
    assert all(torch.equal(a, b) for a, b in zip(ts, before))


def test_others_of_other_strides_are_refused():
    _, ts = layouts("f32", 1)
    with pytest.raises(ValueError):
        ops().clip_grads(ts, 1.0, out=[torch.empty(a.shape, device="cuda") for a in ts])
    with pytest.raises(ValueError):
        ops().clip_grads([ts[1][::2]], 1.0)
    with pytest.raises(ValueError):
        ops().grad_norm([torch.randn(3, 1, device="cuda").expand(3, 4)])
