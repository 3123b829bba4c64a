"""The softmax loss far from where its numbers are easy: logits that are all low, finite masks, values and weights of very
different sizes, items and rows that hardly count.  Compared with plain float64 torch on the GPU, row by row and item by item.

Tolerances.  A logit and a log-sum-exp z have 32 bits: 5e-7 (1 + |z|) each, Z the largest |z| of what is not masked, so a loss
is within 1e-6 (1 + Z) and a probability within that relative to itself."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def ops():
    from paper_1511_02433_amd import ops as o
    return o


def make(t, v, d, dtype, seed=0, spread=2.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(t, d, generator=gen, device="cuda").to(DT[dtype])
    e = (torch.randn(v, d, generator=gen, device="cuda") * (spread / math.sqrt(d))).to(DT[dtype])
    y = torch.randint(0, v, (t,), generator=gen, device="cuda")
    return x, e, y


def logits(x, e, scale=1.0, offset=None):
    z = scale * torch.mm(x.double(), e.double().t())
    return z if offset is None else z + offset.double()


def check_loss(x, e, y, loss, lse, offset=None, masked=None):
    z = logits(x, e, 1.0, offset)
    want = torch.logsumexp(z, dim=1)
    rows = torch.arange(len(y), device="cuda")
    size = z if masked is None else z[:, ~masked]
    tol = 1e-6 * (1 + float(size.abs().max()))
    assert float((lse.double() - want).abs().max()) <= tol
    assert float((loss.double() - (want - z[rows, y])).abs().max()) <= tol
    return z, want


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("t", [32, 33, 200])
@pytest.mark.parametrize("d", [8, 40, 128, 136])
@pytest.mark.parametrize("shift", [-85.0, -100.0, -1000.0, 500.0])
def test_a_shift_of_all_logits(t, d, shift, dtype):
    x, e, y = make(t, 1000, d, dtype, seed=d)
    offset = torch.full((1000,), shift, device="cuda")
    loss, lse, dx, de = ops().softmax_loss_train(x, e, y, offset=offset)
    z, want = check_loss(x, e, y, loss, lse, offset)
    g = torch.exp(z - want[:, None])
    g[torch.arange(t, device="cuda"), y] -= 1
    tol = {"f32": 2e-5, "bf16": 1e-2, "f16": 2e-3}[dtype] + 1e-6 * (1 + abs(shift))
    for a, b in ((dx, torch.mm(g, e.double())), (de, torch.mm(g.t().contiguous(), x.double()))):
        assert float((a.double() - b).norm()) <= tol * float(b.norm())


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("t", [32, 33, 200])
@pytest.mark.parametrize("d", [8, 40, 128, 136])
@pytest.mark.parametrize("mask", [-300.0, -1e4, -65504.0, -1e6, -1e9])
@pytest.mark.parametrize("first,last", [(0, 32), (0, 64), (128, 160), (480, 640)])
def test_finite_masks(t, d, mask, first, last, dtype):
    """Masks over whole tiles of 32 items, where a share of the table begins among them."""
    x, e, y = make(t, 1000, d, dtype, seed=d)
    offset = torch.zeros(1000, device="cuda")
    offset[first:last] = mask
    masked = offset < 0
    y = torch.where(masked[y], torch.full_like(y, 700), y)
    loss, lse = ops().softmax_loss(x, e, y, offset=offset)
    check_loss(x, e, y, loss, lse, offset, masked)
    l2, s2, dx, de = ops().softmax_loss_train(x, e, y, offset=offset)
    assert torch.equal(loss, l2) and torch.equal(lse, s2)
    assert bool(torch.isfinite(dx).all()) and float(de[masked].float().abs().max()) == 0.0


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("t,d", [(40, 40), (300, 100)])
def test_a_distance_softmax(t, d, dtype):
    """offset = -|e|^2 / 2: every logit of rows near none of the items is low."""
    x, e, y = make(t, 3000, d, dtype, seed=t, spread=30.0)
    x = (x.float() * 0.1).to(DT[dtype])
    offset = -0.5 * e.float().square().sum(1)
    loss, lse = ops().softmax_loss(x, e, y, offset=offset)
    check_loss(x, e, y, loss, lse, offset)


SIZES32 = [(32, 1000, 40), (33, 1000, 40), (200, 1000, 128), (100, 700, 200), (200, 1000, 512), (400, 20_000, 160)]


def grads64(x, e, y, z, lse, g, scale=1.0):
    """(G, dx, dtable) in 64 bits."""
    p = torch.exp(z - lse[:, None])
    p[torch.arange(len(y), device="cuda"), y] -= 1
    p = p * (g.double() * scale)[:, None]
    return p, torch.mm(p, e.double()), torch.mm(p.t().contiguous(), x.double())


@pytest.mark.parametrize("t,v,d", SIZES32)
@pytest.mark.parametrize("size", [30.0, 1e3, 1e4])
@pytest.mark.parametrize("where", ["an item", "a column of the table", "a whole item", "a row of x"])
def test_one_large_value_costs_the_others_nothing(t, v, d, size, where):
    """32-bit values; the other side holds zeros where the large ones are, so that no logit is large.  The planes hold 22 bits
    of each value down to 2^-17 of its row's largest (1e4 is 2^13 here), so the tolerance is that of plain inputs."""
    x, e, y = make(t, v, d, "f32", seed=d)
    if where == "a row of x":
        e[:, 3] = 0
        x[5, 3] = size
    else:
        x[:, 3] = 0
        if where == "an item":
            e[v // 2, 3] = size
        elif where == "a column of the table":
            e[:, 3] *= size
        else:
            x[:, ::2] = 0
            e[v // 2, ::2] *= size
    loss, lse, dx, de = ops().softmax_loss_train(x, e, y)
    z, want = check_loss(x, e, y, loss, lse)
    g, wx, we = grads64(x, e, y, z, want, torch.ones(t, device="cuda"))
    cols = [c for c in range(d) if c != 3] if where != "a whole item" else list(range(1, d, 2))
    # 2e-5 as for plain inputs, of the terms' sum where they cancel
    assert float((dx.double() - wx)[:, cols].norm()) <= 2e-5 * float(wx[:, cols].norm())
    assert float((de.double() - we)[:, cols].norm()) <= 2e-5 * float(we[:, cols].norm())


@pytest.mark.parametrize("t,v,d", SIZES32)
def test_items_and_rows_of_very_different_sizes(t, v, d):
    """Items and rows over eight powers of ten, their products still within 32 bits' reach: the small ones' logits are as near
    to their own size as the large ones'."""
    x, e, y = make(t, v, d, "f32", seed=d + 1)
    e *= torch.logspace(-8, 0, v, device="cuda")[torch.randperm(v, device="cuda", generator=torch.Generator("cuda").manual_seed(3))][:, None]
    x *= torch.logspace(-4, 0, t, device="cuda")[:, None]
    loss, lse = ops().softmax_loss(x, e, y)
    check_loss(x, e, y, loss, lse)
    big = x * 1e6
    small = e * 1e-6
    loss, lse = ops().softmax_loss(big, small, y)
    check_loss(big, small, y, loss, lse)


def check_rows(got, want, terms, dtype, z):
    """Each row of a gradient against its own size.  got_v = sum_t G_tv x_t: every term has the probability's relative error,
    1e-6 (1 + z), and that of its representation, 2^-20 (two planes) or 2^-11 (one); what is compared with is the 2-norm of
    `terms`, sum_t |G_tv| |x_t|, as terms may cancel.  The result is rounded once, by 2^-24, 2^-8 or 2^-11 of
    itself (half precision: 2^-25 at least)."""
    tol = {"f32": 2.0 ** -20, "bf16": 2.0 ** -11, "f16": 2.0 ** -11}[dtype] + 1e-6 * (1 + z)
    once = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}[dtype]
    floor = 2.0 ** -25 * math.sqrt(got.shape[1]) if dtype == "f16" else 1e-38
    off = (got.double() - want).norm(dim=1) - (tol * terms.norm(dim=1) + once * want.norm(dim=1) + floor)
    assert float(off.max()) <= 0.0, (int(off.argmax()), float(((got.double() - want).norm(dim=1) / terms.norm(dim=1)).nan_to_num().max()))


# rows, items, factors: few rows; few factors; logits from the table as it lies; contractions that are cut; products in tiles,
# logits kept or not; more rows than one group of terms
ROWS = [(8, 600, 40), (20, 600, 200), (33, 600, 40), (300, 600, 128), (500, 5000, 17), (40, 600, 200), (100, 600, 136), (200, 600, 200),
        (300, 20_000, 160), (300, 15_000, 400), (2100, 3000, 136)]


def rare_items(t, v, d, dtype, offsets, seed):
    x, e, y = make(t, v, d, dtype, seed=seed)
    offset = torch.zeros(v, device="cuda")
    which = torch.arange(3, v, 11, device="cuda")
    offset[which] = torch.tensor(offsets, device="cuda")[torch.arange(len(which), device="cuda") % len(offsets)]
    y = torch.where(offset[y] < 0, (y + 1) % v, y)
    assert not bool((offset[y] < 0).any())
    return x, e, y, offset


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("t,v,d", ROWS)
def test_items_that_are_unlikely_for_every_row(t, v, d, dtype):
    """An item's gradient is as near to its own size as a popular one's: rare tokens are learned from it and nothing else."""
    offsets = [-4.0, -8.0, -14.0] if dtype == "f16" else [-4.0, -8.0, -12.0, -16.0, -20.0, -30.0, -60.0]
    x, e, y, offset = rare_items(t, v, d, dtype, offsets, seed=t)
    g = torch.full((t,), 2000.0 if dtype == "f16" else 1.0, device="cuda")
    loss, lse, dx, de = ops().softmax_loss_train(x, e, y, grad=g, offset=offset)
    z, want = check_loss(x, e, y, loss, lse, offset)
    p, wx, we = grads64(x, e, y, z, want, g)
    size = float(z.abs().max())
    check_rows(de, we, torch.mm(p.abs().t().contiguous(), x.double().abs()), dtype, size)
    check_rows(dx, wx, torch.mm(p.abs(), e.double().abs()), dtype, size)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("t,v,d", ROWS)
@pytest.mark.parametrize("negative", [False, True])
def test_weights_of_very_different_sizes(t, v, d, dtype, negative):
    """Seven powers of ten (half precision: six): every row's dx by its own weight, every item's gradient by its rows'."""
    x, e, y, offset = rare_items(t, v, d, dtype, [-3.0, -10.0], seed=t + 1)
    gen = torch.Generator(device="cuda").manual_seed(t)
    g = 10.0 ** (torch.rand(t, generator=gen, device="cuda") * (6 if dtype == "f16" else 7) - (3 if dtype == "f16" else 7))
    if negative:
        g[::3] *= -1
        g[1] = 0
    loss, lse, dx, de = ops().softmax_loss_train(x, e, y, grad=g, offset=offset)
    z, want = check_loss(x, e, y, loss, lse, offset)
    p, wx, we = grads64(x, e, y, z, want, g)
    size = float(z.abs().max())
    check_rows(dx, wx, torch.mm(p.abs(), e.double().abs()), dtype, size)
    check_rows(de, we, torch.mm(p.abs().t().contiguous(), x.double().abs()), dtype, size)


@pytest.mark.parametrize("t,v,d", [(8, 20_000, 40), (20, 20_000, 100), (31, 3000, 72), (40, 20_000, 40), (100, 20_000, 136), (300, 20_000, 136)])
def test_half_precision_weights_up_to_the_types_range(t, v, d):
    """From 10^-3 to 3 10^4: the largest gradients are near half precision's end, the smallest still far above its beginning."""
    x, e, y = make(t, v, d, "f32", seed=t)
    x, e = (x * 0.25).half(), (e * 4).half()
    gen = torch.Generator(device="cuda").manual_seed(t)
    g = 10.0 ** (torch.rand(t, generator=gen, device="cuda") * 7.5 - 3)
    g[0], g[1] = 3e4, 1e-3
    y[0] = 7
    y[1:] = torch.where(y[1:] == 7, torch.full_like(y[1:], 8), y[1:])
    loss, lse, dx, de = ops().softmax_loss_train(x, e, y, grad=g)
    z, want = check_loss(x, e, y, loss, lse)
    p, wx, we = grads64(x, e, y, z, want, g)
    size = float(z.abs().max())
    for got, w, terms in ((dx, wx, torch.mm(p.abs(), e.double().abs())), (de, we, torch.mm(p.abs().t().contiguous(), x.double().abs()))):
        fits = w.abs().amax(dim=1) < 6e4
        assert int(fits.sum()) >= len(fits) - 2
        check_rows(got[fits], w[fits], terms[fits], "f16", size)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("t,v,d", [(1, 300, 40), (20, 300, 40), (32, 300, 200), (33, 300, 40), (40, 300, 200), (150, 300, 200)])
def test_an_infinite_lse_leaves_the_targets_part(t, v, d, dtype):
    """From the definition: every probability is 0, and G is -1 at the target, whatever the number of rows: dx is the target's
    item, 16-bit values as they are, 32-bit ones with 22 bits."""
    x, e, y = make(t, v, d, dtype, seed=t)
    lse = torch.logsumexp(logits(x, e), dim=1).float()
    lse[0] = math.inf
    y[-1] = 3 if t == 1 else -1
    dx, de = ops().softmax_loss_grad(x, e, y, lse)
    assert float((dx[0] + e[y[0]]).abs().max()) <= (2.0 ** -21 if dtype == "f32" else 0.0) * float(e[y[0]].abs().max())
    assert t == 1 or float(dx[-1].float().abs().max()) == 0.0
    p = torch.exp(logits(x, e) - lse.double()[:, None])
    p[torch.arange(t, device="cuda"), y.clamp(min=0)] -= 1
    p[y < 0] = 0
    want = torch.mm(p.t().contiguous(), x.double())
    assert float((de.double() - want).norm()) <= {"f32": 2e-5, "bf16": 1e-2, "f16": 2e-3}[dtype] * float(want.norm())
