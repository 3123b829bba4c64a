"""The softmax loss where its ways of computing meet: few rows straight from the table, few factors, products in pieces,
products whose contraction is cut, long tables.  Compared with plain float64 torch on the GPU.

Tolerances as in test_gpu_softmax_loss.py: logits to 1e-5 (1 + max |z|); gradients, relative in the 2-norm, to 2e-5 (float32),
2^-8 (bfloat16) and 2e-3 (float16), one rounding of the result and of half-precision terms included, plus what the
probabilities' own error leaves where they cancel against the target: a logit and its lse in 32 bits differ by 4 roundings,
5e-7 (1 + max |z|) in all, times the norm of the gradients' first part, sum_v g p e (for one item the gradient is zero and
that is all there is)."""
import math
import random

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
GTOL = {"f32": 2e-5, "bf16": 2.0 ** -8, "f16": 2e-3}


def ops():
    from paper_1511_02433_amd import ops as o
    return o


def make(t, v, d, dtype, seed=0, spread=2.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(t, d, generator=gen, device="cuda").to(DT[dtype])
    e = (torch.randn(v, d, generator=gen, device="cuda") * (spread / math.sqrt(d))).to(DT[dtype])
    y = torch.randint(0, v, (t,), generator=gen, device="cuda")
    g = torch.rand(t, generator=gen, device="cuda") + 0.5
    return x, e, y, g


def plain(x, e, y, g, scale=1.0, offset=None, rows=1 << 26):
    """(loss, lse, dx, de) in 64 bits, a block of rows after another."""
    x, e, g = x.double(), e.double(), g.double()
    t, v = x.shape[0], e.shape[0]
    loss, lse = torch.zeros(t, dtype=torch.float64, device="cuda"), torch.zeros(t, dtype=torch.float64, device="cuda")
    dx, de = torch.zeros_like(x), torch.zeros_like(e)
    first = [torch.zeros_like(x), torch.zeros_like(e)]
    step = max(1, rows // v)
    for a in range(0, t, step):
        b = min(t, a + step)
        z = scale * torch.mm(x[a:b], e.t())
        if offset is not None:
            z = z + offset.double()
        l = torch.logsumexp(z, dim=1)
        lse[a:b] = l
        at = torch.arange(b - a, device="cuda")
        live = y[a:b] >= 0
        k = y[a:b].clamp(min=0)
        loss[a:b] = torch.where(live, l - z[at, k], torch.zeros_like(l))
        w = (torch.where(live, g[a:b], torch.zeros_like(l)) * scale)[:, None]
        p = torch.exp(z - l[:, None])
        first[0][a:b] = torch.mm(p * w, e)
        first[1] += torch.mm((p * w).t().contiguous(), x[a:b])
        p[at, k] -= 1
        p = p * w
        dx[a:b] = torch.mm(p, e)
        de += torch.mm(p.t().contiguous(), x[a:b])
    return loss, lse, dx, de, float(first[0].norm()), float(first[1].norm())


def check(got, want, dtype):
    for a, b in zip(got[:2], want[:2]):
        assert float((a.double() - b).abs().max()) <= 1e-5 * (1 + float(want[1].abs().max()))
    slack = 5e-7 * (1 + float(want[1].abs().max()))
    for a, b, n in zip(got[2:], want[2:4], want[4:]):
        assert float((a.double() - b).norm()) <= GTOL[dtype] * float(b.norm()) + slack * n


def both(t, v, d, dtype, seed=0, **kw):
    x, e, y, g = make(t, v, d, dtype, seed, kw.pop("spread", 2.0))
    if t > 3:
        y[t // 2] = -1
    got = ops().softmax_loss_train(x, e, y, grad=g, **kw)
    check(got, plain(x, e, y, g, **kw), dtype)
    return x, e, y, g, got


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("t", [1, 2, 15, 16, 17, 31, 32, 33, 64, 65, 127, 128, 129, 160])
@pytest.mark.parametrize("v,d", [(500, 130), (1033, 517)])
def test_rows_around_the_limits(t, v, d, dtype):
    both(t, v, d, dtype, seed=t)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("d", [1, 15, 16, 17, 32, 33, 48, 49, 64, 65, 96, 97, 112, 128, 129, 144])
def test_factors_around_the_limits(d, dtype):
    both(70, 700, d, dtype, seed=d)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("v", [1, 2, 15, 16, 31, 32, 33, 127, 128, 129, 255, 256, 257])
@pytest.mark.parametrize("t,d", [(5, 40), (40, 40), (20, 200), (140, 200)])
def test_short_tables(t, v, d, dtype):
    both(t, v, d, dtype, seed=v)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("t,v,d", [(3, 900, 4099), (100, 900, 3000), (200, 700, 3001), (300, 3000, 1000), (5, 40_000, 300),
                                   (70, 40_000, 200)])
def test_long_rows_and_tables(t, v, d, dtype):
    """Columns shared by waves, rows of x brought by columns, contractions that are cut, waves of two groups."""
    both(t, v, d, dtype, seed=d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pieces_of_wide_tables_join(dtype):
    """More than one piece of G: 8192 rows, 32,768 (16,384) table entries a piece."""
    both(8192, 36_000, 136, dtype, seed=1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_rows_of_few_factors(dtype):
    both(5000, 9000, 24, dtype, seed=2)


@pytest.mark.parametrize("t,d,dtype", [(3, 2048, "bf16"), (200, 2048, "bf16"), (150, 100, "f32")])
def test_offsets_past_32_bits(t, d, dtype):
    """A table (or its operands) of more than 4 GiB; targets at its end."""
    v = (5 << 30) // (2 * d) if dtype == "bf16" else (5 << 30) // (12 * d)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(t, d, generator=gen, device="cuda").to(DT[dtype])
    e = torch.empty(v, d, dtype=DT[dtype], device="cuda").normal_(0, 2 / math.sqrt(d), generator=gen)
    y = v - 1 - torch.randint(0, 1000, (t,), generator=gen, device="cuda")
    loss, lse, dx, de = ops().softmax_loss_train(x, e, y)
    sums, top = torch.zeros(t, dtype=torch.float64, device="cuda"), 20.0
    want_dx = torch.zeros(t, d, dtype=torch.float64, device="cuda")
    for a in range(0, v, 1 << 18):
        z = torch.mm(x.float(), e[a:a + (1 << 18)].float().t()).double()
        sums += torch.exp(z - top).sum(1)
        want_dx += torch.mm(torch.exp(z - lse.double()[:, None]).float(), e[a:a + (1 << 18)].float()).double()
    want = top + torch.log(sums)
    assert float((lse.double() - want).abs().max()) <= 1e-4
    want_dx -= e[y].double()
    assert float((dx.double() - want_dx).norm()) <= 2 * GTOL[dtype] * float(want_dx.norm())
    last = slice(v - 1000, v)
    p = torch.exp(torch.mm(x.float(), e[last].float().t()).double() - lse.double()[:, None])
    p[torch.arange(t, device="cuda"), y - (v - 1000)] -= 1
    want_de = torch.mm(p.t().contiguous(), x.double())
    assert float((de[last].double() - want_de).norm()) <= 2 * GTOL[dtype] * float(want_de.norm())


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("t,v,d", [(9, 300, 40), (50, 300, 40), (50, 300, 200), (150, 600, 200)])
def test_weights_of_either_sign_and_zero(t, v, d, dtype):
    x, e, y, g = make(t, v, d, dtype, seed=3)
    g[::2] *= -1
    g[3] = 0
    got = ops().softmax_loss_train(x, e, y, grad=g)
    check(got, plain(x, e, y, g), dtype)
    assert float(got[2][3].float().abs().max()) == 0


@pytest.mark.parametrize("t,v,d", [(3, 300, 40), (70, 300, 40), (70, 300, 200), (150, 600, 200)])
def test_logits_beyond_half_precision(t, v, d):
    """Logits of 10^5 and more; rows whose largest value is in proportion, others that are not."""
    x, e, y, g = make(t, v, d, "f32", seed=4, spread=2e5)
    x[1] *= 1e-6
    got = ops().softmax_loss_train(x, e, y, grad=g)
    want = plain(x, e, y, g)
    for a, b in zip(got[:2], want[:2]):
        assert float((a.double() - b).abs().max()) <= 1e-5 * (1 + float(want[1].abs().max()))
    # a probability is as near as a logit and an lse of this size are in 32 bits (see above)
    slack = 5e-7 * (1 + float(want[1].abs().max()))
    for a, b, n in zip(got[2:], want[2:4], want[4:]):
        assert float((a.double() - b).norm()) <= 2e-5 * float(b.norm()) + slack * n


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("t,v,d", [(20, 500, 150), (140, 500, 150), (600, 500, 150)])
def test_one_gradient_at_a_time(t, v, d, dtype):
    x, e, y, g = make(t, v, d, dtype, seed=5)
    want = ops().softmax_loss_train(x, e, y, grad=g)
    a = ops().softmax_loss_grad(x, e, y, want[1], grad=g, need=("x",))
    b = ops().softmax_loss_grad(x, e, y, want[1], grad=g, need=("table",))
    assert a[1] is None and b[0] is None
    assert torch.equal(a[0], want[2]) and torch.equal(b[1], want[3])
    assert ops().softmax_loss_grad(x, e, y, want[1], grad=g, need=()) == (None, None)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("t,v,d,pad", [(140, 300, 136, 3), (140, 300, 135, 0), (4, 40, 9, 0), (70, 333, 131, 1)])
def test_rows_apart_and_ends_of_memory(t, v, d, pad, dtype):
    """Rows that start anywhere; the last one ends where its memory does."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    bx = torch.full((t * (d + pad) - pad + 1,), math.nan, device="cuda").to(DT[dtype])
    be = torch.full((v * (d + pad) - pad + 1,), math.nan, device="cuda").to(DT[dtype])
    x, e = bx[1:].as_strided((t, d), (d + pad, 1)), be[1:].as_strided((v, d), (d + pad, 1))
    x.copy_(torch.randn(t, d, generator=gen, device="cuda"))
    e.copy_(torch.randn(v, d, generator=gen, device="cuda") * 0.2)
    y = torch.randint(0, v, (t,), generator=gen, device="cuda")
    g = torch.ones(t, device="cuda")
    sx, se = torch.zeros_like(bx), torch.zeros_like(be)
    dx, de = sx[1:].as_strided((t, d), (d + pad, 1)), se[1:].as_strided((v, d), (d + pad, 1))
    check(ops().softmax_loss_train(x, e, y, grad=g, dx=dx, dtable=de), plain(x, e, y, g), dtype)
    dx.zero_(), de.zero_()
    assert float(sx.float().abs().max()) == 0 and float(se.float().abs().max()) == 0


@pytest.mark.parametrize("seed", range(24))
def test_drawn_sizes(seed):
    r = random.Random(seed)
    t = int(math.exp(r.uniform(0, math.log(600))))
    d = int(math.exp(r.uniform(0, math.log(600))))
    v = int(math.exp(r.uniform(0, math.log(6000))))
    dtype = r.choice(list(DT))
    offset = None
    x, e, y, g = make(t, v, d, dtype, seed)
    if r.random() < 0.5:
        offset = torch.randn(v, device="cuda")
        if v > 4:
            drop = torch.rand(v, device="cuda") < 0.2
            drop[y] = False
            offset[drop] = -math.inf
    got = ops().softmax_loss_train(x, e, y, grad=g, offset=offset, scale=r.choice([1.0, 0.3, -0.8]))
    # (the scale of the call, again)
    r = random.Random(seed)
    [r.uniform(0, 1) for _ in range(3)], r.choice(list(DT)), r.random()
    scale = r.choice([1.0, 0.3, -0.8])
    check(got, plain(x, e, y, g, scale, offset), dtype)
    again = ops().softmax_loss_train(x, e, y, grad=g, offset=offset, scale=scale)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("t,v,d,dtype", [(5, 3000, 300, "bf16"), (60, 3000, 300, "bf16"), (200, 1000, 2000, "f32"), (300, 9000, 200, "f16")])
def test_graphs_of_other_ways_replay(t, v, d, dtype):
    x, e, y, g = make(t, v, d, dtype, seed=7)
    want = [a.clone() for a in ops().softmax_loss_train(x, e, y, grad=g)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        ops().softmax_loss_train(x, e, y, grad=g)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = ops().softmax_loss_train(x, e, y, grad=g)
        norm = ops().clip_grads([got[2], got[3]], math.inf)
    for k in range(3):
        for a in got:
            a.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k
        assert bool(torch.isfinite(norm))
        _ = (x.float() @ x.float().t()).sum().item()


@pytest.mark.parametrize("t,v,d,dtype", [(300, 40_001, 400, "f32"), (33, 290_000, 390, "f16"), (1500, 9_999, 1030, "bf16"), (1500, 9_999, 1030, "f16"),
                                         (8300, 33_100, 388, "f32")])
def test_logits_kept_for_the_gradients(t, v, d, dtype):
    """All of them, or those of the first pieces (8,300 rows of 32 bits: 16,128 entries a piece, two pieces).  They are the
    logits that a call of its own computes again, so the gradients are the same, bit for bit."""
    x, e, y, g = make(t, v, d, dtype, seed=d)
    offset = torch.zeros(v, device="cuda")
    offset[::7] = -0.5
    offset[1::1001] = float("-inf")
    y[t // 2] = -1
    y[3] = 1  # excluded
    loss, lse, dx, de = ops().softmax_loss_train(x, e, y, grad=g, offset=offset)
    l2, s2 = ops().softmax_loss(x, e, y, offset=offset)
    dx2, de2 = ops().softmax_loss_grad(x, e, y, lse, grad=g, offset=offset)
    assert torch.equal(loss, l2) and torch.equal(lse, s2) and torch.equal(dx, dx2) and torch.equal(de, de2)
    only = ops().softmax_loss_train(x, e, y, grad=g, offset=offset, need=("table",))
    assert only[2] is None and torch.equal(only[3], de)
    without = (y >= 0) & torch.isinf(offset[y.clamp(min=0)])  # rows whose target is excluded: the plain form ignores them
    assert bool(without[3]) and bool(torch.isposinf(loss[without]).all())
    assert float(dx[without].abs().max()) == 0 and float(de[1::1001].abs().max()) == 0
    keep = torch.where(without, torch.full_like(y, -1), y)
    loss = torch.where(without, torch.zeros_like(loss), loss)
    check((loss, lse, dx, de), plain(x, e, keep, g, offset=offset), dtype)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("t,v,d", [(17, 700, 33), (25, 701, 333), (32, 1999, 130), (31, 5, 9)])
def test_two_groups_of_few_rows(t, v, d, dtype):
    """Rows in both groups of 16 that are ignored, excluded or hold NaN, weights of either sign, int32 targets, rows apart."""
    x, e, y, g = make(t, v, d, dtype, seed=t)
    y[y == 1] = 0
    offset = torch.zeros(v, device="cuda")
    offset[::3] = -1.25
    offset[1] = float("-inf")
    g[::2] *= -1
    g[5] = 0
    y[2], y[t - 1] = -1, 1
    wide = torch.full((t, d + 3), float("nan"), device="cuda", dtype=DT[dtype])
    wide[:, 2:d + 2] = x
    x1 = wide[:, 2:d + 2]
    x1[2] = float("nan")
    e1 = e.clone()
    e1[1] = float("inf")
    loss, lse, dx, de = ops().softmax_loss_train(x1, e1, y.int(), grad=g, offset=offset)
    assert float(loss[2]) == 0 and float(loss[t - 1]) == float("inf")
    assert float(dx[2].abs().max()) == 0 and float(dx[t - 1].abs().max()) == 0 and float(de[1].abs().max()) == 0
    l2, s2 = ops().softmax_loss(x1, e1, y, offset=offset)
    dx2, de2 = ops().softmax_loss_grad(x1, e1, y, lse, grad=g, offset=offset)
    assert torch.equal(loss, l2) and torch.equal(dx, dx2) and torch.equal(de, de2)
    ex, ee = x.clone(), e.clone()
    ex[2], ee[1] = 0, 0
    keep = y.clone()
    keep[t - 1] = -1
    want = plain(ex, ee, keep, g, offset=offset)
    loss, lse = loss.clone(), lse.clone()
    loss[t - 1] = 0
    lse[2] = want[1][2]
    check((loss, lse, dx, de), want, dtype)
