"""Softmax loss over a whole table and its gradients, against plain float64 torch on the CPU.

Tolerances.  lse and loss: a logit is a sum of d products, each exact to 2^-21 of (largest of the row) x (largest of the
table) for 32-bit values (22-bit halves on both sides) and exact for 16-bit ones, summed in 32 bits; with |z| <= Z that is
within (d 2^-21 max|x| max|e| + a few 2^-24 Z); the tests bound it by ZTOL = 1e-5 (1 + max |z|).  Gradients: the
relative error in the 2-norm is at most the error of the terms G (2^-9 for bfloat16, 2^-11 for float16, 2^-21 for
32-bit values plus the logits' absolute error) plus one rounding of the result: 1e-2, 2e-3 and 2e-5.
"""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
GTOL = {"f32": 2e-5, "bf16": 1e-2, "f16": 2e-3}


def ops():
    from paper_1511_02433_amd import ops as o
    return o


def plain(x, e, y, scale=1.0, offset=None, grad=None):
    """The definition in 64 bits (CPU): loss, lse, dx, de."""
    x, e, y = x.double().cpu(), e.double().cpu(), y.long().cpu()
    t, v = x.shape[0], e.shape[0]
    o = torch.zeros(v, dtype=torch.float64) if offset is None else offset.double().cpu()
    excluded = o < -1e38
    live = ~excluded
    z = torch.full((t, v), -math.inf, dtype=torch.float64)
    z[:, live] = scale * (x @ e[live].t()) + o[live]
    lse = torch.logsumexp(z, dim=1)
    loss = torch.zeros(t, dtype=torch.float64)
    g = torch.ones(t, dtype=torch.float64) if grad is None else grad.double().cpu()
    p = torch.exp(z - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)[:, None])
    counts = torch.zeros(t, dtype=torch.bool)
    for i in range(t):
        if y[i] < 0:
            continue
        if excluded[y[i]]:
            loss[i] = math.inf
            continue
        loss[i] = lse[i] - z[i, y[i]]
        p[i, y[i]] -= 1
        counts[i] = True
    p = torch.where(counts[:, None], p * g[:, None], torch.zeros_like(p))
    dx = scale * (p[:, live] @ e[live])
    de = torch.zeros(v, e.shape[1], dtype=torch.float64)
    de[live] = scale * (p[counts][:, live].t() @ x[counts])
    return loss, lse, dx, de


def make(t, v, d, dtype, seed=0, spread=2.0):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(t, d, generator=gen).to(DT[dtype]).cuda()
    e = (torch.randn(v, d, generator=gen) * (spread / math.sqrt(d))).to(DT[dtype]).cuda()
    y = torch.randint(0, v, (t,), generator=gen).cuda()
    g = (torch.rand(t, generator=gen) + 0.5).cuda()
    return x, e, y, g


def rel(a, b):
    a, b = a.double().cpu(), b.double().cpu()
    n = b.norm()
    return float((a - b).norm() / n) if n > 0 else float(a.norm())


def check(got, want, dtype):
    loss, lse, dx, de = got
    wl, wz, wx, we = want
    z = 1e-5 * (1 + float(wz[torch.isfinite(wz)].abs().max() if torch.isfinite(wz).any() else 0))
    for a, b in ((loss, wl), (lse, wz)):
        a = a.double().cpu()
        assert torch.equal(torch.isfinite(a), torch.isfinite(b))
        assert torch.equal(a[~torch.isfinite(b)], b[~torch.isfinite(b)])
        f = torch.isfinite(b)
        assert float((a[f] - b[f]).abs().max() if f.any() else 0) <= z
    assert rel(dx, wx) <= GTOL[dtype]
    assert rel(de, we) <= GTOL[dtype]


SIZES = [(1, 1, 1), (1, 2, 3), (2, 31, 8), (3, 33, 40), (31, 255, 17), (33, 257, 64), (1, 1000, 40), (5, 777, 1000),
         (65, 300, 129), (257, 511, 100), (130, 2500, 33), (300, 40, 260), (17, 5000, 96), (64, 1000, 8), (600, 129, 128)]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("t,v,d", SIZES)
def test_train_matches_float64(t, v, d, dtype):
    x, e, y, g = make(t, v, d, dtype, seed=t * 7 + v + d)
    if t > 4:
        y[3] = -1
        y[4] = -100
    got = ops().softmax_loss_train(x, e, y, grad=g, scale=0.7)
    check(got, plain(x, e, y, 0.7, None, g), dtype)
    # the parts alone give the same
    loss, lse = ops().softmax_loss(x, e, y, scale=0.7)
    assert torch.equal(loss, got[0]) and torch.equal(lse, got[1])
    dx, de = ops().softmax_loss_grad(x, e, y, lse, grad=g, scale=0.7)
    assert torch.equal(dx, got[2]) and torch.equal(de, got[3])


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("t,v,d", [(1, 300, 40), (7, 513, 64), (40, 300, 40), (130, 1030, 150)])
def test_offsets_and_excluded_items(t, v, d, dtype):
    x, e, y, g = make(t, v, d, dtype, seed=5)
    off = torch.randn(v, generator=torch.Generator().manual_seed(1)).cuda()
    off[::5] = -math.inf
    off[1::7] = torch.finfo(torch.float32).min
    bad = off < -1e38
    e[bad] = math.nan  # what an excluded item holds does not matter
    e[10] = math.inf
    y = torch.where(bad[y], torch.full_like(y, 2), y)
    off[2] = 0.5
    e[2] = 0.25
    y[0] = 5 if t > 1 else 2  # excluded target: loss +inf, out of the gradients
    want = plain(x, e, y, 1.0, off, g)
    got = ops().softmax_loss_train(x, e, y, grad=g, offset=off)
    check(got, want, dtype)
    assert float(got[3][bad].float().abs().max()) == 0.0
    if t > 1:
        assert math.isinf(float(got[0][0])) and float(got[2][0].float().abs().max()) == 0.0


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("t,v,d", [(1, 100, 40), (33, 300, 40), (20, 600, 200)])
def test_everything_excluded(t, v, d, dtype):
    x, e, y, g = make(t, v, d, dtype)
    for low in (-math.inf, torch.finfo(torch.float32).min):
        off = torch.full((v,), low, device="cuda")
        loss, lse, dx, de = ops().softmax_loss_train(x, e, y, grad=g, offset=off)
        assert bool((lse == -math.inf).all()) and bool((loss == math.inf).all())
        assert float(dx.float().abs().max()) == 0.0 and float(de.float().abs().max()) == 0.0


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("t,v,d", [(3, 100, 40), (40, 300, 40), (70, 600, 200)])
def test_ignored_rows_may_hold_anything(t, v, d, dtype):
    x, e, y, g = make(t, v, d, dtype, seed=3)
    y[1], y[2] = -1, -(1 << 40)
    want = plain(x, e, y, 1.0, None, g)
    x[1], x[2] = math.nan, 6e4  # a row of NaN, a row of large values
    g[1] = math.nan
    got = ops().softmax_loss_train(x, e, y, grad=g)
    keep = torch.arange(t) != 1
    keep[2] = False
    assert float(got[0][1]) == 0.0 and float(got[0][2]) == 0.0
    assert float(got[2][1].float().abs().max()) == 0.0
    check((got[0][keep.cuda()], got[1][keep.cuda()], got[2], got[3]), (want[0][keep], want[1][keep], want[2], want[3]), dtype)


@pytest.mark.parametrize("t,v,d", [(3, 100, 40), (40, 300, 40)])
def test_all_rows_ignored(t, v, d):
    x, e, y, g = make(t, v, d, "f32")
    y[:] = -1
    loss, lse, dx, de = ops().softmax_loss_train(x, e, y, grad=g)
    assert float(loss.abs().max()) == 0 and bool(torch.isfinite(lse).all())
    assert float(dx.abs().max()) == 0 and float(de.abs().max()) == 0


@pytest.mark.parametrize("t,v,d", [(3, 100, 40), (40, 300, 200)])
def test_target_past_the_table_is_loud(t, v, d):
    x, e, y, g = make(t, v, d, "f32")
    y[1] = v
    loss, lse, dx, de = ops().softmax_loss_train(x, e, y, grad=g)
    assert math.isnan(float(loss[1])) and bool(torch.isfinite(lse).all())
    assert bool(torch.isfinite(loss[0])) and bool(torch.isnan(dx[1]).all()) and bool(torch.isnan(de).any())
    assert bool(torch.isfinite(dx[0]).all())


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("t,v,d", [(2, 300, 24), (50, 300, 24), (40, 300, 136)])
def test_strides_alignment_and_int32_targets(t, v, d, dtype):
    gen = torch.Generator().manual_seed(2)
    bx = torch.full((t, d + 13), math.nan).to(DT[dtype]).cuda()
    be = torch.full((v, d + 5), math.nan).to(DT[dtype]).cuda()
    x, e = bx[:, 3:3 + d], be[:, 1:1 + d]
    x.copy_(torch.randn(t, d, generator=gen))
    e.copy_(torch.randn(v, d, generator=gen) * 0.3)
    y = torch.randint(0, v, (t,), generator=gen).int().cuda()
    bdx, bde = torch.zeros_like(bx), torch.zeros_like(be)
    dx, de = bdx[:, 3:3 + d], bde[:, 1:1 + d]
    got = ops().softmax_loss_train(x, e, y, scale=-1.3, dx=dx, dtable=de)
    check(got, plain(x, e, y, -1.3), dtype)
    assert got[2].data_ptr() == dx.data_ptr()
    dx.zero_(), de.zero_()
    assert float(bdx.float().abs().max()) == 0 and float(bde.float().abs().max()) == 0  # nothing beside them


def test_only_one_gradient():
    x, e, y, g = make(70, 300, 40, "f32")
    both = ops().softmax_loss_train(x, e, y, grad=g)
    a = ops().softmax_loss_train(x, e, y, grad=g, need=("x",))
    b = ops().softmax_loss_train(x, e, y, grad=g, need=("table",))
    assert a[3] is None and b[2] is None
    assert torch.equal(a[2], both[2]) and torch.equal(b[3], both[3])


@pytest.mark.parametrize("dtype", list(DT))
def test_no_rows(dtype):
    x, e, y, g = make(0, 30, 40, dtype)
    loss, lse, dx, de = ops().softmax_loss_train(x, e, y, grad=g)
    assert loss.shape == (0,) and lse.shape == (0,) and dx.shape == (0, 40)
    assert float(de.float().abs().max()) == 0.0


@pytest.mark.parametrize("t,v,d", [(4, 60, 24), (40, 60, 24), (40, 60, 200)])
def test_gradients_against_differences(t, v, d):
    """Central differences of the operator's own loss.  Its rounding (1e-6 of a loss near 5, over a step of 2 h)
    allows 4 x 5e-6 / 2 h + the third derivative's h^2: 2e-3 of the direction's norm at h = 1e-2."""
    x, e, y, g = make(t, v, d, "f32", seed=9)
    _, _, dx, de = ops().softmax_loss_train(x, e, y, grad=g)
    gen = torch.Generator().manual_seed(4)
    h = 1e-2
    for _ in range(4):
        ux, ue = torch.randn(t, d, generator=gen).cuda(), torch.randn(v, d, generator=gen).cuda()
        ux, ue = ux / ux.norm(), ue / ue.norm()
        up = (g.double() * ops().softmax_loss(x + h * ux, e + h * ue, y)[0].double()).sum()
        dn = (g.double() * ops().softmax_loss(x - h * ux, e - h * ue, y)[0].double()).sum()
        along = float((dx.double() * ux).sum() + (de.double() * ue).sum())
        size = float(dx.norm() + de.norm())
        assert abs(float(up - dn) / (2 * h) - along) <= 2e-3 * size


@pytest.mark.parametrize("scale_x,scale_e", [(1e-20, 1e18), (1e15, 1e-16), (1e-30, 1e-30)])
def test_f32_ranges(scale_x, scale_e):
    """32-bit values far from one, a row a million times the others, tiny weights."""
    x, e, y, g = make(60, 400, 40, "f32", seed=8)
    x = x * scale_x
    e = e * scale_e
    x[7] *= 1e-6
    x[8] = 0
    want = plain(x, e, y, 1.0, None, g * 1e-9)
    got = ops().softmax_loss_train(x, e, y, grad=g * 1e-9)
    check(got, want, "f32")


def test_large_logits_and_one_hot_rows():
    x, e, y, g = make(50, 500, 40, "f32", spread=60.0)
    check(ops().softmax_loss_train(x, e, y, grad=g), plain(x, e, y, 1.0, None, g), "f32")


@pytest.mark.parametrize("t,v,d", [(2, 3000, 40), (40, 3000, 40), (300, 2000, 160)])
def test_repeated_calls_are_identical_and_other_streams(t, v, d):
    x, e, y, g = make(t, v, d, "f32", seed=1)
    a = ops().softmax_loss_train(x, e, y, grad=g)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        b = ops().softmax_loss_train(x, e, y, grad=g)
    s.synchronize()
    for p, q in zip(a, b):
        assert torch.equal(p, q)


def test_pieces_join():
    """More rows and items than one piece of the gradients holds."""
    x, e, y, g = make(2100, 40_000, 24, "bf16", seed=6)
    got = ops().softmax_loss_train(x, e, y, grad=g)
    xf, ef = x.float(), e.float()
    z = (xf @ ef.t()).double()
    lse = torch.logsumexp(z, dim=1)
    assert float((got[1].double() - lse).abs().max()) <= 1e-4
    p = torch.exp(z - lse[:, None])
    p[torch.arange(2100, device="cuda"), y] -= 1
    p *= g[:, None].double()
    assert rel(got[2], (p @ ef.double())) <= 1e-2
    assert rel(got[3], (p.t().contiguous() @ xf.double())) <= 1e-2


def test_graph_capture_replays():
    x, e, y, g = make(64, 1000, 40, "f32")
    want = [a.clone() for a in ops().softmax_loss_train(x, e, y, grad=g)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        ops().softmax_loss_train(x, e, y, grad=g)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = ops().softmax_loss_train(x, e, y, grad=g)
    for k in range(3):
        for a in got:
            a.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), k
        _ = (x @ x.t()).sum().item()


def test_refusals():
    o = ops()
    x, e, y, g = make(4, 10, 8, "f32")
    with pytest.raises(TypeError):
        o.softmax_loss(x.double(), e.double(), y)
    with pytest.raises(ValueError):
        o.softmax_loss(x, e.half(), y)
    with pytest.raises(ValueError):
        o.softmax_loss(x, e[:, :7], y)
    with pytest.raises(ValueError):
        o.softmax_loss(x, e, y[:3])
    with pytest.raises(TypeError):
        o.softmax_loss(x, e, y.float())
    with pytest.raises(ValueError):
        o.softmax_loss(x.t().contiguous().t(), e, y)
    with pytest.raises(ValueError):
        o.softmax_loss(x.cpu(), e, y)
    with pytest.raises(ValueError):
        o.softmax_loss_grad(x, e, y, g[:2])
    with pytest.raises(ValueError):
        o.softmax_loss_train(x, e, y, grad=g, need=("w",))
    with pytest.raises(ValueError):
        o.softmax_loss_train(x, e, y, dx=torch.empty(4, 9, device="cuda"))
    from paper_1511_02433_amd.ccdpp import CCDPP_EINVAL, CCDPPError
    with pytest.raises(CCDPPError) as err:
        o.softmax_loss(x, e, y, scale=math.inf)
    assert err.value.code == CCDPP_EINVAL and "scale" in str(err.value)
    with pytest.raises(CCDPPError) as err:
        o.softmax_loss(x[:1].expand(4, 8), e, y)  # rows on top of one another
    assert "ldx" in str(err.value)
    with pytest.raises(CCDPPError):
        o.softmax_loss(x, e[:0], y)
