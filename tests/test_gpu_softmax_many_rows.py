"""More rows than one piece of the wide products holds, than one launch of logits, and than one launch of blocks, against
plain torch on the GPU.  Tolerances as in test_gpu_softmax_paths.py."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
GTOL = {"f32": 2e-5, "bf16": 2.0 ** -8, "f16": 2e-3}


def ops():
    from paper_1511_02433_amd import ops as o
    return o


def make(t, v, d, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(t, d, generator=gen, device="cuda", dtype=DT[dtype])
    e = torch.randn(v, d, generator=gen, device="cuda", dtype=DT[dtype]) * (2 / math.sqrt(d))
    y = torch.randint(0, v, (t,), generator=gen, device="cuda")
    g = torch.rand(t, generator=gen, device="cuda") + 0.5
    return x, e, y, g


@pytest.mark.parametrize("t,v,d,dtype", [(140_000, 5_000, 130, "bf16"), (140_000, 2_100, 130, "f16"), (66_000, 5_000, 130, "f32"), (66_000, 5_000, 400, "f32")])
def test_pieces_of_rows_join(t, v, d, dtype):
    """Two pieces of rows, two or three of items; the last call keeps a part of its logits."""
    x, e, y, g = make(t, v, d, dtype, seed=d)
    y[::5] = -1
    offset = torch.zeros(v, device="cuda")
    offset[7::100] = -25.0  # items that are unlikely for every row
    y = torch.where((y >= 0) & (offset[y.clamp(min=0)] < 0), torch.zeros_like(y), y)
    g[t // 3] = 1e-6
    loss, lse, dx, de = ops().softmax_loss_train(x, e, y, grad=g, offset=offset)
    dx2, de2 = ops().softmax_loss_grad(x, e, y, lse, grad=g, offset=offset)
    assert torch.equal(dx, dx2) and torch.equal(de, de2)
    want_de = torch.zeros(v, d, dtype=torch.float64, device="cuda")
    size = wrong = 0.0
    for a in range(0, t, 10_000):
        s = slice(a, a + 10_000)
        z = torch.mm(x[s].double(), e.double().t()) + offset.double()
        l = torch.logsumexp(z, dim=1)
        assert float((lse[s].double() - l).abs().max()) <= 1e-5 * (1 + float(l.abs().max()))
        at, k, live = torch.arange(len(l), device="cuda"), y[s].clamp(min=0), y[s] >= 0
        assert float((loss[s].double() - torch.where(live, l - z[at, k], torch.zeros_like(l))).abs().max()) <= 1e-5 * (1 + float(z.abs().max()))
        p = torch.exp(z - l[:, None])
        p[at, k] -= 1
        p = torch.where(live[:, None], p * g[s, None].double(), torch.zeros_like(p))
        want = torch.mm(p, e.double())
        size, wrong = size + float(want.square().sum()), wrong + float((dx[s].double() - want).square().sum())
        want_de += torch.mm(p.t().contiguous(), x[s].double())
        if a <= t // 3 < a + 10_000 and dtype != "f16":  # the light row, by itself
            one = t // 3 - a
            assert float((dx[s][one].double() - want[one]).norm()) <= (GTOL[dtype] + 1e-5 * (1 + float(z.abs().max()))) * float(want[one].norm())
    assert wrong ** 0.5 <= GTOL[dtype] * size ** 0.5
    assert float((de.double() - want_de).norm()) <= GTOL[dtype] * float(want_de.norm())
    if dtype != "f16":
        rare, found = want_de[7::100], de[7::100].double()
        assert float((found - rare).norm()) <= (GTOL[dtype] + 5e-5) * float(rare.norm())


def test_more_logits_than_one_launch():
    x, e, y, _ = make(66_000, 131_072, 130, "bf16", seed=1)
    loss, lse = ops().softmax_loss(x, e, y)
    for s in (slice(0, 300), slice(65_400, 65_700), slice(65_900, 66_000)):
        z = torch.mm(x[s].double(), e.double().t())
        l = torch.logsumexp(z, dim=1)
        assert float((lse[s].double() - l).abs().max()) <= 1e-4
        assert float((loss[s].double() - (l - z[torch.arange(len(l), device="cuda"), y[s]])).abs().max()) <= 1e-4


@pytest.mark.parametrize("t,v,d", [((1 << 26) - 1, 2, 1), ((1 << 24) + 5, 40, 257)])
def test_as_many_rows_as_a_launch_has_blocks(t, v, d):
    x, e, y, _ = make(t, v, d, "bf16", seed=2)
    y = y.int()
    loss, lse = ops().softmax_loss(x, e, y)
    for a in range(0, t, 1 << 22):
        s = slice(a, min(t, a + (1 << 22)))
        z = torch.mm(x[s].float(), e.float().t())
        l = torch.logsumexp(z, dim=1)
        assert float((lse[s] - l).abs().max()) <= 1e-4
        assert float((loss[s] - (l - z.gather(1, y[s, None].long())[:, 0])).abs().max()) <= 1e-4
