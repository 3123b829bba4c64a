"""More rows than a launch has blocks, against plain torch on the GPU.  Tolerances as in test_gpu_softmax_paths.py."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


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
