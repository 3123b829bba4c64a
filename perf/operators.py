"""The operators that train and judge factors as a choice among all items, as cases with sizes.

`loss`: the softmax cross entropy of rows of factors (users) against a table of factors (all items), its value per row and
its log-sum-exp.  `grad`: its gradients from a known log-sum-exp.  `train`: loss and gradients in one call.  `clip`: the
global norm of many gradient tensors, and the tensors scaled down to a largest norm.

Rows are t, the table's length (the catalogue or vocabulary) v, the factors' length d.  Inputs are drawn from the seed on
the GPU: logits with a deviation of about two, targets by a power law over the table, one row in sixteen ignored, and where
the case says so an offset per item: a popularity correction, with one item in fifty excluded.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
MAX_LOGITS = 1 << 30            # t * v: the plain form holds the logits a few times over
MAX_FLOPS = 8192 * 131072 * 4096  # t * v * d


def _softmax(name, kind, t, v, d, dtype, offset=False):
    return dict(name=name, kind=kind, t=t, v=v, d=d, dtype=dtype, offset=offset)


def _clip(name, tensors, total, dtype, over):
    return dict(name=name, kind="clip", tensors=tensors, total=total, dtype=dtype, over=over)


def listed():
    return [
        # One user's answer over the catalogue of the large rating matrix, at the usual rank: latency.
        _softmax("loss_one", "loss", 1, 17_770, 40, "f32", offset=True),
        # A few requests' next token or item, from a wide 16-bit table: the table is read once.
        _softmax("loss_serve", "loss", 5, 131_072, 4096, "bf16"),
        # Held-out log-likelihood of users over the very large matrix's catalogue.
        _softmax("loss_catalogue", "loss", 1500, 624_961, 40, "f32"),
        # One mini-batch over the tiny matrix's items: launches count.
        _softmax("train_tiny", "train", 64, 1_000, 8, "f32"),
        # A mini-batch over the medium matrix's items.
        _softmax("train_medium", "train", 1024, 10_681, 40, "f32", offset=True),
        # A large batch over the large matrix's items at the highest rank of the rank sweep.
        _softmax("train_large", "train", 4096, 17_770, 100, "f32"),
        # Odd sizes in half precision, from a kept log-sum-exp.
        _softmax("grad_odd", "grad", 1003, 50_021, 777, "f16", offset=True),
        # Wide factors kept in 32 bits.
        _softmax("train_wide_f32", "train", 2000, 32_003, 1024, "f32"),
        # The head of a large model: the largest.
        _softmax("train_head", "train", 8192, 131_072, 4096, "bf16"),
        # Gradients of the tiny matrix's factors, a few small tensors: launches count.
        _clip("clip_tiny", 6, 24_000, "f32", 3.0),
        # Gradients of W and H of the large matrix at k = 40 among others, below the largest norm.
        _clip("clip_factors", 7, 20_000_003, "f32", 0.5),
        # Gradients of a large model's shard.
        _clip("clip_shard", 60, 1_000_000_007, "bf16", 20.0),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    if rng.random() < 0.25:
        return dict(kind="clip", tensors=rng.randint(2, 60), total=log_int(2_000, 1_000_000_000),
                    dtype=rng.choice(["f32", "f32", "bf16", "f16"]), over=rng.choice([0.5, 2.0, 10.0]))
    kind = rng.choice(["loss", "grad", "train", "train"])
    d = log_int(8, 4096)
    v = log_int(1_000, 624_961)
    t = log_int(1, 8192)
    t = max(1, min(t, MAX_LOGITS // v, MAX_FLOPS // (v * d)))
    dtype = rng.choice(["f32", "bf16", "f16"])
    if dtype == "f32":  # products of 32-bit values cost more
        t = max(1, min(t, MAX_FLOPS // 8 // (v * d)))
    while v * d > 1 << 29:
        v = (v + 1) // 2
    return dict(kind=kind, t=t, v=v, d=d, dtype=dtype, offset=rng.random() < 0.4)


def _sizes(case):
    """Lengths of the tensors: some small ones alike, then each a third of what is left, as they fall."""
    n, left, got = case["tensors"], case["total"], []
    for i in range(n):
        size = left if i == n - 1 else max(1, left // 3 if n - i < 40 and left > 64 * (n - i) else left // (n - i))
        got.append(size)
        left -= size
    return got


def _weights(case):
    """The gradient of the mean over the rows that count, scaled up where the type's range is short."""
    up = 1024.0 if case["dtype"] == "f16" else 1.0
    return (1 + 0.5 * torch.cos(torch.arange(case["t"], device="cuda"))) * (up / case["t"])


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    if case["kind"] == "clip":
        sizes = _sizes(case)
        grads = [torch.randn(n, generator=gen, device="cuda", dtype=dt) for n in sizes]
        return dict(case=case, grads=grads, out=[torch.empty_like(g) for g in grads],
                    max_norm=math.sqrt(case["total"]) / case["over"])
    t, v, d = case["t"], case["v"], case["d"]
    x = torch.randn(t, d, generator=gen, device="cuda", dtype=torch.float32)
    table = torch.randn(v, d, generator=gen, device="cuda", dtype=dt).mul_(2.0 / math.sqrt(d))
    u = torch.rand(t, generator=gen, device="cuda")
    target = (u ** 3 * v).long().clamp_(max=v - 1)
    if t >= 16:
        target[5::16] = -1
    offset = None
    if case["offset"]:
        offset = -0.3 * torch.log(1.0 + torch.arange(v, device="cuda", dtype=torch.float32))
        drop = torch.rand(v, generator=gen, device="cuda") < 0.02
        drop[target.clamp(min=0)] = False
        offset[drop] = -math.inf
    state = dict(case=case, x=x.to(dt), table=table, target=target, offset=offset, scale=1.0, grad=_weights(case))
    if case["kind"] == "grad":
        state["lse"] = _lse(_logits(state))
    return state


def _logits(s):
    z = (s["x"].float() @ s["table"].float().t()).mul_(s["scale"])
    return z if s["offset"] is None else z.add_(s["offset"])


def _lse(z):
    top = z.max(dim=1, keepdim=True).values
    return (top + (z - top).exp_().sum(dim=1, keepdim=True).log())[:, 0]


def _plain_loss(s, z):
    lse = _lse(z)
    at = z.gather(1, s["target"].clamp(min=0)[:, None])[:, 0]
    return torch.where(s["target"] < 0, torch.zeros_like(lse), lse - at), lse


def _plain_grads(s, z, lse):
    dt, counts = s["x"].dtype, s["target"] >= 0
    g = torch.where(counts, s["grad"], torch.zeros_like(s["grad"]))
    p = z.sub_(lse[:, None]).exp_()
    p.scatter_add_(1, s["target"].clamp(min=0)[:, None], -torch.ones_like(g)[:, None])
    p.mul_(g[:, None]).mul_(s["scale"])
    return (p @ s["table"].float()).to(dt), (p.t() @ s["x"].float()).to(dt)


def _plain_clip(s):
    norm = torch.stack([g.float().square().sum() for g in s["grads"]]).sum().sqrt()
    c = (s["max_norm"] / (norm + 1e-6)).clamp(max=1.0)
    return [norm] + [torch.mul(g.float(), c).to(g.dtype) for g in s["grads"]]


def run(state):
    s, kind = state, state["case"]["kind"]
    if own:
        from paper_1511_02433_amd import ops

        if kind == "clip":
            return [ops.clip_grads(s["grads"], s["max_norm"], out=s["out"])] + s["out"]
        args = (s["x"], s["table"], s["target"])
        if kind == "loss":
            return ops.softmax_loss(*args, scale=s["scale"], offset=s["offset"])
        if kind == "grad":
            return ops.softmax_loss_grad(*args, s["lse"], grad=s["grad"], scale=s["scale"], offset=s["offset"])
        return ops.softmax_loss_train(*args, grad=s["grad"], scale=s["scale"], offset=s["offset"])
    if kind == "clip":
        return _plain_clip(s)
    z = _logits(s)
    if kind == "loss":
        return _plain_loss(s, z)
    if kind == "grad":
        return _plain_grads(s, z, s["lse"])
    loss, lse = _plain_loss(s, z)
    return (loss, lse) + _plain_grads(s, z, lse)


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "clip":
        return {"bytes": 2 * size * case["total"], "flops": 3 * case["total"]}
    t, v, d = case["t"], case["v"], case["d"]
    moved = size * (t + v) * d + 8 * t + (4 * v if case["offset"] else 0)  # x, the table, targets and offsets
    if case["kind"] == "loss":
        return {"bytes": moved + 8 * t, "flops": 2 * t * v * d}
    moved += size * (t + v) * d + 4 * t + (4 if case["kind"] == "grad" else 8) * t  # gradients, rows' weights, lse (and loss)
    return {"bytes": moved, "flops": 6 * t * v * d}


def exact(case, seed):
    """The definition in 64 bits, a block of rows after another."""
    s = prepare(case, seed)
    if case["kind"] == "clip":
        norm = math.sqrt(sum(float(torch.sum(g.double() ** 2)) for g in s["grads"]))
        c = min(1.0, s["max_norm"] / (norm + 1e-6))
        return [torch.tensor(norm, dtype=torch.float64)] + [g.double() * c for g in s["grads"]]
    x, e, y = s["x"].double(), s["table"].double(), s["target"]
    t, v = case["t"], case["v"]
    loss = torch.zeros(t, dtype=torch.float64, device="cuda")
    lse, dx, de = torch.zeros_like(loss), torch.zeros_like(x), torch.zeros_like(e)
    step = max(1, (1 << 28) // v)
    for a in range(0, t, step):
        b = min(t, a + step)
        z = s["scale"] * torch.mm(x[a:b], e.T)
        if s["offset"] is not None:
            z += s["offset"].double()
        top = z.max(dim=1, keepdim=True).values
        w = torch.exp(z - top)
        total = w.sum(dim=1, keepdim=True)
        lse[a:b] = (top + total.log())[:, 0]
        rows = torch.nonzero(y[a:b] >= 0)[:, 0]
        hit = y[a:b][rows]
        loss[a + rows] = lse[a + rows] - z[rows, hit]
        if case["kind"] == "loss":
            continue
        del z
        if case["kind"] == "grad":  # from the log-sum-exp that is given, as it was rounded
            w *= torch.exp(top - s["lse"][a:b].double()[:, None])
        else:
            w /= total
        w[rows, hit] -= 1.0
        g = torch.zeros(b - a, dtype=torch.float64, device="cuda")
        g[rows] = s["grad"][a:b][rows].double()
        w *= s["scale"] * g[:, None]
        dx[a:b] = torch.mm(w, e)
        de += torch.mm(w.T, x[a:b])
    return {"loss": (loss, lse), "grad": (dx, de), "train": (loss, lse, dx, de)}[case["kind"]]
