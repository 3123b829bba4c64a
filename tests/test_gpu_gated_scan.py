"""Gated recurrences over packed sequences and their gradients against 64 bits (bounds: seq_util)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from seq_util import DT, U, backward, close, forward, problem, terms, to64

pytestmark = pytest.mark.gpu


def seq():
    from paper_1511_02433_amd import seq as o
    return o


def check(kind, d, dtype, mode, seed=0, initial=True, dlast=True, lead=0, behind=0, pad=0, bits=64, gates=None):
    n, starts, gen, rows = problem(kind, d, dtype, seed, lead, behind, pad)
    s = len(starts) - 1
    x, dy = rows(lambda a: a), rows(lambda a: a)
    gate = rows(gates or (lambda a: a * 1.5 + 1.0))
    if mode == "given" and gates is None:
        gate = torch.sigmoid(gate.float()).to(gate.dtype)
    first = torch.randn(s, d, generator=gen).cuda() if initial else None
    dl = torch.randn(s, d, generator=gen).cuda() if dlast else None
    at = torch.from_numpy(starts).cuda().to(torch.int64 if bits == 64 else torch.int32)
    y, last, kept = seq().gated_scan(x, gate, starts=at, initial=first, mode=mode, keep=True)
    y2, last2 = seq().gated_scan(x, gate, starts=at, initial=first, mode=mode)
    assert torch.equal(y, y2) and torch.equal(last, last2)
    dx, dg, di = seq().gated_scan_grad(x, gate, dy, kept, starts=at, initial=first, mode=mode, dlast=dl)
    X, G, D, I = to64(x), to64(gate), to64(dy), None if first is None else to64(first)
    wy, wl, before, ey, el, eb = forward(X, G, starts, I, mode)
    close(y, wy, ey, "y")
    close(last, wl, el, "last")
    wx, wg, wi, ex, eg, ei = backward(X, G, D, None if dl is None else to64(dl), starts, before, eb, mode)
    close(dx, wx, ex, "dx")
    close(dg, wg, eg, "dgate")
    if initial:
        close(di, wi, ei, "dinitial")
    else:
        assert di is None


KINDS = ["none", "empty", "one", "empties", "ones", "sixteen", "seventeen", "around", "two", "many", "mixed", "emptyrun"]


@pytest.mark.parametrize("mode", ["sigmoid", "given"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("kind", KINDS)
def test_sequences(kind, dtype, mode):
    check(kind, 40, dtype, mode, seed=len(kind), initial=kind != "ones", dlast=kind != "many")


@pytest.mark.parametrize("mode", ["sigmoid", "given"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d", [1, 2, 3, 5, 7, 8, 16, 31, 64, 65, 100, 127, 129, 257, 777])
def test_columns(d, dtype, mode):
    check("around", d, dtype, mode, seed=d, pad=d % 3, lead=d % 5, behind=(d % 4) * 7, bits=32 if d % 2 else 64, initial=d % 3 != 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [1, 4096, 4097])
def test_wide_and_narrow_long(d, dtype):
    check("long" if d == 1 else "seventeen", d, dtype, "sigmoid", seed=3)


@pytest.mark.parametrize("mode", ["sigmoid", "given"])
@pytest.mark.parametrize("lead, behind", [(1, 0), (0, 1), (16, 16), (5, 300), (333, 2)])
def test_rows_of_no_sequence_are_not_read_and_get_zeros(lead, behind, mode):
    n, starts, gen, rows = problem("mixed", 24, "f32", 1, lead, behind)
    x, gate, dy = rows(lambda a: a), rows(lambda a: a * 0.1 + 0.8), rows(lambda a: a)
    at = torch.from_numpy(starts).cuda()
    outside = torch.ones(n, dtype=torch.bool, device="cuda")
    outside[starts[0]:starts[-1]] = False
    y, last, kept = seq().gated_scan(x, gate, starts=at, mode=mode, keep=True)
    dx, dg, _ = seq().gated_scan_grad(x, gate, dy, kept, starts=at, mode=mode)
    for a in (x, gate, dy):
        a[outside] = float("nan")
    y2, last2, kept2 = seq().gated_scan(x, gate, starts=at, mode=mode, keep=True)
    dx2, dg2, _ = seq().gated_scan_grad(x, gate, dy, kept2, starts=at, mode=mode)
    for a, b in ((y, y2), (last, last2), (dx, dx2), (dg, dg2)):
        assert torch.equal(a, b)
    assert bool((y[outside] == 0).all()) and bool((dx[outside] == 0).all()) and bool((dg[outside] == 0).all())


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("where", [0, 1, 15, 16, 400, 899, 901])
def test_what_is_not_finite_stays_in_its_column_and_sequence(where, value):
    n, starts, gen, rows = problem("mixed", 10, "f32", 2)
    x, gate, dy = rows(lambda a: a), rows(lambda a: a), rows(lambda a: a)
    at = torch.from_numpy(starts).cuda()

    def run():
        y, last, kept = seq().gated_scan(x, gate, starts=at, keep=True)
        return (y, last) + seq().gated_scan_grad(x, gate, dy, kept, starts=at)[:2]

    base = run()
    q = int(np.searchsorted(starts, where, side="right")) - 1
    x[where, 3] = value
    dy[where, 3] = value
    got = run()
    touched = torch.zeros(n, 10, dtype=torch.bool, device="cuda")
    touched[starts[q]:starts[q + 1], 3] = True
    for a, b in ((base[0], got[0]), (base[2], got[2]), (base[3], got[3])):
        assert torch.equal(a[~touched], b[~touched])
    assert not bool(torch.isfinite(got[0][where:starts[q + 1], 3]).any())
    assert not bool(torch.isfinite(got[2][starts[q]:where + 1, 3]).any())
    assert torch.equal(base[0][starts[q]:where, 3], got[0][starts[q]:where, 3])
    seqs = torch.arange(len(starts) - 1, device="cuda") != q
    assert torch.equal(base[1][seqs], got[1][seqs])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_gates(dtype):
    """Gates whose sigmoid is 0 or 1 to 32 bits, and infinite ones."""
    def gates(a):
        g = a * 30
        g[a > 2.0] = float("inf")
        g[a < -2.0] = float("-inf")
        return g
    check("mixed", 33, dtype, "sigmoid", seed=5, gates=gates)


def test_given_decays_may_be_zero_negative_or_above_one():
    def gates(a):
        g = (a * 0.7).clamp(-1.2, 1.05)
        g[a.abs() < 0.1] = 0.0
        return g
    check("around", 20, "f32", "given", seed=6, gates=gates)


@pytest.mark.parametrize("mode", ["sigmoid", "given"])
@pytest.mark.parametrize("n, d, s", [(70_001, 5, 1), (70_001, 3, 3), (30_000, 40, 2), (40_000, 2, 9000)])
def test_long(n, d, s, mode):
    """Sequences that many blocks share, with decays near 1."""
    rng = np.random.default_rng(n + s)
    starts = np.concatenate([[0], np.sort(rng.integers(0, n + 1, s - 1)), [n]]).astype(np.int64)
    gen = torch.Generator().manual_seed(s)
    x, dy = torch.randn(n, d, generator=gen).cuda(), torch.randn(n, d, generator=gen).cuda()
    gate = (torch.randn(n, d, generator=gen) * 2 + 5).cuda()
    if mode == "given":
        gate = torch.sigmoid(gate)
    first, dl = torch.randn(s, d, generator=gen).cuda(), torch.randn(s, d, generator=gen).cuda()
    at = torch.from_numpy(starts).cuda()
    y, last, kept = seq().gated_scan(x, gate, starts=at, initial=first, mode=mode, keep=True)
    dx, dg, di = seq().gated_scan_grad(x, gate, dy, kept, starts=at, initial=first, mode=mode, dlast=dl)
    wy, wl, before, ey, el, eb = forward(to64(x), to64(gate), starts, to64(first), mode)
    close(y, wy, ey, "y")
    close(last, wl, el, "last")
    wx, wg, wi, ex, eg, ei = backward(to64(x), to64(gate), to64(dy), to64(dl), starts, before, eb, mode)
    close(dx, wx, ex, "dx")
    close(dg, wg, eg, "dgate")
    close(di, wi, ei, "dinitial")


@pytest.mark.parametrize("mode", ["sigmoid", "given"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n, d, s", [(8_300, 4097, 9), (8_300, 4097, 700), (900, 40_000, 3), (300_000, 130, 40)])
def test_much(n, d, s, dtype, mode):
    """Sizes from which the gradients take two columns a thread, and wide rows one block a CU; columns here and there against 64 bits."""
    rng = np.random.default_rng(n + s)
    starts = np.sort(np.concatenate([[0], rng.integers(0, n - 20, s - 1), [n - 20]])).astype(np.int64)
    gen = torch.Generator(device="cuda").manual_seed(s)

    def rows(scale=1.0, add=0.0):
        return torch.randn(n, d, generator=gen, device="cuda").mul_(scale).add_(add).to(DT[dtype])

    x, gate, dy = rows(), rows(2.0, 2.0), rows()
    if mode == "given":
        gate = torch.sigmoid(gate.float()).to(gate.dtype)
    first, dl = (torch.randn(s, d, generator=gen, device="cuda") for _ in range(2))
    at = torch.from_numpy(starts).cuda()
    y, last, kept = seq().gated_scan(x, gate, starts=at, initial=first, mode=mode, keep=True)
    dx, dg, di = seq().gated_scan_grad(x, gate, dy, kept, starts=at, initial=first, mode=mode, dlast=dl)
    for a in (y, dx, dg):
        assert bool((a[n - 20:] == 0).all()) and bool(torch.isfinite(a).all())
    some = torch.tensor([0, 1, 2, 127, d // 2, d // 2 + 1, d - 3, d - 2, d - 1]).cuda()
    if n > 100_000:
        some = some[[1, 5, 8]]
    X, G, D, I, L = (to64(a[:, some]) for a in (x, gate, dy, first, dl))
    wy, wl, before, ey, el, eb = forward(X, G, starts, I, mode)
    close(y[:, some], wy, ey, "y")
    close(last[:, some], wl, el, "last")
    wx, wg, wi, ex, eg, ei = backward(X, G, D, L, starts, before, eb, mode)
    close(dx[:, some], wx, ex, "dx")
    close(dg[:, some], wg, eg, "dgate")
    close(di[:, some], wi, ei, "dinitial")


@pytest.mark.parametrize("seed", range(24))
def test_random_problems(seed):
    """Sizes, types, layouts and lengths at random: sequences by a power law, some without rows, rows before and behind them."""
    rng = np.random.default_rng(1000 + seed)
    n, s = int(2 ** rng.uniform(3, 13.5)), int(2 ** rng.uniform(0, 8))
    d = int(2 ** rng.uniform(0, 9 if n < 2000 else 5.5))
    dtype, mode = ("f32", "bf16", "f16")[seed % 3], ("sigmoid", "given")[seed % 2]
    share = (rng.random(s) + 0.01) ** -1.5 * (rng.random(s) > 0.1)
    share[rng.integers(s)] += 1e-9
    L = np.floor(share / share.sum() * n).astype(np.int64)
    lead, behind = int(rng.integers(0, 40)) * (seed % 4 == 0), int(rng.integers(0, 400)) * (seed % 4 == 1)
    starts = np.concatenate([[0], np.cumsum(L)]) + lead
    n = int(starts[-1]) + behind
    gen = torch.Generator().manual_seed(seed)
    pad = int(rng.integers(0, 4))

    def rows(f):
        return f(torch.randn(n, d + pad, generator=gen)).to(DT[dtype]).cuda()[:, :d]

    x, dy = rows(lambda a: a), rows(lambda a: a)
    gate = rows(lambda a: a * 2 + 2 if mode == "sigmoid" else torch.sigmoid(a * 2 + 2))
    first = torch.randn(s, d, generator=gen).cuda() if rng.random() < 0.6 else None
    dl = torch.randn(s, d, generator=gen).cuda() if rng.random() < 0.6 else None
    at = torch.from_numpy(starts).cuda().to(torch.int32 if seed % 5 == 0 else torch.int64)
    y, last, kept = seq().gated_scan(x, gate, starts=at, initial=first, mode=mode, keep=True)
    dx, dg, di = seq().gated_scan_grad(x, gate, dy, kept, starts=at, initial=first, mode=mode, dlast=dl)
    I, D = None if first is None else to64(first), None if dl is None else to64(dl)
    wy, wl, before, ey, el, eb = forward(to64(x), to64(gate), starts, I, mode)
    close(y, wy, ey, "y")
    close(last, wl, el, "last")
    wx, wg, wi, ex, eg, ei = backward(to64(x), to64(gate), to64(dy), D, starts, before, eb, mode)
    close(dx, wx, ex, "dx")
    close(dg, wg, eg, "dgate")
    if first is not None:
        close(di, wi, ei, "dinitial")


@pytest.mark.parametrize("n", [0, 1, 700])
def test_rows_without_any_sequence(n):
    x, at = torch.full((n, 9), float("nan"), device="cuda"), torch.tensor([min(n, 3)], device="cuda")
    y, last, kept = seq().gated_scan(x, x, starts=at, keep=True)
    dx, dg, di = seq().gated_scan_grad(x, x, x, kept, starts=at, initial=torch.empty(0, 9, device="cuda"))
    assert last.shape == di.shape == (0, 9)
    for a in (y, dx, dg):
        assert torch.equal(a, torch.zeros(n, 9, device="cuda"))


@pytest.mark.parametrize("mode", ["sigmoid", "given"])
def test_gradients_against_differences(mode):
    """Central differences of the sum in 64 bits: what they leave out is of the order of 1e-8 of the terms here, and they round
    off 1e-16 / 1e-5; the bound is the gradients' own in 32 bits plus 1e-7 of the largest gradient."""
    n, starts, gen, rows = problem("around", 3, "f32", 9)
    s = len(starts) - 1
    x, dy = rows(lambda a: a), rows(lambda a: a)
    gate = rows(lambda a: a if mode == "sigmoid" else torch.sigmoid(a))
    first, dl = torch.randn(s, 3, generator=gen).cuda(), torch.randn(s, 3, generator=gen).cuda()
    at = torch.from_numpy(starts).cuda()
    _, _, kept = seq().gated_scan(x, gate, starts=at, initial=first, mode=mode, keep=True)
    dx, dg, di = seq().gated_scan_grad(x, gate, dy, kept, starts=at, initial=first, mode=mode, dlast=dl)
    X, G, D, I, L = map(to64, (x, gate, dy, first, dl))

    def total(X, G, I):
        y, last, *_ = forward(X, G, starts, I, mode)
        return (D * y).sum() + (L * last).sum()

    _, _, before, _, _, eb = forward(X, G, starts, I, mode)
    *_, ex, eg, ei = backward(X, G, D, L, starts, before, eb, mode)
    rng = np.random.default_rng(0)
    for name, a, got, err in (("dx", X, dx, ex), ("dgate", G, dg, eg), ("dinitial", I, di, ei)):
        for _ in range(8):
            i = (rng.integers(a.shape[0]), rng.integers(3))
            keep, h = a[i], 1e-5
            a[i] = keep + h
            up = total(X, G, I)
            a[i] = keep - h
            down = total(X, G, I)
            a[i] = keep
            assert abs((up - down) / (2 * h) - float(got[i])) <= err[i] + 1e-7 * float(got.abs().max()) + 1e-7, (name, i)


@pytest.mark.parametrize("mode", ["sigmoid", "given"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n, d, pad", [(1, 1, 0), (1, 40, 0), (64, 40, 0), (5, 777, 1), (512, 4096, 0), (3, 6, 3), (33, 130, 6), (0, 8, 0)])
def test_step(n, d, pad, dtype, mode):
    gen = torch.Generator().manual_seed(n + d)
    x = torch.randn(n, d + pad, generator=gen).to(DT[dtype]).cuda()[:, :d]
    gate = torch.randn(n, d + pad, generator=gen).to(DT[dtype]).cuda()[:, :d]
    whole = torch.randn(n, d + pad, generator=gen).cuda()
    state = whole[:, :d]
    rest = whole[:, d:].clone()
    was = to64(state)
    a, u, _ = terms(to64(x), to64(gate), mode)
    want, size = a * was + u, np.abs(a * was) + np.abs(u)
    version = state._version
    y = seq().gated_scan_step(x, gate, state, mode=mode)
    assert state._version == version + 1
    close(state, want, 13 * U * size, "state")
    close(y, want, 13 * U * size, "y")
    assert torch.equal(whole[:, d:], rest)


@pytest.mark.parametrize("mode", ["sigmoid", "given"])
def test_steps_are_the_scan(mode):
    n, d = 37, 20
    gen = torch.Generator().manual_seed(1)
    x, gate = torch.randn(n, d, generator=gen).cuda(), torch.rand(n, d, generator=gen).cuda()
    first = torch.randn(1, d, generator=gen).cuda()
    y, last = seq().gated_scan(x, gate, starts=torch.tensor([0, n]).cuda(), initial=first, mode=mode)
    state = first.clone()
    got = torch.cat([seq().gated_scan_step(x[t:t + 1], gate[t:t + 1], state, mode=mode) for t in range(n)])
    _, _, _, ey, el, _ = forward(to64(x), to64(gate), [0, n], to64(first), mode)
    close(got, to64(y), 2 * ey, "y")
    close(state, to64(last), 2 * el, "last")


def test_refusals():
    x, gate, at = torch.randn(6, 4, device="cuda"), torch.randn(6, 4, device="cuda"), torch.tensor([0, 2, 6], device="cuda")
    _, _, kept = seq().gated_scan(x, gate, starts=at, keep=True)
    for kw, error in ((dict(gate=gate[:5]), ValueError), (dict(gate=gate.half()), ValueError), (dict(gate=gate.cpu()), ValueError), (dict(x=x.T), ValueError),
                      (dict(starts=at.float()), TypeError), (dict(starts=at[:0]), ValueError), (dict(starts=[0, 6]), ValueError), (dict(starts=at.cpu()), ValueError),
                      (dict(mode="tanh"), ValueError), (dict(initial=torch.zeros(3, 4, device="cuda")), ValueError),
                      (dict(initial=torch.zeros(2, 4, device="cuda").half()), TypeError), (dict(y=x[:5].clone()), ValueError), (dict(y=x.half()), ValueError)):
        args = {"x": x, "gate": gate, "starts": at, **kw}
        with pytest.raises(error):
            seq().gated_scan(args.pop("x"), args.pop("gate"), **args)
    for kw, error in ((dict(kept=kept[:, :3]), ValueError), (dict(kept=torch.zeros(2, 4, device="cuda")), ValueError), (dict(dy=x[:5]), ValueError),
                      (dict(dlast=torch.zeros(1, 4, device="cuda")), ValueError), (dict(dx=x.half()), ValueError), (dict(dgate=x[:3]), ValueError)):
        args = {"dy": x, "kept": kept, "starts": at, **kw}
        with pytest.raises(error):
            seq().gated_scan_grad(x, gate, args.pop("dy"), args.pop("kept"), **args)
    for kw in (dict(y=x), dict(y=gate)):
        with pytest.raises(Exception, match="must not be an input"):
            seq().gated_scan(x, gate, starts=at, **kw)
    same = torch.empty_like(x)
    for kw in (dict(dx=x), dict(dgate=gate), dict(dx=same, dgate=same)):
        with pytest.raises(Exception, match="must not be an input"):
            seq().gated_scan_grad(x, gate, torch.randn_like(x), kept, starts=at, **kw)
    for state in (torch.zeros(6, 4, device="cuda").half(), torch.zeros(5, 4, device="cuda"), torch.zeros(1, 4, device="cuda").expand(6, 4)):
        with pytest.raises(Exception):
            seq().gated_scan_step(x, gate, state)


def test_given_outputs_are_written_with_their_strides():
    n, starts, gen, rows = problem("around", 21, "bf16", 4, lead=3, behind=9)
    x, gate, dy = rows(lambda a: a), rows(lambda a: a), rows(lambda a: a)
    at = torch.from_numpy(starts).cuda()
    y, last, kept = seq().gated_scan(x, gate, starts=at, keep=True)
    dx, dg, _ = seq().gated_scan_grad(x, gate, dy, kept, starts=at)
    wide = [torch.full((n, 30), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    v = [a[:, 5:26] for a in wide]
    versions = [a._version for a in v]
    y2, last2, kept2 = seq().gated_scan(x, gate, starts=at, keep=True, y=v[0])
    dx2, dg2, _ = seq().gated_scan_grad(x, gate, dy, kept2, starts=at, dx=v[1], dgate=v[2])
    assert y2 is v[0] and dx2 is v[1] and dg2 is v[2]
    assert [a._version for a in v] == [k + 1 for k in versions]
    for a, b in ((y, y2), (dx, dx2), (dg, dg2), (last, last2)):
        assert torch.equal(a, b)
    for a in wide:
        assert bool((a[:, :5] == 7).all()) and bool((a[:, 26:] == 7).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_rows_aligned_to_their_type_alone(dtype):
    n, starts, gen, rows = problem("around", 37, dtype, 4, pad=6)
    x, gate, dy = rows(lambda a: a), rows(lambda a: a), rows(lambda a: a)
    at = torch.from_numpy(starts).cuda()
    y, last, kept = seq().gated_scan(x, gate, starts=at, keep=True)
    want = (y, last) + seq().gated_scan_grad(x, gate, dy, kept, starts=at)[:2]

    def moved(a):
        wide = torch.zeros(n, 50, dtype=a.dtype, device="cuda")
        wide[:, 1:38] = a
        return wide[:, 1:38]

    y, last, kept = seq().gated_scan(moved(x), moved(gate), starts=at, keep=True, y=moved(x))
    got = (y, last) + seq().gated_scan_grad(moved(x), moved(gate), moved(dy), kept, starts=at, dx=moved(x), dgate=moved(x))[:2]
    for a, b in zip(want, got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("n, empties", [(5000, 400), (3000, 3000), (70_000, 9000)])
def test_many_sequences_without_rows_and_short_ones(n, empties):
    """Starts that lie close together and far apart in the same tables: sequences of one row, and runs of none, at random places."""
    rng = np.random.default_rng(n)
    at = np.sort(np.concatenate([rng.integers(0, n + 1, empties // 2), rng.integers(n // 3, n // 3 + 20, empties // 2), [0, n]]))
    s, d = len(at) - 1, 3
    gen = torch.Generator().manual_seed(n)
    x, gate = torch.randn(n, d, generator=gen).cuda(), torch.randn(n, d, generator=gen).cuda()
    first = torch.randn(s, d, generator=gen).cuda()
    y, last, kept = seq().gated_scan(x, gate, starts=torch.from_numpy(at).cuda(), initial=first, keep=True)
    dx, dg, di = seq().gated_scan_grad(x, gate, x, kept, starts=torch.from_numpy(at).cuda(), initial=first, dlast=first)
    wy, wl, before, ey, el, eb = forward(to64(x), to64(gate), at, to64(first), "sigmoid")
    close(y, wy, ey, "y")
    close(last, wl, el, "last")
    wx, wg, wi, ex, eg, ei = backward(to64(x), to64(gate), to64(x), to64(first), at, before, eb, "sigmoid")
    close(dx, wx, ex, "dx")
    close(dg, wg, eg, "dgate")
    close(di, wi, ei, "dinitial")


def test_offsets_beyond_32_bits():
    """Rows more than 2^31 values apart."""
    d, ld = 40, (1 << 31) + 64
    gen = torch.Generator().manual_seed(8)
    small = torch.randn(3, 3, d, generator=gen).to(torch.bfloat16).cuda()
    big = [torch.empty(2 * ld + d, dtype=torch.bfloat16, device="cuda").as_strided((3, d), (ld, 1)) for _ in range(4)]
    for i in range(3):
        big[i].copy_(small[i])
    at = torch.tensor([0, 1, 3]).cuda()
    y, last, kept = seq().gated_scan(small[0], small[1], starts=at, keep=True)
    y2, last2, kept2 = seq().gated_scan(big[0], big[1], starts=at, keep=True, y=big[3])
    assert torch.equal(y, y2) and torch.equal(last, last2)
    want = seq().gated_scan_grad(small[0], small[1], small[2], kept, starts=at)
    got = seq().gated_scan_grad(big[0], big[1], big[2], kept2, starts=at, dx=big[3])
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


@pytest.mark.parametrize("starts", [[5, 3, 40], [0, 90, 20, 64], [-7, 10, 200], [64, 0], [-5, -3], [70, 80, 90]])
def test_starts_that_do_not_ascend_or_lie_outside_stay_within_memory(starts):
    """What lies around the tensors is left as it is, and what is written to them is theirs."""
    n, d = 64, 8
    at = torch.tensor(starts).cuda()
    s = len(starts) - 1
    x, gate, dy = (torch.randn(n, d, device="cuda") for _ in range(3))
    wide = [torch.full((n + 64, d), 7.0, device="cuda") for _ in range(3)]
    y, last, kept = seq().gated_scan(x, gate, starts=at, keep=True, y=wide[0][32:32 + n])
    seq().gated_scan_grad(x, gate, dy, kept, starts=at, dx=wide[1][32:32 + n], dgate=wide[2][32:32 + n], initial=torch.zeros(s, d, device="cuda"))
    torch.cuda.synchronize()
    for a in wide:
        assert bool((a[:32] == 7).all()) and bool((a[32 + n:] == 7).all())


def test_captured_and_replayed_between_eager_work():
    n, starts, gen, rows = problem("mixed", 40, "bf16", 4)
    x, gate, dy = rows(lambda a: a), rows(lambda a: a), rows(lambda a: a)
    at = torch.from_numpy(starts).cuda()
    first = torch.randn(len(starts) - 1, 40, generator=gen).cuda()

    def run():
        y, last, kept = seq().gated_scan(x, gate, starts=at, initial=first, keep=True)
        return (y, last) + seq().gated_scan_grad(x, gate, dy, kept, starts=at, initial=first)

    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = run()
    for i in range(4):
        x.copy_(torch.randn(x.shape, generator=gen).to(x.dtype))
        if i == 2:  # other sequences of the same number
            moved = np.sort(np.random.default_rng(3).integers(0, n + 1, len(starts)))
            at.copy_(torch.from_numpy(moved))
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, run()):
            assert torch.equal(a, b)


def test_on_another_stream():
    n, starts, gen, rows = problem("mixed", 40, "f32", 4)
    x, gate = rows(lambda a: a), rows(lambda a: a)
    at = torch.from_numpy(starts).cuda()
    want, _ = seq().gated_scan(x, gate, starts=at)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for st in streams:
        with torch.cuda.stream(st):
            got.append(seq().gated_scan(x, gate, starts=at)[0])
    torch.cuda.synchronize()
    for a in got:
        assert torch.equal(a, want)
