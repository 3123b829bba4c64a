"""Beam selection against 64 bits, and the reordering of states.

Items and beams have to be those of the oracle wherever its scores differ by more than what the log sums may be off: a sum of
exponentials in 32 bits, each within (|z - reference| + 3) 2^-24 of itself and added in pieces, is within 2^-18 here (|z - reference|
below 50 where a term counts), in the logarithm 2^-18 absolute, and the score is rounded once.  Between beams the tests' scores are
further apart or equal by construction; within a beam the order is exact."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
LOG = 2.0 ** -18


def seq():
    from paper_1511_02433_amd import seq as o
    return o


def oracle(logits, score, k, offset=None, done=None, end=None):
    """Continuations as (score, beam, item), on the host: by score (NaN first), beam, z (NaN as infinity), item."""
    g, b = score.shape
    z = logits.float()
    if offset is not None:
        z = torch.where(offset < -1e38, torch.tensor(-math.inf), z + offset)
    z = z.double().view(g, b, -1)
    out = []
    for i in range(g):
        found = []
        for j in range(b):
            s = float(score[i, j])
            if s == -math.inf:
                continue
            if done is not None and bool(done[i, j]):
                found.append((s, j, 0, end))
                continue
            row = z[i, j]
            bad = bool(torch.isnan(row).any() or (row == math.inf).any())
            total = math.nan if bad else float(torch.logsumexp(row, 0))
            key = torch.where(torch.isnan(row), torch.tensor(math.inf, dtype=torch.float64), row)
            order = torch.sort(key, descending=True, stable=True).indices
            for r, item in enumerate(order[:k].tolist()):
                if float(row[item]) != -math.inf:
                    found.append((s + (float(row[item]) - total), j, r, item))
        found.sort(key=lambda c: (not math.isnan(c[0]), -c[0] if not math.isnan(c[0]) else 0, c[1], c[2]))
        found = found[:k] + [(-math.inf, -1, 0, -1)] * (k - min(k, len(found)))
        out.append([(c[0], c[1], c[3]) for c in found])
    return (torch.tensor([[c[0] for c in r] for r in out], dtype=torch.float64).view(g, k), torch.tensor([[c[1] for c in r] for r in out]).view(g, k),
            torch.tensor([[c[2] for c in r] for r in out]).view(g, k))


def check(logits, score, k, **kw):
    host = {n: a.cpu() if isinstance(a, torch.Tensor) else a for n, a in kw.items()}
    ws, wp, wi = oracle(logits.cpu(), score.cpu(), k, **host)
    s, p, i, f = seq().beam_select(logits, score, k, **kw)
    assert s.dtype == torch.float32 and p.dtype == i.dtype == torch.int64
    assert torch.equal(p.cpu(), wp) and torch.equal(i.cpu(), wi)
    if kw.get("end") is None:
        assert f is None
    else:
        assert f.dtype == torch.bool and torch.equal(f.cpu(), (wi == kw["end"]) | (wi == -1))
    s = s.double().cpu()
    assert torch.equal(torch.isnan(s), torch.isnan(ws))
    fin = torch.isfinite(ws)
    assert torch.equal(s[~fin & ~torch.isnan(ws)], ws[~fin & ~torch.isnan(ws)])
    assert bool(((s - ws)[fin].abs() <= LOG + 2.0 ** -23 * ws[fin].abs()).all())
    return s, p, i


def make(g, b, v, dtype, seed, pad=0, spread=2.0):
    gen = torch.Generator().manual_seed(seed)
    logits = (torch.randn(g * b, v + pad, generator=gen) * spread).to(DT[dtype]).cuda()[:, :v]
    score = (-torch.rand(g, b, generator=gen) * 3).cumsum(1).cuda()
    return gen, logits, score


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("g, b, k, v, pad", [
    (1, 1, 1, 1, 0), (1, 1, 4, 2, 0), (2, 3, 5, 7, 1), (1, 4, 4, 63, 0), (3, 2, 8, 64, 3), (1, 8, 8, 65, 0), (2, 5, 3, 255, 0), (2, 5, 3, 257, 2),
    (1, 4, 4, 1000, 0), (4, 4, 4, 4097, 1), (2, 16, 16, 2049, 0), (1, 64, 64, 300, 5), (3, 7, 64, 1023, 0), (1, 64, 1, 5000, 1), (1, 1, 64, 10_001, 0),
    (5, 8, 8, 17_770, 0), (1, 2, 10, 140_003, 1), (1, 1, 8, 624_961, 0), (1, 3, 64, 600_001, 1), (40, 16, 4, 5000, 0)])
def test_select(g, b, k, v, pad, dtype):
    _, logits, score = make(g, b, v, dtype, g * 1000 + v, pad)
    check(logits, score, k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v", [50, 3001, 70_000])
def test_offsets_ends_and_beams_that_are_none(v, dtype):
    gen, logits, score = make(6, 4, v, dtype, v)
    offset = torch.randn(v, generator=gen)
    offset[torch.rand(v, generator=gen) < 0.1] = -math.inf
    offset[3], offset[4] = -2e38, -math.inf
    offset = offset.cuda()
    logits[:, 4] = math.nan   # excluded, whatever it holds
    logits[1, 3] = math.inf
    logits[2, 7] = -math.inf
    score[1, 1:] = -math.inf
    score[2] = -math.inf
    done = torch.rand(6, 4, generator=gen) < 0.3
    done[2, 1] = done[3, 0] = True
    done[4] = True
    done = done.cuda()
    logits.view(6, 4, v)[4] = math.nan  # not read
    logits.view(6, 4, v)[2] = math.nan
    check(logits, score, 6, offset=offset, done=done, end=v // 2)
    check(logits[:4], score[:1], 6, offset=offset, end=0)
    offset[:] = -math.inf  # nothing left but what has ended
    _, p, i = check(logits, score, 6, offset=offset, done=done, end=5)
    assert set(i.unique().tolist()) <= {-1, 5}


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("v", [5, 1024, 40_001])
def test_equal_scores_go_to_the_lowest_beam_and_item(v, dtype):
    g, b, k = 2, 4, 8
    logits = torch.zeros(g * b, v, dtype=DT[dtype], device="cuda")
    score = torch.zeros(g, b, device="cuda")
    _, p, i = check(logits, score, k)
    for j in range(k):
        assert (int(p[0, j]), int(i[0, j])) == (j // min(v, 99), j % v)
    logits[:, ::2] = -0.0  # equal to 0
    check(logits, score, k)
    logits[:] = torch.randint(-2, 3, (v,), generator=torch.Generator().manual_seed(1)).to(logits.dtype).cuda()  # the same row in every beam
    check(logits, score, k)


@pytest.mark.parametrize("order", ["up", "down", "saw"])
@pytest.mark.parametrize("k", [1, 8, 64])
def test_rows_in_order(k, order):
    v = 30_011
    at = torch.arange(v, dtype=torch.float32)
    row = {"up": at / 1000, "down": -at / 1000, "saw": (at * 7919 % 1009) / 100 + at * 1e-6}[order]
    logits = torch.stack([row, row + 0.5]).cuda()
    check(logits, torch.tensor([[-0.25, -3.0]]).cuda(), k)


def test_what_is_not_finite():
    _, logits, score = make(5, 2, 500, "f32", 3)
    logits[0, 17] = math.nan
    logits[3, 400] = math.inf
    logits[4] = -math.inf
    logits[6] = -math.inf
    logits[7] = -math.inf
    logits[6, 9] = 0.0
    score[4, 0] = math.nan
    check(logits, score, 5)


@pytest.mark.parametrize("score", [math.inf, 3.0e38, -3.0e38])
def test_scores_at_the_ends_of_their_range(score):
    _, logits, s = make(2, 3, 700, "f32", 4)
    s[0, 1] = score
    s[1] = score
    check(logits, s, 7)


@pytest.mark.parametrize("k", [1, 8, 64])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_large_values_side_by_side(k, dtype):
    """A run of items far above the others, more than are put aside at a time, some of them equal."""
    gen, logits, score = make(1, 2, 20_000, dtype, k)
    logits[0, 4000:6500] += 30
    logits[1, 9000:9300] = 25.0
    logits[1, 15_000:15_100] = 26.0
    check(logits, score, k)


@pytest.mark.parametrize("low", [-1e30, -1e38, -3.0e38])
def test_masks_of_very_low_values_are_not_exclusions(low):
    """A mask that is finite takes part where nothing else is left."""
    _, logits, score = make(1, 2, 300, "f32", 3)
    logits[:, 3:] = low
    check(logits, score, 8)
    logits[:] = low
    check(logits, score, 8)


@pytest.mark.parametrize("spread", [0.0, 1e-3, 40.0, 1e4])
def test_spread(spread):
    _, logits, score = make(2, 3, 5000, "f32", 11, spread=spread)
    check(logits, score, 4)


def test_offsets_beyond_32_bits():
    v, ld = 1000, (1 << 31) + 8
    _, logits, score = make(1, 3, v, "bf16", 5)
    big = torch.empty(2 * ld + v, dtype=torch.bfloat16, device="cuda").as_strided((3, v), (ld, 1))
    big.copy_(logits)
    for a, b in zip(seq().beam_select(logits, score, 4)[:3], seq().beam_select(big, score, 4)[:3]):
        assert torch.equal(a, b)


def test_refusals():
    _, logits, score = make(2, 3, 50, "f32", 1)
    good = dict(logits=logits, score=score, k=2)
    for kw, error in ((dict(k=0), ValueError), (dict(k=65), ValueError), (dict(k=2 ** 32 + 2), ValueError), (dict(score=score[:1]), ValueError),
                      (dict(score=score.double()), TypeError), (dict(score=score.cpu()), ValueError), (dict(logits=logits[:, ::2]), ValueError),
                      (dict(offset=torch.zeros(49, device="cuda")), ValueError), (dict(done=torch.zeros(2, 3, dtype=torch.bool, device="cuda")), ValueError),
                      (dict(done=torch.zeros(2, 2, dtype=torch.bool, device="cuda"), end=1), ValueError), (dict(end=50), ValueError), (dict(end=-1), ValueError),
                      (dict(done=torch.zeros(2, 3, device="cuda"), end=1), TypeError)):
        args = {**good, **kw}
        with pytest.raises(error):
            seq().beam_select(args.pop("logits"), args.pop("score"), args.pop("k"), **args)
    parent = torch.zeros(2, 3, dtype=torch.int64, device="cuda")
    state = torch.randn(6, 4, device="cuda")
    for kw, error in ((dict(states=[state[:5]]), ValueError), (dict(states=[state.cpu()]), ValueError), (dict(states=[state[:, ::2]]), ValueError),
                      (dict(beams=0), ValueError), (dict(beams=65), ValueError), (dict(parent=parent.int()), TypeError), (dict(parent=parent.T), ValueError),
                      (dict(out=[]), ValueError), (dict(out=[state[:5].clone()]), ValueError), (dict(out=[state.double()]), ValueError), (dict(states=[1.0]), TypeError)):
        args = {"parent": parent, "states": [state], "beams": 3, **kw}
        with pytest.raises(error):
            seq().beam_reorder(args.pop("parent"), args.pop("states"), **args)
    with pytest.raises(Exception, match="must not be an input"):
        seq().beam_reorder(parent, [state], beams=3, out=[state])


def test_no_groups():
    s, p, i, f = seq().beam_select(torch.zeros(0, 10, device="cuda"), torch.zeros(0, 4, device="cuda"), 3, end=1)
    assert s.shape == p.shape == i.shape == f.shape == (0, 3)
    assert seq().beam_reorder(p, [torch.zeros(0, 5, device="cuda")], beams=4)[0].shape == (0, 5)


@pytest.mark.parametrize("g, b, k", [(1, 1, 1), (3, 4, 2), (2, 5, 9), (17, 8, 8)])
def test_reorder(g, b, k):
    gen = torch.Generator().manual_seed(g)
    parent = torch.randint(-1, b, (g, k), generator=gen)
    parent[0, 0] = -1
    if g > 1:
        parent[1, 0], parent[1, 1] = b, -(1 << 62)  # no beams: zeros, too
    n = g * b
    wide = torch.randn(n, 50, generator=gen)
    states = [torch.randn(n, 40, generator=gen), torch.randn(n, 7, generator=gen).to(torch.float16), torch.randint(0, 99, (n, 24), generator=gen, dtype=torch.int32),
              torch.randint(0, 9, (n,), generator=gen), torch.rand(n, 3, generator=gen) < 0.5, torch.randn(n, 2, 3, 5, generator=gen).to(torch.bfloat16),
              torch.randn(n, 0, generator=gen), wide[:, 3:40], torch.randn(n, 4096, generator=gen).to(torch.bfloat16)]
    states += [torch.randint(0, 255, (n, i + 1), generator=gen, dtype=torch.uint8) for i in range(19)]
    there = ((parent >= 0) & (parent < b)).view(-1)
    row = (torch.arange(g)[:, None] * b + parent.clamp(0, b - 1)).view(-1)
    dev = [a.cuda() if a.is_contiguous() else wide.cuda()[:, 3:40] for a in states]
    got = seq().beam_reorder(parent.cuda(), dev, beams=b)
    given = [torch.full_like(a, 1) for a in got]
    again = seq().beam_reorder(parent.cuda(), dev, beams=b, out=given)
    for a, o, u in zip(states, got, again):
        want = a[row].clone()
        want[~there] = 0
        assert torch.equal(o.cpu(), want) and torch.equal(u.cpu(), want) and o.dtype == a.dtype
    assert all(a is o and a._version == 1 for a, o in zip(given, again))


def test_captured_and_replayed_between_eager_work():
    gen, logits, score = make(3, 4, 20_000, "f32", 5)
    state = torch.randn(12, 33, generator=gen).cuda()

    def run():
        s, p, i, f = seq().beam_select(logits, score, 4, end=7)
        return s, p, i, f, seq().beam_reorder(p, [state], beams=4)[0]

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run()
    for _ in range(4):
        logits.copy_(torch.randn(logits.shape, generator=gen))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, run()):
            assert torch.equal(a, b)


def test_the_same_row_in_another_place_has_the_same_score():
    """A log sum depends on the row's values alone, not on where it lies: equal beams are equal."""
    v = 33_333
    row = torch.randn(v, generator=torch.Generator().manual_seed(2)).to(torch.float16)
    wide = torch.zeros(8, v + 3, dtype=torch.float16)
    wide[:, 1:1 + v] = row
    logits = wide.cuda()[:, 1:1 + v]
    s, p, i, _ = seq().beam_select(logits, torch.zeros(1, 8, device="cuda"), 8)
    assert p[0].tolist() == list(range(8)) and len(set(i[0].tolist())) == 1 and len(set(s[0].tolist())) == 1
