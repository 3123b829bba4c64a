"""The operators on sequences together with the softmax loss over all items and clipping, as a program uses them: training on what
users took one after another, and answering with several items in sequence."""
import itertools
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


def modules():
    from paper_1511_02433_amd import ops, seq
    return ops, seq


def train_step(H, G, items, starts, target, weight, p, seed, max_norm=None):
    """Loss per row and the gradients of the item factors H and the gates' table G: each row takes the item before its target."""
    ops, seq = modules()
    x, gate = H[items], G[items]
    h, last, kept = seq.gated_scan(x, gate, starts=starts, keep=True)
    z = seq.dropout(h, p, seed)
    loss, _, dz, dH = ops.softmax_loss_train(z, H, target, grad=weight)
    dh = seq.dropout(dz, p, seed)
    dx, dgate, _ = seq.gated_scan_grad(x, gate, dh, kept, starts=starts)
    dH.index_add_(0, items, dx)
    dG = torch.zeros_like(G).index_add_(0, items, dgate)
    if max_norm is not None:
        ops.clip_grads([dH, dG], max_norm)
    return loss, dH, dG


def test_a_training_step_against_autograd_in_64_bits():
    """The same model by torch's operators and autograd on the host, in 64 bits, with the mask that the call drew.  Its parts are
    held to bounds of their own in their tests; together they are within 1e-4 of the largest gradient (22 bits of the softmax's terms,
    a few hundred rows each)."""
    _, seq = modules()
    gen = torch.Generator().manual_seed(0)
    v, d, n = 300, 24, 411
    starts = torch.tensor([0, 0, 100, 101, 130, 400, 405])  # six rows behind the last sequence
    items = torch.randint(0, v, (n,), generator=gen)
    target = torch.randint(0, v, (n,), generator=gen)
    target[starts[1:][starts[1:] > starts[:-1]] - 1] = -1  # nothing follows
    target[405:] = -1
    H, G = torch.randn(v, d, generator=gen) * 0.5, torch.randn(v, d, generator=gen)
    weight = torch.full((n,), 1.0 / n)
    p, seed = 0.2, 77
    loss, dH, dG = train_step(H.cuda(), G.cuda(), items.cuda(), starts.cuda(), target.cuda(), weight.cuda(), p, seed)
    mask = (seq.dropout(torch.ones(n, d, device="cuda"), p, seed) != 0).cpu().double()

    H64, G64 = H.double().requires_grad_(), G.double().requires_grad_()
    x, g = H64[items], G64[items]
    a = torch.sigmoid(g)
    rows = []
    for q in range(len(starts) - 1):
        h = torch.zeros(d, dtype=torch.float64)
        for t in range(int(starts[q]), int(starts[q + 1])):
            h = a[t] * h + (1 - a[t]) * x[t]
            rows.append(h)
    h = torch.cat([torch.stack(rows), torch.zeros(n - 405, d, dtype=torch.float64)])
    z = h * mask / (1 - p)
    logits = z @ H64.T
    use = target >= 0
    want = torch.zeros(n, dtype=torch.float64)
    want[use] = torch.logsumexp(logits[use], 1) - logits[use].gather(1, target[use, None])[:, 0]
    (want * weight).sum().backward()
    assert float((loss.cpu() - want.detach()).abs().max()) <= 1e-5 * float(want.detach().abs().max())
    for got, ref in ((dH, H64.grad), (dG, G64.grad)):
        assert float((got.cpu() - ref).abs().max()) <= 1e-4 * float(ref.abs().max())


def test_a_captured_training_step_draws_a_mask_for_each_replay():
    gen = torch.Generator().manual_seed(1)
    v, d, n = 500, 40, 700
    starts = torch.tensor([0, 250, 260, 700]).cuda()
    items, target = (torch.randint(0, v, (n,), generator=gen).cuda() for _ in range(2))
    H, G = torch.randn(v, d, generator=gen).cuda(), torch.randn(v, d, generator=gen).cuda()
    weight, seed = torch.full((n,), 1.0 / n, device="cuda"), torch.tensor([3], device="cuda")
    _, seq = modules()

    def run(seed):
        ops, _ = modules()
        x, gate = H[items], G[items]
        h, _, kept = seq.gated_scan(x, gate, starts=starts, keep=True)
        loss, _, dz, dH = ops.softmax_loss_train(seq.dropout(h, 0.3, seed), H, target, grad=weight)
        return (loss, dH) + seq.gated_scan_grad(x, gate, seq.dropout(dz, 0.3, seed), kept, starts=starts)[:2]

    run(seed)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run(seed)
    for s in (9, 10, 9):
        seed.fill_(s)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, run(s)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("k", [1, 3, 6])
def test_beams_answer_with_the_best_sequences(k):
    """Three items in sequence: with as many beams as there are pairs, beam search is exhaustive, and its answers are the best of
    all sequences by their log probability in 64 bits; with fewer it is the same search by hand."""
    _, seq = modules()
    gen = torch.Generator().manual_seed(k)
    v, d = 6, 8
    H, G = torch.randn(v, d, generator=gen), torch.randn(v, d, generator=gen)
    first = torch.randn(1, d, generator=gen)

    def step64(state, item):
        a = torch.sigmoid(G[item].double())
        return a * state + (1 - a) * H[item].double()

    def logp(state):
        z = state @ H.double().T
        return z - torch.logsumexp(z, -1)

    # by hand
    beams = [(0.0, (), first[0].double())]
    for _ in range(3):
        found = [(s + float(logp(state)[i]), items + (i,), state) for s, items, state in beams for i in range(v)]
        found.sort(key=lambda c: -c[0])
        beams = [(s, items, step64(state, items[-1])) for s, items, state in found[:k]]

    Hc, Gc = H.cuda(), G.cuda()
    state = first.repeat(k, 1).cuda()
    score = torch.full((1, k), -math.inf, device="cuda")
    score[0, 0] = 0.0
    taken = torch.zeros(k, 0, dtype=torch.int64, device="cuda")
    for _ in range(3):
        score, parent, item, _ = seq.beam_select(state @ Hc.T, score, k)
        state, taken = seq.beam_reorder(parent, [state, taken], beams=k)
        taken = torch.cat([taken, item.view(-1, 1)], 1)
        seq.gated_scan_step(Hc[item.view(-1).clamp(min=0)], Gc[item.view(-1).clamp(min=0)], state)
    assert [tuple(t) for t in taken.tolist()] == [b[1] for b in beams]
    assert all(abs(a - b[0]) <= 1e-5 for a, b in zip(score[0].tolist(), beams))
    if k == 6:  # the first answer of a wide search is at least as good as the greedy one
        assert beams[0][0] <= max(s for s in (_total(step64, logp, first[0].double(), items) for items in itertools.product(range(v), repeat=3))) + 1e-12


def _total(step, logp, state, items):
    s = 0.0
    for i in items:
        s += float(logp(state)[i])
        state = step(state, i)
    return s
