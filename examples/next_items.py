"""From ratings to what a user takes next: factors learned by CCD++ go on as a model of sequences.

1. CCD++ (Algorithm 3) factorises the rating matrix; each user's liked items, in the order in which they were taken, are one
   sequence of a packed batch.
2. A gated recurrence (gated_scan) turns the factors of the items so far into the row that chooses the next one among all
   (softmax_loss_train), with dropout between them.  Its gradients go back through dropout and the recurrence to the items' factors
   and gates, clipped together (clip_grads).
3. Held-out steps are judged by their mean loss over the catalogue.  For a user, the recurrence's last state answers with the best
   next items in sequence: beams over the catalogue (beam_select), their states in order (beam_reorder), one more row of each
   (gated_scan_step).

    python examples/next_items.py [--users 6041 --items 3707 --ratings 1000209 --k 40 --steps 100 --batch 256]
"""
import argparse
import math
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from examples.choose_items import make_ratings  # noqa: E402
from paper_1511_02433_amd import ops, seq  # noqa: E402
from paper_1511_02433_amd.ccdpp import CCDPP  # noqa: E402


def pack(sequences):
    """(items, next, starts) of a batch on the GPU: each row's item, the one after it (-1 behind a sequence's last), where sequences begin."""
    lengths = [len(s) for s in sequences]
    items = np.concatenate(sequences) if sequences else np.zeros(0, np.int64)
    following = np.concatenate([np.append(s[1:], -1) if len(s) else s for s in sequences])
    starts = np.concatenate([[0], np.cumsum(lengths)])
    return tuple(torch.from_numpy(a.astype(np.int64)).cuda() for a in (items, following, starts))


def gradients(H, G, offset, batch, p, seed):
    """The mean loss of the batch's steps, and its gradients by the items' factors H and gates G."""
    items, following, starts = batch
    weight = (following >= 0).float() / (following >= 0).sum().clamp(min=1)
    x, gate = H[items], G[items]
    h, _, kept = seq.gated_scan(x, gate, starts=starts, keep=True)
    loss, _, dz, dH = ops.softmax_loss_train(seq.dropout(h, p, seed), H, following, grad=weight, offset=offset)
    dx, dgate, _ = seq.gated_scan_grad(x, gate, seq.dropout(dz, p, seed), kept, starts=starts)
    dH.index_add_(0, items, dx)
    dG = torch.zeros_like(G).index_add_(0, items, dgate)
    return (loss * weight).sum(), dH, dG


def judge(H, G, offset, batch):
    items, following, starts = batch
    h, last = seq.gated_scan(H[items], G[items], starts=starts)
    loss, _ = ops.softmax_loss(h, H, following, offset=offset)
    use = (following >= 0) & torch.isfinite(loss)
    return float(loss[use].mean()), last


def answer(H, G, offset, state, beams, length):
    """The best `length` next items for each row of states: (scores, items), g x beams and g x beams x length."""
    g = state.shape[0]
    state = state.repeat_interleave(beams, 0)
    taken = torch.zeros(g * beams, 0, dtype=torch.int64, device="cuda")
    score = torch.full((g, beams), -math.inf, device="cuda")
    score[:, 0] = 0.0
    for _ in range(length):
        score, parent, item, _ = seq.beam_select(state @ H.T, score, beams, offset=offset)
        state, taken = seq.beam_reorder(parent, [state, taken], beams=beams)
        item = item.view(-1).clamp(min=0)
        taken = torch.cat([taken, item[:, None]], 1)
        seq.gated_scan_step(H[item], G[item], state)
    return score, taken.view(g, beams, length)


def main(argv=None):
    p = argparse.ArgumentParser()
    for name, value in (("users", 6041), ("items", 3707), ("ratings", 1_000_209), ("k", 40), ("steps", 100), ("batch", 256), ("seed", 1)):
        p.add_argument("--" + name, type=int, default=value)
    p.add_argument("--rate", type=float, default=200.0)
    p.add_argument("--dropout", type=float, default=0.1)
    p.add_argument("--max-norm", type=float, default=0.25)
    a = p.parse_args(argv)
    row, col, val = make_ratings(a.users, a.items, a.ratings, a.seed)
    with CCDPP(a.users, a.items, a.k, 0.05, row, col, val) as model:
        model.use_torch_stream()
        model.run(5, 3)
        H = torch.from_numpy(model.factors()[1]).cuda()
        print(f"CCD++: training RMSE {model.train_rmse():.4f}")

    # A user takes what many take first, more or less.
    rng = np.random.default_rng(a.seed)
    count = np.bincount(col, minlength=a.items)
    liked = np.flatnonzero(val >= 4)
    liked = liked[np.lexsort((-np.log(count[col[liked]]) + 0.5 * rng.normal(size=liked.size), row[liked]))]
    sequences = np.split(col[liked].astype(np.int64), np.searchsorted(row[liked], np.arange(1, a.users)))
    test, train = pack(sequences[::20]), [s for i, s in enumerate(sequences) if i % 20 and len(s) > 1]

    share = torch.from_numpy(count).cuda().float() / count.sum()
    offset = torch.log(share)  # -inf where an item was never rated: it is excluded
    H = H - share @ H  # (the softmax does not see what all items share)
    H *= 0.3 / H.square().mean().sqrt()
    G = torch.full_like(H, 2.0)
    first, _ = judge(H, G, offset, test)
    for step in range(a.steps):
        batch = pack([train[i] for i in rng.integers(0, len(train), a.batch)])
        loss, dH, dG = gradients(H, G, offset, batch, a.dropout, step)
        norm = ops.clip_grads([dH, dG], a.max_norm)
        H.add_(dH, alpha=-a.rate), G.add_(dG, alpha=-a.rate)
        if (step + 1) % max(1, a.steps // 5) == 0:
            print(f"step {step + 1}: training loss {float(loss):.4f}, gradient norm {float(norm):.4f}", flush=True)
    last, state = judge(H, G, offset, test)
    print(f"held-out loss of the next item among {a.items}: {first:.4f} -> {last:.4f}")
    score, items = answer(H, G, offset, state[:4].contiguous(), 4, 3)
    for u in range(items.shape[0]):
        print(f"user {20 * u}: next {items[u, 0].tolist()} (log probability {float(score[u, 0]):.2f}), or {items[u, 1].tolist()}")
    return first, last, score, items


if __name__ == "__main__":
    main()
