"""From ratings to choices: factors learned by CCD++ go on as a model of which item a user takes next.

1. CCD++ (Algorithm 3) factorises the rating matrix.
2. Mini-batches of (user, item) choices follow the gradient of the softmax cross entropy over the whole catalogue
   (softmax_loss_train), with the gradients' global norm clipped (clip_grads) before each step.  The offset is the log of
   an item's share of all ratings, so that the factors explain what popularity does not; items without any are excluded.
3. Held-out choices are judged by their mean loss over the catalogue (softmax_loss).

    python examples/choose_items.py [--users 6041 --items 3707 --ratings 1000209 --k 40 --steps 200 --batch 1024]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1511_02433_amd import ops  # noqa: E402
from paper_1511_02433_amd.ccdpp import CCDPP  # noqa: E402


def make_ratings(users, items, ratings, seed):
    """Triplets with distinct positions; items by a power law; what a user takes, and how it is rated, by a latent score."""
    rng = np.random.default_rng(seed)
    u, v = rng.normal(size=(users, 8)), rng.normal(size=(items, 8)) / 8 ** 0.5
    row = rng.integers(0, users, 6 * ratings)
    col = (items * rng.random(6 * ratings) ** 2.5).astype(np.int64)
    score = (u[row] * v[col]).sum(1)
    taken = rng.random(row.size) < 1 / (1 + np.exp(-3 * (score - 0.5)))
    at = rng.permutation(np.unique(row[taken] * items + col[taken]))[:ratings]
    row, col = (at // items).astype(np.int32), (at % items).astype(np.int32)
    val = np.clip(np.round(3 + (u[row] * v[col]).sum(1)), 1, 5).astype(np.float32)
    return row, col, val


def main(argv=None):
    p = argparse.ArgumentParser()
    for name, value in (("users", 6041), ("items", 3707), ("ratings", 1_000_209), ("k", 40), ("steps", 200), ("batch", 1024),
                        ("seed", 1)):
        p.add_argument("--" + name, type=int, default=value)
    p.add_argument("--rate", type=float, default=0.5)
    p.add_argument("--max-norm", type=float, default=0.25)
    a = p.parse_args(argv)
    row, col, val = make_ratings(a.users, a.items, a.ratings, a.seed)
    liked = np.flatnonzero(val >= 4)
    test, train = liked[::20], np.setdiff1d(liked, liked[::20])

    with CCDPP(a.users, a.items, a.k, 0.05, row, col, val) as model:
        model.use_torch_stream()
        model.run(5, 3)
        W, H = model.factors()
        print(f"CCD++: training RMSE {model.train_rmse():.4f}")

    W, H = torch.from_numpy(W).cuda(), torch.from_numpy(H).cuda()
    rows, cols = torch.from_numpy(row.astype(np.int64)).cuda(), torch.from_numpy(col.astype(np.int64)).cuda()
    count = torch.bincount(cols, minlength=a.items).float()
    offset = torch.log(count / count.sum())  # -inf where an item was never rated: it is excluded
    # The softmax sees neither what all items share nor how a product is shared out between W and H.
    H -= (count / count.sum()) @ H
    ratio = (W.square().mean() / H.square().mean()).sqrt().sqrt()
    W, H = W / ratio, H * ratio

    def held_out():
        at = torch.from_numpy(test).cuda()
        loss, _ = ops.softmax_loss(W[rows[at]], H, cols[at], offset=offset)
        return float(loss[torch.isfinite(loss)].mean())

    first = held_out()
    gen = torch.Generator().manual_seed(a.seed)
    weight = torch.full((a.batch,), 1.0 / a.batch, device="cuda")
    for step in range(a.steps):
        at = torch.from_numpy(train)[torch.randint(len(train), (a.batch,), generator=gen)].cuda()
        users = rows[at]
        loss, _, dx, dH = ops.softmax_loss_train(W[users], H, cols[at], grad=weight, offset=offset)
        norm = ops.clip_grads([dx, dH], a.max_norm)
        W.index_add_(0, users, dx, alpha=-a.rate)
        H.add_(dH, alpha=-a.rate)
        if (step + 1) % max(1, a.steps // 5) == 0:
            print(f"step {step + 1}: training loss {float(loss.mean()):.4f}, gradient norm {float(norm):.4f}", flush=True)
    last = held_out()
    print(f"held-out loss over {a.items} items: {first:.4f} -> {last:.4f}")
    return first, last


if __name__ == "__main__":
    main()
