"""A small text classifier trained by simulated workers that send sparse signs: every operator of the library in one loop.

Each of the M workers holds texts of its own, in which some classes are more common than others (non-IID).  Per step

  1. s3gd_embed          looks the workers' tokens up in the embedding table,
  2. the model           averages a text's rows and applies two matrices (plain torch, gradients by autograd),
  3. s3gd_embed_grad     lays the table's gradient into each worker's row of the gradient buffer, the matrices' go beside it,
  4. s3gd_topk_sign, s3gd_majority_vote   turn the rows into one vote per coordinate,
  5. s3gd_apply          moves the table by the vote, and
     s3gd_step_ortho     moves each matrix by the orthogonalised momentum of its part of the vote.

    python examples/train_text_classifier.py [--steps 60] [--workers 8]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2302_07475_b200 as S  # noqa: E402

VOCAB, DIM, HIDDEN, CLASSES, LENGTH = 5000, 128, 256, 10, 24


def make_texts(workers, texts, seed, device):
    """Token ids [workers, texts, LENGTH] (-1: padding) and classes: a quarter of a text's words are its class's own."""
    gen = torch.Generator(device).manual_seed(seed)
    favourite = torch.randint(0, CLASSES, (workers, texts), generator=gen, device=device)
    own = torch.arange(workers, device=device)[:, None] % CLASSES
    labels = torch.where(torch.rand((workers, texts), generator=gen, device=device) < 0.4, own, favourite)
    shape = (workers, texts, LENGTH)
    common = (torch.rand(shape, generator=gen, device=device) ** 3 * VOCAB).long()
    special = VOCAB // 2 + labels[..., None] * 50 + torch.randint(0, 50, shape, generator=gen, device=device)
    ids = torch.where(torch.rand(shape, generator=gen, device=device) < 0.25, special, common)
    length = torch.randint(LENGTH // 2, LENGTH + 1, (workers, texts, 1), generator=gen, device=device)
    return torch.where(torch.arange(LENGTH, device=device) < length, ids, torch.full_like(ids, -1)), labels


def train(steps=60, workers=8, texts=64, keep=0.02, seed=0, device="cuda"):
    """Returns the mean loss over the workers before each step."""
    gen = torch.Generator(device).manual_seed(seed)
    sizes = (VOCAB * DIM, HIDDEN * DIM, CLASSES * HIDDEN)
    d = sum(sizes)
    x = torch.cat([torch.randn(n, generator=gen, device=device) * s for n, s in zip(sizes, (0.02, DIM ** -0.5, HIDDEN ** -0.5))])
    table, w1, w2 = (p.view(shape) for p, shape in zip(x.split(sizes), ((VOCAB, DIM), (HIDDEN, DIM), (CLASSES, HIDDEN))))
    v1, v2 = torch.zeros_like(w1), torch.zeros_like(w2)

    tokens = texts * LENGTH
    K = max(1, int(keep * d))
    grads = torch.empty((workers, d), device=device)
    idx = torch.empty((workers, K), dtype=torch.int32, device=device)
    signs = torch.empty((workers, (K + 31) // 32), dtype=torch.int32, device=device)
    vote = torch.empty(d, dtype=torch.int8, device=device)
    emb = torch.empty((workers, tokens, DIM), device=device)
    ws = S.alloc_workspace(workers, d, K, device)
    ws_embed = S.alloc_embed_workspace(workers, tokens, VOCAB, DIM, device)
    ws1, ws2 = S.alloc_ortho_workspace(1, HIDDEN, DIM, device), S.alloc_ortho_workspace(1, CLASSES, HIDDEN, device)
    scale, losses = math.sqrt(DIM), []

    for step in range(steps):
        ids, labels = make_texts(workers, texts, 1000 + step, device)
        flat = ids.view(workers, tokens)
        S.s3gd_embed(table, flat, emb, scale=scale)
        rows = emb.detach().requires_grad_()
        each1 = w1.expand(workers, -1, -1).clone().requires_grad_()          # a copy per worker: gradients of their own
        each2 = w2.expand(workers, -1, -1).clone().requires_grad_()
        there = (ids >= 0).sum(-1, keepdim=True)
        pooled = rows.view(workers, texts, LENGTH, DIM).sum(2) / there
        logits = torch.relu(pooled @ each1.mT) @ each2.mT
        loss = torch.nn.functional.cross_entropy(logits.reshape(-1, CLASSES), labels.reshape(-1), reduction="none").view(workers, texts).mean(1)
        loss.sum().backward()

        part = grads.split(sizes, dim=1)
        S.s3gd_embed_grad(rows.grad, flat, part[0], VOCAB, ws_embed, scale=scale)
        part[1].copy_(each1.grad.view(workers, -1))
        part[2].copy_(each2.grad.view(workers, -1))

        S.s3gd_topk_sign(grads, K, idx, signs, ws)
        S.s3gd_majority_vote(idx, signs, workers, K, d, vote, ws)
        table_vote, vote1, vote2 = vote.split(sizes)
        S.s3gd_apply(table.view(-1), table_vote, 2e-3)
        S.s3gd_step_ortho(w1, vote1.view_as(w1), 0.02, ws1, v=v1, mu=0.9, nesterov=False, weight_decay=0.01)
        S.s3gd_step_ortho(w2, vote2.view_as(w2), 0.02, ws2, v=v2, mu=0.9, nesterov=False, weight_decay=0.01)
        losses.append(loss.mean().detach())
    for w in (ws, ws_embed, ws1, ws2):
        S.s3gd_device_status(w)
    return [float(v) for v in losses]


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--workers", type=int, default=8)
    a = p.parse_args()
    history = train(a.steps, a.workers)
    for i in range(0, len(history), max(1, len(history) // 10)):
        print(f"step {i:4d}  loss {history[i]:.4f}")
    print(f"step {len(history) - 1:4d}  loss {history[-1]:.4f}   (chance: {math.log(CLASSES):.4f})")
