"""A text classifier with a residual block and layer norms, trained by simulated workers that clip their gradients and remember
what they did not send.

Each of the M workers holds texts of its own.  Per step

  1. s3gd_embed             looks the workers' tokens up in the embedding table,
  2. s3gd_layer_norm        normalises their rows (padding stays zero),
  3. the model              averages a text's rows and puts the result through two matrices (plain torch, gradients by autograd),
  4. s3gd_layer_norm        adds the block's result to what went in and normalises the sum; a third matrix gives the classes,
  5. s3gd_layer_norm_grad, s3gd_embed_grad   lay the norms' and the table's gradients into each worker's row of the gradient buffer,
  6. s3gd_clip              takes each worker's norm over all tensors and scales it into its row: the matrices' gradients come from
                            where autograd left them, the others lie there already,
  7. s3gd_step_ex           adds the error memory, keeps the largest entries' signs, votes and moves the parameters.

    python examples/train_residual_classifier.py [--steps 60] [--workers 8]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2302_07475_b200 as S  # noqa: E402
from train_text_classifier import CLASSES, LENGTH, VOCAB, make_texts  # noqa: E402

DIM, HIDDEN, EPS = 96, 192, 1e-5
SHAPES = {"table": (VOCAB, DIM), "w1": (HIDDEN, DIM), "w2": (DIM, HIDDEN), "w3": (CLASSES, DIM), "scale1": (DIM,), "shift1": (DIM,),
          "scale2": (DIM,), "shift2": (DIM,)}
SIZES = [math.prod(s) for s in SHAPES.values()]


def parameters(seed, device):
    """The flat parameters, and a view of each by its name."""
    gen = torch.Generator(device).manual_seed(seed)
    x = torch.cat([torch.randn(n, generator=gen, device=device) * (0.02 if k == "table" else s[-1] ** -0.5)
                   for (k, s), n in zip(SHAPES.items(), SIZES)])
    views = {k: p.view(s) for (k, s), p in zip(SHAPES.items(), x.split(SIZES))}
    for k in ("scale1", "scale2"):
        views[k].fill_(1.0)
    for k in ("shift1", "shift2"):
        views[k].zero_()
    return x, views


class Workers:
    """The buffers of M workers with `texts` texts each, and their gradients for a batch."""

    def __init__(self, workers, texts, device):
        self.M, self.texts = workers, texts
        tokens = texts * LENGTH
        self.grads = torch.empty((workers, sum(SIZES)), device=device)
        self.parts = dict(zip(SHAPES, self.grads.split(SIZES, dim=1)))
        self.emb, self.y, self.demb = (torch.empty((workers, tokens, DIM), device=device) for _ in range(3))
        self.total, self.z, self.dtotal = (torch.empty((workers, texts, DIM), device=device) for _ in range(3))
        self.norm = torch.empty(workers, device=device)
        self.ws_embed = S.alloc_embed_workspace(workers, tokens, VOCAB, DIM, device)
        self.ws_norm = S.alloc_layer_norm_workspace(workers, tokens, DIM, device)       # serves the texts' rows too
        self.ws_clip = S.alloc_clip_workspace(workers, device)

    def gradients(self, p, ids, labels, max_norm):
        """Each worker's clipped gradient in its row of self.grads, its norm before that in self.norm; returns the workers' losses."""
        M, texts, parts = self.M, self.texts, self.parts
        flat = ids.view(M, texts * LENGTH)
        S.s3gd_embed(p["table"], flat, self.emb)
        S.s3gd_layer_norm(self.emb, self.y, p["scale1"], p["shift1"], EPS, ids=flat)
        each = {k: p[k].expand(M, -1, -1).clone().requires_grad_() for k in ("w1", "w2", "w3")}     # a copy per worker
        rows = self.y.requires_grad_()
        pooled = rows.view(M, texts, LENGTH, DIM).sum(2) / (ids >= 0).sum(-1, keepdim=True)
        block = torch.relu(pooled @ each["w1"].mT) @ each["w2"].mT
        S.s3gd_layer_norm(block.detach(), self.z, p["scale2"], p["shift2"], EPS, add=pooled.detach(), total=self.total)
        top = self.z.requires_grad_()
        logits = top @ each["w3"].mT
        loss = torch.nn.functional.cross_entropy(logits.reshape(-1, CLASSES), labels.reshape(-1), reduction="none").view(M, texts).mean(1)
        loss.sum().backward()
        S.s3gd_layer_norm_grad(top.grad, self.total, self.dtotal, p["scale2"], parts["scale2"], parts["shift2"], self.ws_norm, EPS)
        torch.autograd.backward([block, pooled], [self.dtotal, self.dtotal])            # the sum's gradient goes both ways
        S.s3gd_layer_norm_grad(rows.grad, self.emb, self.demb, p["scale1"], parts["scale1"], parts["shift1"], self.ws_norm, EPS, ids=flat)
        S.s3gd_embed_grad(self.demb, flat, parts["table"], VOCAB, self.ws_embed)
        for t in (rows, top):
            t.grad = None
            t.requires_grad_(False)
        found = [each[k].grad if k in each else parts[k] for k in SHAPES]
        S.s3gd_clip(found, max_norm, self.norm, self.ws_clip, out=[parts[k].view(M, *f.shape[1:]) if k not in each else parts[k].unflatten(1, SHAPES[k])
                                                                   for k, f in zip(SHAPES, found)])
        return loss.detach()


def train(steps=60, workers=8, texts=64, keep=0.02, max_norm=1.0, lr=2e-3, seed=0, device="cuda"):
    """Returns the mean loss over the workers before each step."""
    x, p = parameters(seed, device)
    d = x.numel()
    K = max(1, int(keep * d))
    w = Workers(workers, texts, device)
    memory, ws, losses = torch.zeros_like(w.grads), S.alloc_workspace(workers, d, K, device), []
    for step in range(steps):
        ids, labels = make_texts(workers, texts, 1000 + step, device)
        losses.append(w.gradients(p, ids, labels, max_norm).mean())
        S.s3gd_step_ex(x, w.grads, K, lr, ws, err=memory, eta=1.0)
    for t in (ws, w.ws_embed, w.ws_norm, w.ws_clip):
        S.s3gd_device_status(t)
    return [float(v) for v in losses]


if __name__ == "__main__":
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    a.add_argument("--steps", type=int, default=60)
    a.add_argument("--workers", type=int, default=8)
    a = a.parse_args()
    history = train(a.steps, a.workers)
    for i in range(0, len(history), max(1, len(history) // 10)):
        print(f"step {i:4d}  loss {history[i]:.4f}")
    print(f"step {len(history) - 1:4d}  loss {history[-1]:.4f}   (chance: {math.log(CLASSES):.4f})")
