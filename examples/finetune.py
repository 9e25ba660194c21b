"""Finetunes the adapters of two decomposed layers on synthetic data: decompose W ~ Q + L1 L2, keep Q as it is stored, train L1, L2.

A token's row of a fixed embedding goes through two layers with a rectifier between them and meets the rows of a fixed output matrix:
the cross entropy of the target token over the vocabulary is what falls.  Targets are a fixed permutation of the tokens.  A step is

    x = drop(E[tokens])                                    lq.dropout
    y, t = x Q + (drop(x) L1) L2, twice                     lq.adapter_forward
    loss, dX over the vocabulary                            lq.cross_entropy
    dX, dL1, dL2, twice                                     lq.adapter_backward

with a mask of its own for every step and place: the seed names the step, the offset the place.  Workspaces are made once.  The update is
written out in torch, or with --bits 32 or 8 (of the optimizer's states) it is

    norm of all gradients, factor that clips them           lq.grad_norm
    the update of all factors                               lq.AdamW

    python examples/finetune.py --steps 60 --dtype bf16 --bits 8
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2311_12023_amd import lq  # noqa: E402


class Adam:
    def __init__(self, params, lr):
        self.params, self.lr, self.step_count = params, lr, 0
        self.m = [torch.zeros_like(p) for p in params]
        self.v = [torch.zeros_like(p) for p in params]

    def step(self, grads):
        self.step_count += 1
        for p, g, m, v in zip(self.params, grads, self.m, self.v):
            m.mul_(0.9).add_(g, alpha=0.1)
            v.mul_(0.99).addcmul_(g, g, value=0.01)
            size = (v / (1 - 0.99 ** self.step_count)).sqrt_().add_(1e-8)
            p.addcdiv_(m, size, value=-self.lr / (1 - 0.9 ** self.step_count))


class ClippedAdamW:
    """The library's step over all factors at once, gradients clipped to a norm of 1."""

    def __init__(self, params, lr, bits):
        self.adamw, self.lr = lq.AdamW(params, bits=bits), lr

    def step(self, grads):
        _, coef = lq.grad_norm(grads, 1.0)
        self.adamw.step(grads, self.lr, betas=(0.9, 0.99), weight_decay=0.0, coef=coef)


class Layer:
    """A decomposed d x k matrix, its adapter and what its calls need."""

    def __init__(self, w, rank, cfg, rows, dtype, place):
        d, k = w.shape
        dec = lq.decompose(w, rank, cfg, 2)
        self.cfg, self.q = cfg, (dec["codes"], dec["scale_idx"], dec["v"])
        self.l1, self.l2 = dec["L1"], dec["L2"]
        self.offset = place << 32
        self.ws = [lq.adapter_workspace(rows, d, k, rank, dtype, backward) for backward in (False, True)]

    def forward(self, x, p, step):
        self.x, self.drop = x, (p, step, self.offset)
        y, self.t = lq.adapter_forward(x, *self.q, self.cfg, self.l1, self.l2, *self.drop, workspace=self.ws[0])
        return y

    def backward(self, dy, want_dx):
        return lq.adapter_backward(dy, self.x, *self.q, self.cfg, self.l1, self.l2, self.t, *self.drop, want_dx=want_dx,
                                   workspace=self.ws[1])


def finetune(steps=60, dtype=torch.float32, rows=200, width=256, hidden=512, vocab=1000, rank=16, p=0.05, lr=4e-3, seed=0,
             device="cuda", bits=None):
    """-> the loss of every step.  bits: None, or those of lq.AdamW's states."""
    gen = torch.Generator().manual_seed(seed)

    def normal(*shape, std):
        return (torch.randn(*shape, generator=gen) * std).to(device)

    cfg = lq.config(4, 32, 64)
    embedding = normal(vocab, width, std=1.0).to(dtype)
    output = normal(vocab, width, std=width ** -0.5).to(dtype)
    layers = [Layer(normal(width, hidden, std=width ** -0.5), rank, cfg, rows, dtype, 1),
              Layer(normal(hidden, width, std=hidden ** -0.5), rank, cfg, rows, dtype, 2)]
    tokens = torch.randperm(vocab, generator=gen)[:rows].to(device)
    targets = torch.randperm(vocab, generator=gen).to(device)[tokens]
    loss_ws = lq.cross_entropy_workspace(rows, width, vocab, dtype)
    factors = [w for layer in layers for w in (layer.l1, layer.l2)]
    adam = Adam(factors, lr) if bits is None else ClippedAdamW(factors, lr, bits)
    losses = []
    for step in range(steps):
        x = lq.dropout(embedding[tokens], p, seed=step)
        h = layers[0].forward(x, p, step).relu_()
        y = layers[1].forward(h, p, step)
        out = lq.cross_entropy(y, output, targets, workspace=loss_ws)
        losses.append(out["loss"])
        dh, dl1_b, dl2_b = layers[1].backward(out["dx"], want_dx=True)
        _, dl1_a, dl2_a = layers[0].backward(dh * (h > 0), want_dx=False)
        adam.step([dl1_a, dl2_a, dl1_b, dl2_b])
    return torch.stack([v.reshape(()) for v in losses]).tolist()


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--dtype", choices=("fp32", "bf16"), default="fp32")
    ap.add_argument("--bits", type=int, choices=(8, 32), default=None)
    a = ap.parse_args()
    losses = finetune(a.steps, torch.bfloat16 if a.dtype == "bf16" else torch.float32, bits=a.bits)
    for i in range(0, len(losses), 10):
        print(f"step {i:4d}  loss {losses[i]:.4f}")
    print(f"step {len(losses) - 1:4d}  loss {losses[-1]:.4f}")


if __name__ == "__main__":
    main()
