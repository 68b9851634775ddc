"""Adapting an encoder to several collections at once, and serving them from one weight.

Two post-LN sublayers, x <- LayerNorm(x + dropout(x W^T + bias + its collection's adapter)), stand for an encoder's.  W stays as it is; the adapters of
three collections and the LayerNorms' scale and shift learn what a teacher does, whose weights differ from W by a low-rank matrix per collection.  Then
requests of all collections, and some of none, go through in one call.

    python examples/adapt_block.py
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np
import torch

import paper_2506_08276_amd as L

DEV, HIDDEN, RANK, EPS = "cuda:0", 384, 16, 1e-12
COLLECTIONS, TEACHER_RANK = 3, 4
SCALE = [1.0] * COLLECTIONS


class Sublayer:
    """W and bias, frozen; per collection down [rank][hidden] and up [hidden][rank]; LayerNorm's scale and shift.  What learns is kept in fp32 and handed
    to the projection in bf16."""

    def __init__(self, ctx, g, w, gradient):
        self.ctx, self.w = ctx, w.bfloat16()
        self.proj = L.leann_projection_create(ctx, self.w, torch.zeros(HIDDEN, device=DEV), gradient=gradient)
        self.params = {"down": torch.randn((COLLECTIONS, RANK, HIDDEN), generator=g, device=DEV) / HIDDEN ** 0.5,
                       "up": torch.zeros((COLLECTIONS, HIDDEN, RANK), device=DEV),
                       "gamma": torch.ones(HIDDEN, device=DEV), "beta": torch.zeros(HIDDEN, device=DEV)}

    def forward(self, rows, x, drop=None, keep=False):
        p = self.params
        self.half = p["down"].bfloat16(), p["up"].bfloat16()
        branch = L.leann_adapter_project(self.ctx, self.proj, rows, x, *self.half, keep=keep)
        if not keep:
            return L.leann_layernorm(self.ctx, branch, p["gamma"], p["beta"], EPS, residual=x)
        branch, low = branch
        out, *stats = L.leann_layernorm(self.ctx, branch, p["gamma"], p["beta"], EPS, residual=x, drop=drop, keep=True)
        self.kept = rows, x, low, stats, drop
        return out

    def backward(self, dout, need_dx):
        """(gradients of the parameters, the two ways' gradients of x)."""
        rows, x, low, stats, drop = self.kept
        dres, dbranch, dgamma, dbeta = L.leann_layernorm_backward(self.ctx, dout, *stats, self.params["gamma"], drop=drop)
        dx, ddown, dup = L.leann_adapter_project_backward(self.ctx, self.proj, rows, dbranch, x, low, *self.half, need_dx=need_dx)
        return {"down": ddown, "up": dup, "gamma": dgamma, "beta": dbeta}, (dres, dx)

    def close(self):
        L.leann_projection_free(self.proj)


class Adam:
    """Adam without weight decay; a step's gradients are what the sublayer's backward pass returned."""

    def __init__(self, params, rate):
        self.params, self.rate, self.t = params, rate, 0
        self.moments = {k: (torch.zeros_like(v), torch.zeros_like(v)) for k, v in params.items()}

    def step(self, grads):
        self.t += 1
        for k, g in grads.items():
            m, v = self.moments[k]
            m.lerp_(g, 0.1)
            v.lerp_(g * g, 0.01)
            self.params[k] -= self.rate * (m / (1 - 0.9 ** self.t)) / ((v / (1 - 0.99 ** self.t)).sqrt() + 1e-12)


def normalise(t):
    c = t - t.mean(1, keepdim=True)
    return c / ((c * c).mean(1, keepdim=True) + EPS).sqrt()


def main(steps=60, p=0.05):
    g = torch.Generator(device=DEV).manual_seed(7)
    rng = np.random.default_rng(7)
    ctx = L.leann_create(dict(layers=0, hidden=128, heads=2, ffn=128, vocab=1, max_pos=1), torch.zeros(640, device=DEV))
    weights = [0.05 * torch.randn((HIDDEN, HIDDEN), generator=g, device=DEV) for _ in range(2)]
    change = [[0.05 * torch.randn((HIDDEN, TEACHER_RANK), generator=g, device=DEV) @ torch.randn((TEACHER_RANK, HIDDEN), generator=g, device=DEV)
               for _ in range(COLLECTIONS)] for _ in range(2)]
    layers = [Sublayer(ctx, g, w, gradient=i > 0) for i, w in enumerate(weights)]
    optimizers = [Adam(l.params, 5e-3) for l in layers]

    lengths = rng.integers(8, 129, 48)  # chunks of a training batch
    of = rng.integers(0, COLLECTIONS, 48)
    rows = L.leann_adapter_rows_create(ctx, lengths, of, [RANK] * COLLECTIONS, SCALE, RANK)
    collection_of_row = torch.from_numpy(np.repeat(of, lengths)).to(DEV)
    losses = []
    for step in range(steps):
        x = normalise(torch.randn((rows.T, HIDDEN), generator=g, device=DEV)).bfloat16()
        target = x.float()
        for w, c in zip(layers, change):
            branch = target @ w.w.float().t()
            for a in range(COLLECTIONS):
                mine = collection_of_row == a
                branch[mine] += target[mine] @ c[a].t()
            target = normalise(target + branch)
        h = x
        for i, layer in enumerate(layers):
            h = layer.forward(rows, h, drop=(p, 2024 + i, step), keep=True)  # a mask per layer (seed) and step (offset)
        error = h.float() - target
        losses.append(error.square().mean().item())
        dout = (error / rows.T).bfloat16()
        for i in (1, 0):
            grads, (dres, dx) = layers[i].backward(dout, need_dx=i > 0)
            optimizers[i].step(grads)
            if i:
                dout = dres + dx
    L.leann_adapter_rows_free(rows)

    # Serving: requests of every collection and of none, a single token or a few, in one call; each as by itself.
    lengths, of = rng.integers(1, 20, 30), rng.integers(-1, COLLECTIONS, 30)
    lengths[:10] = 1
    x = normalise(torch.randn((int(lengths.sum()), HIDDEN), generator=g, device=DEV)).bfloat16()

    def serve(lengths, of, x):
        rows = L.leann_adapter_rows_create(ctx, lengths, of, [RANK] * COLLECTIONS, SCALE, RANK)
        h = layers[1].forward(rows, layers[0].forward(rows, x))
        L.leann_adapter_rows_free(rows)
        return h

    together = serve(lengths, of, x)
    starts = np.concatenate([[0], np.cumsum(lengths)])
    apart = torch.cat([serve(lengths[i:i + 1], of[i:i + 1], x[starts[i]:starts[i + 1]]) for i in range(30)])
    difference = (together.float() - apart.float()).abs().max().item()
    for layer in layers:
        layer.close()
    L.leann_destroy(ctx)
    return losses, difference


if __name__ == "__main__":
    losses, difference = main()
    print("loss by step:", " ".join(f"{v:.4f}" for v in losses[::6] + losses[-1:]))
    print(f"30 requests in one call against 30 calls: largest difference {difference:.2e}")
