"""A training step through an encoder's whole block: projections with adapters, attention with learned relative positions, LayerNorm, GELU kept in 8 bits, forward and
backward together, against the same block in 64 bits."""
import math

import numpy as np
import pytest

from gpu_util import say

pytestmark = pytest.mark.gpu
CTX = dict(layers=0, hidden=128, heads=2, ffn=128, vocab=1, max_pos=1)
HIDDEN, HEADS, FFN, RANK, EPS, BUCKETS, DISTANCE = 128, 4, 384, 8, 1e-12, 16, 40
DEV = "cuda:0"


class Block:
    """Weights, adapters of two collections (one projection's are enough: the attention's output), LayerNorms and the bias; what learns is fp32."""

    def __init__(self, ctx, L, g):
        import torch
        self.ctx, self.L = ctx, L
        r = lambda *s, scale=1.0: scale * torch.randn(s, generator=g, device=DEV)
        self.w = {k: r(*s, scale=s[1] ** -0.5).half() for k, s in
                  {"qkv": (3 * HIDDEN, HIDDEN), "o": (HIDDEN, HIDDEN), "up": (FFN, HIDDEN), "down": (HIDDEN, FFN)}.items()}
        self.proj = {k: L.leann_projection_create(ctx, w, r(w.shape[0], scale=0.1), gradient=True) for k, w in self.w.items()}
        self.params = {"bias": r(BUCKETS, HEADS), "g1": 1 + r(HIDDEN, scale=0.1), "b1": r(HIDDEN, scale=0.1), "g2": 1 + r(HIDDEN, scale=0.1), "b2": r(HIDDEN, scale=0.1)}
        self.adapters = {k: ((r(2, RANK, w.shape[1]) / w.shape[1] ** 0.5).half(), r(2, w.shape[0], RANK, scale=0.1).half()) for k, w in self.w.items()}

    def begin(self, lengths, of, window, sinks):
        L = self.L
        self.rows = L.leann_adapter_rows_create(self.ctx, lengths, of, [RANK, RANK], [1.0, 0.5], RANK)
        self.plan = L.leann_attention_create(self.ctx, lengths, heads=HEADS, head_dim=HIDDEN // HEADS, window=window, sinks=sinks,
                                             bucket_of=L.leann_position_buckets(BUCKETS, DISTANCE))

    def end(self):
        self.L.leann_adapter_rows_free(self.rows)
        self.L.leann_attention_free(self.plan)

    def project(self, name, x):
        return self.L.leann_adapter_project(self.ctx, self.proj[name], self.rows, x, *self.adapters[name], keep=True)

    def forward(self, x, drop):
        L, ctx, p = self.L, self.ctx, self.params
        qkv, low_qkv = self.project("qkv", x)
        q, k, v = qkv[:, :HIDDEN], qkv[:, HIDDEN:2 * HIDDEN], qkv[:, 2 * HIDDEN:]
        att, lse = L.leann_attention(ctx, self.plan, q, k, v, bias=p["bias"], keep=True)
        branch, low_o = self.project("o", att)
        mid, *stats1 = L.leann_layernorm(ctx, branch, p["g1"], p["b1"], EPS, residual=x, drop=drop, keep=True)
        hidden, low_up = self.project("up", mid)
        act, kept = L.leann_activation(ctx, hidden, keep=True)
        branch, low_down = self.project("down", act)
        out, *stats2 = L.leann_layernorm(ctx, branch, p["g2"], p["b2"], EPS, residual=mid, keep=True)
        self.kept = x, qkv, low_qkv, att, lse, low_o, stats1, mid, low_up, kept, low_down, stats2, drop
        return out

    def project_backward(self, name, dout, x, low):
        dx, down, up = self.L.leann_adapter_project_backward(self.ctx, self.proj[name], self.rows, dout, x, low, *self.adapters[name])
        return dx, {name + ".down": down, name + ".up": up}

    def backward(self, dout):
        import torch
        L, ctx, p = self.L, self.ctx, self.params
        x, qkv, low_qkv, att, lse, low_o, stats1, mid, low_up, kept, low_down, stats2, drop = self.kept
        grads = {}
        dmid, dbranch, grads["g2"], grads["b2"] = L.leann_layernorm_backward(ctx, dout, *stats2, p["g2"])
        act = L.leann_activation_backward(ctx, torch.empty_like(kept[0], dtype=x.dtype), kept, again=True)[1]  # the projection's input, not kept
        dact, more = self.project_backward("down", dbranch, act, low_down)
        grads.update(more)
        dhidden = L.leann_activation_backward(ctx, dact, kept)
        d, more = self.project_backward("up", dhidden, mid, low_up)
        grads.update(more)
        dres, dbranch, grads["g1"], grads["b1"] = L.leann_layernorm_backward(ctx, dmid + d, *stats1, p["g1"], drop=drop)
        datt, more = self.project_backward("o", dbranch, att, low_o)
        grads.update(more)
        dqkv = torch.empty_like(qkv)
        parts = [slice(i * HIDDEN, (i + 1) * HIDDEN) for i in range(3)]
        grads["bias"] = L.leann_attention_backward(ctx, self.plan, datt, *(qkv[:, s] for s in parts), att, lse, bias=p["bias"],
                                                   dq=dqkv[:, parts[0]], dk=dqkv[:, parts[1]], dv=dqkv[:, parts[2]])[3]
        d, more = self.project_backward("qkv", dqkv, x, low_qkv)
        grads.update(more)
        grads["x"] = dres + d
        return grads

    def close(self):
        for p in self.proj.values():
            self.L.leann_projection_free(p)


def wide(block, biases, x, lengths, of, window, sinks, drop_mask):
    """The same block in 64 bits with torch's differentiation: (out, leaves by name)."""
    import torch
    from attention64 import visible
    leaves = {k: v.double().requires_grad_() for k, v in block.params.items()}
    for k, (down, up) in block.adapters.items():
        leaves[k + ".down"], leaves[k + ".up"] = down.double().requires_grad_(), up.double().requires_grad_()
    leaves["x"] = x.double().requires_grad_()
    row_of = torch.from_numpy(np.repeat(of, lengths)).to(DEV)

    def project(name, t):
        y = t @ block.w[name].double().t() + biases[name].double()
        for a, scale in ((0, 1.0), (1, 0.5)):
            mine = (row_of == a).double()[:, None]
            y = y + mine * scale * ((t @ leaves[name + ".down"][a].t()) @ leaves[name + ".up"][a].t())
        return y

    def normal(t, g, b):
        c = t - t.mean(1, keepdim=True)
        return c / torch.sqrt((c * c).mean(1, keepdim=True) + EPS) * g + b

    qkv = project("qkv", leaves["x"])
    table = torch.as_tensor(block.L.leann_position_buckets(BUCKETS, DISTANCE).astype(np.int64), device=DEV)
    D, parts, at = HIDDEN // HEADS, [], 0
    for n in lengths:
        q, k, v = (qkv[at:at + n, i * HIDDEN:(i + 1) * HIDDEN].view(n, HEADS, D).transpose(0, 1) for i in range(3))
        p = torch.arange(n, device=DEV)
        s = q @ k.transpose(1, 2).contiguous() * D ** -0.5 + leaves["bias"][table[(p[None, :] - p[:, None]).clamp(-DISTANCE, DISTANCE) + DISTANCE]].permute(2, 0, 1)
        s = torch.where(visible(p, n, window, sinks), s, -math.inf)
        parts.append((torch.softmax(s, 2) @ v).transpose(0, 1).reshape(n, HIDDEN))
        at += n
    mid = normal(project("o", torch.cat(parts)) * drop_mask + leaves["x"], leaves["g1"], leaves["b1"])
    hidden = project("up", mid)
    return normal(project("down", 0.5 * hidden * torch.erfc(-hidden / math.sqrt(2))) + mid, leaves["g2"], leaves["b2"]), leaves


@pytest.mark.parametrize("window,sinks", [(None, 0), ((20, 20), 2)])
def test_a_training_step(window, sinks):
    import torch
    import paper_2506_08276_amd as L
    say("whole block", window)
    ctx = L.leann_create(CTX, torch.zeros(640, device=DEV))
    g = torch.Generator(DEV).manual_seed(3)
    state = g.get_state()
    block = Block(ctx, L, g)
    g.set_state(state)  # the projections' biases once more
    biases = {}
    for k, s in {"qkv": (3 * HIDDEN, HIDDEN), "o": (HIDDEN, HIDDEN), "up": (FFN, HIDDEN), "down": (HIDDEN, FFN)}.items():
        torch.randn(s, generator=g, device=DEV)
    for k, w in block.w.items():
        biases[k] = 0.1 * torch.randn(w.shape[0], generator=g, device=DEV)
    lengths, of = np.array([70, 1, 33, 128, 5]), np.array([0, 1, -1, 1, 0])
    x = torch.randn((int(lengths.sum()), HIDDEN), generator=g, device=DEV).half()
    drop = (0.1, 5, 7)
    mask = L.leann_dropout(ctx, torch.ones((len(x), HIDDEN), device=DEV), drop).double()
    block.begin(lengths, of, window, sinks)
    out = block.forward(x, drop)
    dout = (0.05 * torch.randn(out.shape, generator=g, device=DEV)).half()
    grads = block.backward(dout)
    want, leaves = wide(block, biases, x, lengths, of, window or (-1, -1), sinks, mask)
    (want * dout.double()).sum().backward()
    near = lambda a, b: float((a.double() - b.detach()).norm() / b.detach().norm())
    # Every tensor between is rounded to fp16 once, 2^-12 on average of its values at most, some ten in a row, and the block's layers pass errors on at about their size;
    # the 8 bits behind GELU's slope are off by 1 / 254 of their block's largest value, 1 / 80 of the typical one, in a sum of 384 terms of random sign.
    assert near(out, want) < 16 * 2.0 ** -12
    for name, leaf in leaves.items():
        assert grads[name].shape == leaf.shape, name
        assert near(grads[name], leaf.grad) < 16 * 2.0 ** -12 + 1 / 80, name
    block.end()
    block.close()
    L.leann_destroy(ctx)
