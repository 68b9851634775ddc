"""The operators that a training step of an encoder's block needs between its projections, as cases that can be timed and compared.

- `attention`           leann_attention: attention over ragged sequences, with a learned bias by buckets of relative position, a sliding
                        window, first tokens that stay visible, shared key heads; few queries over long keys as well;
- `attention_backward`  leann_attention_backward: gradients of queries, keys, values and of the bias;
- `checkpoint`          leann_checkpoint and leann_checkpoint_restore: an activation kept in 8 bits with scales, and back;
- `activation`          leann_activation: GELU, for serving; in training (`train`) it keeps its input in 8 bits, and
                        leann_activation_backward takes the gradient from those and gives the output again.

With `own` false, `run` computes the same in elementary torch operations in 32 bits, rounded once at the end.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BLOCK = 128  # columns that share a scale
_ctx = None


def listed():
    """The cases."""
    return [
        # the tokens of one query: nothing but latency
        dict(name="attention one query", op="attention", requests=1, q_low=12, q_high=12, k_low=0, k_high=0, at_end=False, heads=12,
             kv_heads=12, dim=64, left=-1, right=-1, sinks=0, buckets=32, distance=128, keep=False, packed=True, dtype="bf16"),
        # serving: the last layer's first token alone over every token of long documents
        dict(name="attention single tokens", op="attention", requests=8, q_low=1, q_high=1, k_low=500, k_high=16384, at_end=False,
             heads=12, kv_heads=12, dim=64, left=-1, right=-1, sinks=0, buckets=32, distance=128, keep=False, packed=False, dtype="bf16"),
        # bulk indexing: chunks of up to the encoder's 512 positions, relative positions learned
        dict(name="attention ragged chunks", op="attention", requests=256, q_low=3, q_high=512, k_low=0, k_high=0, at_end=False, heads=12,
             kv_heads=12, dim=64, left=-1, right=-1, sinks=0, buckets=32, distance=128, keep=True, packed=True, dtype="bf16"),
        # indexing whole documents: a window of 256 tokens to either side, four first tokens visible to all, three heads per key head
        dict(name="attention long documents", op="attention", requests=3, q_low=3001, q_high=4096, k_low=0, k_high=0, at_end=False,
             heads=12, kv_heads=4, dim=64, left=256, right=256, sinks=4, buckets=0, distance=0, keep=False, packed=True, dtype="f16"),
        # a small training step of the lighter encoder: 16 chunks
        dict(name="attention backward small", op="attention_backward", requests=16, q_low=20, q_high=128, k_low=0, k_high=0, at_end=False,
             heads=12, kv_heads=12, dim=32, left=-1, right=-1, sinks=0, buckets=32, distance=128, packed=True, dtype="f16"),
        # training: 512 chunks of the base encoder, the bias learned too
        dict(name="attention backward training batch", op="attention_backward", requests=512, q_low=64, q_high=256, k_low=0, k_high=0,
             at_end=False, heads=12, kv_heads=12, dim=64, left=-1, right=-1, sinks=0, buckets=32, distance=128, packed=True, dtype="bf16"),
        # training on whole documents: window, first tokens and shared key heads
        dict(name="attention backward long documents", op="attention_backward", requests=2, q_low=3001, q_high=4096, k_low=0, k_high=0,
             at_end=False, heads=12, kv_heads=4, dim=64, left=256, right=256, sinks=4, buckets=32, distance=128, packed=False,
             dtype="bf16"),
        # the residual stream of one query's tokens
        dict(name="checkpoint one query", op="checkpoint", rows=12, cols=768, pad=0, dtype="bf16"),
        # training: a residual stream of 1024 chunks of 128 tokens, kept between forward and backward pass
        dict(name="checkpoint training batch", op="checkpoint", rows=131072, cols=768, pad=0, dtype="bf16"),
        # serving: the hidden layer of one query's tokens
        dict(name="activation one query", op="activation", rows=12, cols=1536, pad=0, dtype="bf16", kind="gelu", train=False),
        # a small training step at an odd width
        dict(name="activation odd rows", op="activation", rows=1777, cols=1021, pad=3, dtype="f16", kind="gelu_tanh", train=True),
        # training: the hidden layer of the lighter encoder, forward and backward, 1024 chunks of 128 tokens
        dict(name="activation training batch", op="activation", rows=131072, cols=1536, pad=0, dtype="bf16", kind="gelu", train=True),
    ]


def _log(rng, lo, hi):
    """A whole number in [lo, hi], spread over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    op = rng.choice(["attention", "attention", "attention", "attention_backward", "attention_backward", "checkpoint", "activation"])
    if op in ("checkpoint", "activation"):
        cols = rng.choice([_log(rng, 16, 4096), rng.choice([128, 384, 768, 1536])])
        rows = _log(rng, 1, 131072 * 768 // max(cols, 768))
        case = dict(op=op, rows=rows, cols=cols, pad=rng.choice([0, 0, 3, 64]), dtype=rng.choice(["f32", "bf16", "bf16", "f16"]))
        if op == "activation":
            case.update(kind=rng.choice(["gelu", "gelu_tanh"]), train=rng.random() < 0.7)
        return case
    heads, kv_heads, dim = rng.choice([(12, 12, 64), (12, 12, 32), (12, 4, 64), (8, 2, 128), (16, 16, 64), (6, 6, 40), (4, 1, 96)])
    backward = op == "attention_backward"
    scores = (1.5e8 if backward else 4e8) / heads
    few = not backward and rng.random() < 0.35
    if few:  # few queries over the keys of a document, at its start or at its end
        q_high, k_high = _log(rng, 1, 16), _log(rng, 1, 16384)
        q_low, k_low = rng.randint(1, q_high), rng.randint(0, k_high)
        requests = _log(rng, 1, max(1, min(64, 131072 // k_high)))
    else:
        q_high, k_low, k_high = _log(rng, 1, 4096 if not backward else 3500), 0, 0
        q_low = rng.randint(0, q_high)
        requests = _log(rng, 1, max(1, min(512, int(scores / q_high ** 2))))
    window = rng.choice([(-1, -1), (-1, -1), (_log(rng, 1, 1024),) * 2, (rng.choice([-1, _log(rng, 1, 1024)]), 0)])
    case = dict(op=op, requests=requests, q_low=q_low, q_high=q_high, k_low=k_low, k_high=k_high, at_end=few and rng.random() < 0.5,
                heads=heads, kv_heads=kv_heads, dim=dim, left=window[0], right=window[1], sinks=rng.choice([0, 1, 4, 70]) if window[0] >= 0 else 0,
                buckets=0, distance=0, packed=rng.random() < 0.6 and not few, dtype=rng.choice(["bf16", "bf16", "f16"]))
    if rng.random() < 0.6:
        case.update(buckets=rng.choice([16, 32, 64]), distance=rng.choice([64, 128, 256, 1000]))
    if sum(_lengths(case)[0]) == 0:  # sequences may be empty, not all of them
        case["q_low"] = case["q_high"]
    if not backward:
        case["keep"] = rng.random() < 0.5
    return case


# ------------------------------------------------------------------ what follows from a case alone
def _lengths(case):
    """Query rows and key rows of each sequence (the same rows where k_high is 0)."""
    rng = random.Random(" ".join(str(case[k]) for k in ("requests", "q_low", "q_high", "k_low", "k_high")))
    q = [rng.randint(case["q_low"], case["q_high"]) for _ in range(case["requests"])]
    if not case["k_high"]:
        return q, list(q)
    return q, [rng.randint(case["k_low"], case["k_high"]) for _ in range(case["requests"])]


def _first(case):
    """The position of each sequence's first query."""
    return [max(0, k - q) if case["at_end"] else 0 for q, k in zip(*_lengths(case))]


def _pairs(case):
    """Pairs of a query and a key that it sees, over all sequences."""
    total = 0
    for q, k, first in zip(*_lengths(case), _first(case)):
        p = first + np.arange(q, dtype=np.int64)
        end = np.minimum(k, p + case["right"] + 1) if case["right"] >= 0 else np.full_like(p, k)
        begin = np.maximum(0, p - case["left"]) if case["left"] >= 0 else np.zeros_like(p)
        total += int((np.maximum(0, end - begin) + np.minimum(np.minimum(case["sinks"], begin), end)).sum())
    return total


def work(case):
    """Bytes and operations that one pass cannot do without."""
    size = TYPES[case["dtype"]].itemsize
    if case["op"] in ("checkpoint", "activation"):
        n = case["rows"] * case["cols"]
        kept = n + 4 * case["rows"] * ((case["cols"] + BLOCK - 1) // BLOCK)
        if case["op"] == "checkpoint":
            return {"bytes": 2 * n * size + 2 * kept, "flops": 4 * n}
        if not case["train"]:
            return {"bytes": 2 * n * size, "flops": 10 * n}
        return {"bytes": 5 * n * size + 2 * kept, "flops": 30 * n}  # x to y, kept; kept and the gradient of y to that of x and y again
    q, k = _lengths(case)
    rows_q, rows_k = sum(q) * case["heads"] * case["dim"], sum(k) * case["kv_heads"] * case["dim"]
    table = 4 * case["buckets"] * case["heads"]
    lse = 4 * sum(q) * case["heads"]
    pairs = _pairs(case) * case["heads"] * case["dim"]
    if case["op"] == "attention":
        return {"bytes": size * 2 * (rows_q + rows_k) + table + (lse if case["keep"] else 0), "flops": 4 * pairs}
    return {"bytes": size * (4 * rows_q + 4 * rows_k) + 2 * table + lse, "flops": 10 * pairs}


# ------------------------------------------------------------------ what a program has in hand
class _Handle:
    """A handle of the library that is freed with the state that holds it."""

    def __init__(self, handle, free):
        self.handle, self._free = handle, free

    def __del__(self):
        self._free(self.handle)


def _context():
    """A context, made once per process: an encoder of no layers, as these operators need its stream and workspaces only."""
    global _ctx
    import paper_2506_08276_amd as L
    if _ctx is None:
        desc = dict(layers=0, hidden=128, heads=2, ffn=128, vocab=1, max_pos=1)
        _ctx = L.leann_create(desc, torch.zeros(5 * 128, device=DEV))  # tok_emb, pos_emb, seg_emb, scale, shift
    return _ctx


def _position_buckets(buckets, distance):
    """The bucket of each relative position from -distance to distance, as int32: half of the buckets for keys ahead; of a direction's, the first
    half hold one distance each, the others ranges that grow by equal factors up to `distance`, which belongs to the last one with all beyond."""
    half = buckets // 2
    single = half // 2
    found = np.empty(2 * distance + 1, np.int32)
    for d in range(-distance, distance + 1):
        n = abs(d)
        b = n
        if n >= single:
            b = single
            # the largest b with (n / single)^(half - single) >= (distance / single)^(b - single), in whole numbers
            while b + 1 < half and n ** (half - single) * single ** (b + 1 - single) >= distance ** (b + 1 - single) * single ** (half - single):
                b += 1
        found[d + distance] = b + (half if d > 0 else 0)
    return found


def prepare(case, seed):
    """Inputs of a case, from the seed alone, and the handles that a program keeps."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    dtype = TYPES[case["dtype"]]
    s = dict(case)
    if own:
        import paper_2506_08276_amd as L
        s.update(L=L, ctx=_context())

    def normal(rows, cols, scale=1.0):
        return torch.randn((rows, cols), generator=g, device=DEV) * scale

    if case["op"] in ("checkpoint", "activation"):
        r, c, pad = case["rows"], case["cols"], case["pad"]
        x = normal(r, c + pad)
        x[:, ::97] *= 8  # a few columns are eight times as large, as residual streams and hidden layers have them
        s["x"] = x.to(dtype)[:, :c]
        if case["op"] == "activation" and case["train"]:
            s["dout"] = normal(r, c, 0.01).to(dtype)
        return s
    (q, k), H, G, D = _lengths(case), case["heads"], case["kv_heads"], case["dim"]
    if case["packed"]:  # queries, keys and values side by side, as one projection leaves them
        qkv = normal(sum(q), (H + 2 * G) * D, 1.3).to(dtype)
        s["q"], s["k"], s["v"] = qkv[:, :H * D], qkv[:, H * D:(H + G) * D], qkv[:, (H + G) * D:]
    else:
        s["q"], s["k"], s["v"] = (normal(n, h * D, 1.3).to(dtype) for n, h in ((sum(q), H), (sum(k), G), (sum(k), G)))
    s["scale"] = D ** -0.5
    s["bias"] = normal(case["buckets"], H) if case["buckets"] else None
    s["bucket_of"] = _position_buckets(case["buckets"], case["distance"]) if case["buckets"] else None
    first = _first(case)
    s.update(q_rows=np.array(q, np.int32), k_rows=np.array(k, np.int32), first=np.array(first, np.int32))
    s["q_most"], s["k_most"] = max(q), max(1, max(k))
    for name, rows in (("q", q), ("k", k)):  # where each sequence's rows are, and each row's sequence and place in it
        starts = np.concatenate([[0], np.cumsum(rows)])
        of = np.repeat(np.arange(len(rows)), rows)
        s[name + "_start"], s[name + "_len"], s[name + "_of"], s[name + "_at"] = (
            torch.from_numpy(np.asarray(a, np.int64)).to(DEV) for a in (starts[:-1], rows, of, np.arange(len(of)) - starts[of]))
    s["first_at"] = torch.from_numpy(np.array(first, np.int64)).to(DEV)
    s["bucket_at"] = torch.from_numpy(s["bucket_of"].astype(np.int64)).to(DEV) if case["buckets"] else None
    if case["op"] == "attention_backward":
        s["dout"] = normal(sum(q), H * D, 0.01).to(dtype)
        s["out"], s["lse"] = _plain_attention(s)
    if own:
        s["plan"] = _Handle(L.leann_attention_create(
            s["ctx"], s["q_rows"], s["k_rows"] if case["k_high"] else None, heads=H, head_dim=D, kv_heads=G, first=s["first"],
            window=(case["left"], case["right"]), sinks=case["sinks"], bucket_of=s["bucket_of"]), L.leann_attention_free)
    return s


# ------------------------------------------------------------------ plain forms
def _padded(s, t, side, repeat=1):
    """[sequence][head][row][dim] in 32 bits of the rows of `side`, zeros behind a sequence's end; each head `repeat` times."""
    most = s[side + "_most"]
    at = torch.arange(most, device=DEV)
    index = (s[side + "_start"][:, None] + at).clamp(max=max(0, t.shape[0] - 1))
    if t.shape[0] == 0:
        x = torch.zeros((len(index), most, t.shape[1]), device=DEV)
    else:
        x = torch.where((at < s[side + "_len"][:, None])[:, :, None], t[index].float(), 0.0)
    x = x.view(x.shape[0], most, -1, s["dim"]).permute(0, 2, 1, 3)
    return (x.repeat_interleave(repeat, 1) if repeat > 1 else x).contiguous()


def _rows_of(s, t, side):
    """The rows of `side` from [sequence][head][row][dim], side by side as the inputs have them."""
    return t.permute(0, 2, 1, 3)[s[side + "_of"], s[side + "_at"]].reshape(len(s[side + "_of"]), -1)


def _scores(s, q, k):
    """Scores [sequence][head][query][key], and where a query sees a key."""
    i, j = torch.arange(s["q_most"], device=DEV)[None, :, None], torch.arange(s["k_most"], device=DEV)[None, None, :]
    p = s["first_at"][:, None, None] + i
    seen = (i < s["q_len"][:, None, None]) & (j < s["k_len"][:, None, None])
    if s["right"] >= 0:
        seen = seen & (j <= p + s["right"])
    if s["left"] >= 0:
        seen = seen & ((j >= p - s["left"]) | (j < s["sinks"]))
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(s["scale"])
    if s["bias"] is not None:
        M = s["distance"]
        if s["at_end"]:
            scores += s["bias"][s["bucket_at"][(j - p).clamp(-M, M) + M]].permute(0, 3, 1, 2)
        else:  # the same positions in every sequence
            scores += s["bias"][s["bucket_at"][(j - i)[0].clamp(-M, M) + M]].permute(2, 0, 1)
    return scores, seen[:, None]


def _plain_attention(s):
    share = s["heads"] // s["kv_heads"]
    q, k, v = _padded(s, s["q"], "q"), _padded(s, s["k"], "k", share), _padded(s, s["v"], "k", share)
    scores, seen = _scores(s, q, k)
    scores.masked_fill_(~seen, -math.inf)
    top = scores.amax(3, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)  # a query that sees nothing
    e = scores.sub_(top).exp_()
    total = e.sum(3, keepdim=True)
    out = torch.matmul(e, v) / torch.where(total == 0, 1.0, total)
    lse = (top + total.log())[..., 0]
    return _rows_of(s, out, "q").to(s["q"].dtype), lse.transpose(1, 2)[s["q_of"], s["q_at"]].t().contiguous()


def _bucket_sums(s, ds):
    """Sums [bucket][head] of a gradient [sequence][head][query][key] whose queries begin at position 0: sums over the sequences, then along the
    diagonals, in 64 bits, as the terms of a row cancel."""
    rows, keys = ds.shape[2:]
    ds = ds.sum(0, dtype=torch.float64).flip(1)  # row r is query rows - 1 - r: relative position key + r - (rows - 1)
    wide = torch.zeros((s["heads"], rows, keys + rows), dtype=torch.float64, device=DEV)
    wide[:, :, rows:] = ds.flip(2)  # rows one element shorter shift by one to the left each
    wide = wide.flip(2).reshape(s["heads"], -1)[:, :rows * (keys + rows - 1)].view(s["heads"], rows, keys + rows - 1).sum(1)
    delta = torch.arange(keys + rows - 1, device=DEV) - (rows - 1)
    M = s["distance"]
    sums = torch.zeros((s["buckets"], s["heads"]), dtype=torch.float64, device=DEV)
    return sums.index_add_(0, s["bucket_at"][delta.clamp(-M, M) + M], wide.t()).float()


def _plain_attention_backward(s):
    share = s["heads"] // s["kv_heads"]
    q, k, v = _padded(s, s["q"], "q"), _padded(s, s["k"], "k", share), _padded(s, s["v"], "k", share)
    dout, out = _padded(s, s["dout"], "q"), _padded(s, s["out"], "q")
    lse = torch.full((len(s["q_len"]), s["q_most"], s["heads"]), math.inf, device=DEV)
    lse[s["q_of"], s["q_at"]] = s["lse"].t()
    lse = torch.where(lse == -math.inf, math.inf, lse).transpose(1, 2)[..., None]
    scores, seen = _scores(s, q, k)
    p = torch.where(seen, scores.sub_(lse).exp_(), 0.0)
    del scores
    dv = torch.matmul(p.transpose(2, 3).contiguous(), dout)
    ds = torch.matmul(dout, v.transpose(2, 3).contiguous()).sub_((dout * out).sum(3, keepdim=True)).mul_(p)
    del p
    dq = torch.matmul(ds, k).mul_(s["scale"])
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q).mul_(s["scale"])
    dk, dv = (t.view(t.shape[0], s["kv_heads"], share, *t.shape[2:]).sum(2) for t in (dk, dv))
    dtype = s["q"].dtype
    return (_rows_of(s, dq, "q").to(dtype), _rows_of(s, dk, "k").to(dtype), _rows_of(s, dv, "k").to(dtype),
            _bucket_sums(s, ds) if s["bias"] is not None else None)


def _kept_in_8_bits(x):
    """What x is after it was kept in 8 bits: of each row's BLOCK columns the largest magnitude is 127 steps."""
    rows, cols = x.shape
    blocks = (cols + BLOCK - 1) // BLOCK
    w = torch.zeros((rows, blocks * BLOCK), device=DEV)
    w[:, :cols] = x
    w = w.view(rows, blocks, BLOCK)
    top = w.abs().amax(2, keepdim=True)
    codes = torch.where(top > 0, w * 127 / top, 0.0).round()
    return (codes * (top / 127)).view(rows, -1)[:, :cols]


def _activated(x, kind):
    """(y, dy / dx)"""
    if kind == "gelu":
        phi = 0.5 * torch.erfc(x * -math.sqrt(0.5))
        return x * phi, phi + x * torch.exp(-0.5 * x * x) * (1 / math.sqrt(2 * math.pi))
    a, b = math.sqrt(2 / math.pi), 0.044715
    t = torch.tanh(a * (x + b * x * x * x))
    return 0.5 * x * (1 + t), 0.5 * (1 + t) + 0.5 * x * (1 - t * t) * a * (1 + 3 * b * x * x)


def run(s):
    """One pass through an operator."""
    op = s["op"]
    if own:
        L, ctx = s["L"], s["ctx"]
        if op == "attention":
            return L.leann_attention(ctx, s["plan"].handle, s["q"], s["k"], s["v"], s["scale"], bias=s["bias"], keep=s["keep"])
        if op == "attention_backward":
            return L.leann_attention_backward(ctx, s["plan"].handle, s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["scale"],
                                              bias=s["bias"])
        if op == "checkpoint":
            return L.leann_checkpoint_restore(ctx, L.leann_checkpoint(ctx, s["x"]), s["x"].dtype)
        if not s["train"]:
            return L.leann_activation(ctx, s["x"], s["kind"])
        y, kept = L.leann_activation(ctx, s["x"], s["kind"], keep=True)
        dx, again = L.leann_activation_backward(ctx, s["dout"], kept, s["kind"], again=True)
        return y, dx, again
    if op == "attention":
        out, lse = _plain_attention(s)
        return (out, lse) if s["keep"] else out
    if op == "attention_backward":
        return _plain_attention_backward(s)
    x = s["x"].float()
    if op == "checkpoint":
        return _kept_in_8_bits(x).to(s["x"].dtype)
    y = _activated(x, s["kind"])[0].to(s["x"].dtype)
    if not s["train"]:
        return y
    again, slope = _activated(_kept_in_8_bits(x), s["kind"])
    return y, (s["dout"].float() * slope).to(y.dtype), again.to(y.dtype)


# ------------------------------------------------------------------ the definitions in 64 bits
def _exact_sequence(s, n):
    """Queries, keys, values [head][row][dim] of sequence n, its scores with -inf where a query does not see a key, and buckets."""
    H, G, D = s["heads"], s["kv_heads"], s["dim"]
    q0, k0 = int(s["q_rows"][:n].sum()), int(s["k_rows"][:n].sum())
    lq, lk, first = int(s["q_rows"][n]), int(s["k_rows"][n]), int(s["first"][n])

    def heads(t, row, count, h):
        t = t[row:row + count].double().reshape(count, h, D).transpose(0, 1)
        return t[torch.arange(H, device=DEV) // (H // h)]

    q, k, v = heads(s["q"], q0, lq, H), heads(s["k"], k0, lk, G), heads(s["v"], k0, lk, G)
    away = torch.arange(lk, device=DEV)[None, :] - (first + torch.arange(lq, device=DEV))[:, None]
    hidden = torch.zeros((lq, lk), dtype=torch.bool, device=DEV)
    if s["right"] >= 0:
        hidden |= away > s["right"]
    if s["left"] >= 0:
        hidden |= (away < -s["left"]) & (torch.arange(lk, device=DEV) >= s["sinks"])[None, :]
    scores = torch.stack([torch.mm(a, b.t().contiguous()) for a, b in zip(q, k)]) * s["scale"]
    bucket = None
    if s["bias"] is not None:
        bucket = s["bucket_at"][away.clamp(-s["distance"], s["distance"]) + s["distance"]]
        scores += s["bias"].double().t()[:, bucket]
    scores[:, hidden] = -math.inf
    return slice(q0, q0 + lq), slice(k0, k0 + lk), heads, q, k, v, scores, bucket


def _exact_attention(s):
    H, D = s["heads"], s["dim"]
    out = torch.zeros((len(s["q"]), H * D), dtype=torch.float64, device=DEV)
    lse = torch.full((H, len(s["q"])), -math.inf, dtype=torch.float64, device=DEV)
    for n in range(s["requests"]):
        if s["q_rows"][n] == 0 or s["k_rows"][n] == 0:
            continue
        rows, _, _, _, _, v, scores, _ = _exact_sequence(s, n)
        total = torch.logsumexp(scores, 2)
        p = torch.exp(scores - torch.where(total == -math.inf, math.inf, total)[:, :, None])
        out[rows] = torch.stack([torch.mm(a, b) for a, b in zip(p, v)]).transpose(0, 1).reshape(-1, H * D)
        lse[:, rows] = total
    return (out, lse) if s["keep"] else out


def _exact_attention_backward(s):
    H, G, D = s["heads"], s["kv_heads"], s["dim"]
    dq = torch.zeros((len(s["q"]), H * D), dtype=torch.float64, device=DEV)
    dk, dv = (torch.zeros((len(s["k"]), G * D), dtype=torch.float64, device=DEV) for _ in range(2))
    dbias = torch.zeros((max(1, s["buckets"]), H), dtype=torch.float64, device=DEV)
    for n in range(s["requests"]):
        if s["q_rows"][n] == 0 or s["k_rows"][n] == 0:
            continue
        rows, keys, heads, q, k, v, scores, bucket = _exact_sequence(s, n)
        dout, out = heads(s["dout"], rows.start, len(q[0]), H), heads(s["out"], rows.start, len(q[0]), H)
        lse = s["lse"][:, rows].double()
        for h in range(H):
            g = h // (H // G)
            p = torch.exp(scores[h] - torch.where(lse[h] == -math.inf, math.inf, lse[h])[:, None])
            ds = p * (torch.mm(dout[h], v[h].t().contiguous()) - (dout[h] * out[h]).sum(1)[:, None])
            dq[rows, h * D:(h + 1) * D] = s["scale"] * torch.mm(ds, k[h])
            dk[keys, g * D:(g + 1) * D] += s["scale"] * torch.mm(ds.t().contiguous(), q[h])
            dv[keys, g * D:(g + 1) * D] += torch.mm(p.t().contiguous(), dout[h])
            if bucket is not None:
                dbias[:, h] += torch.bincount(bucket.reshape(-1), weights=ds.reshape(-1), minlength=s["buckets"])
    return dq, dk, dv, dbias if s["bias"] is not None else None


def _exact_kept(x):
    """x after 8 bits, block by block of columns."""
    parts = []
    for c in range(0, x.shape[1], BLOCK):
        part = x[:, c:c + BLOCK].double()
        step = part.abs().max(1, keepdim=True).values / 127
        parts.append(torch.where(step > 0, torch.round(part * 127 / (step * 127)) * step, 0.0))
    return torch.cat(parts, 1)


def _exact_activation(x, kind):
    if kind == "gelu":
        y = 0.5 * x * (1 + torch.erf(x / 2 ** 0.5))
        return y, torch.where(x == 0, 0.5, y / x) + x * torch.exp(-x ** 2 / 2) / (2 * math.pi) ** 0.5
    # (1 + tanh u) / 2 = 1 / (1 + e^(-2u))
    u = (2 / math.pi) ** 0.5 * (x + 0.044715 * x ** 3)
    g = torch.sigmoid(2 * u)
    return x * g, g + x * g * (1 - g) * 2 * (2 / math.pi) ** 0.5 * (1 + 3 * 0.044715 * x ** 2)


def exact(case, seed):
    """What `run` returns, from the definitions in 64 bits."""
    s = prepare(case, seed)
    if case["op"] == "attention":
        return _exact_attention(s)
    if case["op"] == "attention_backward":
        return _exact_attention_backward(s)
    if case["op"] == "checkpoint":
        return _exact_kept(s["x"])
    y = _exact_activation(s["x"].double(), case["kind"])[0]
    if not case["train"]:
        return y
    again, slope = _exact_activation(_exact_kept(s["x"]), case["kind"])
    return y, s["dout"].double() * slope, again
