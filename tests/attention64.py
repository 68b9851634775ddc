"""Attention over ragged sequences and its gradient from the definition, in 64 bits, with the bounds that the kernels' roundings allow."""
import math

import torch


def visible(p, keys, window, sinks):
    """[queries][keys]: whether the query at position p[i] sees key j."""
    left, right = window
    p, j = p[:, None], torch.arange(keys, device=p.device)[None, :]
    see = torch.ones((len(p), keys), dtype=torch.bool, device=p.device)
    if right >= 0:
        see &= j <= p + right
    if left >= 0:
        see &= (j >= p - left) | (j < sinks)
    return see


class Sequences:
    """q [Tq][H D], k and v [Tk][G D] (any floating type), cut into sequences."""

    def __init__(self, q, k, v, q_rows, k_rows, first, heads, kv_heads, dim, window, sinks, bias, bucket_of, scale):
        self.q, self.k, self.v, self.q_rows, self.k_rows, self.first = q, k, v, q_rows, k_rows, first
        self.heads, self.kv_heads, self.dim, self.window, self.sinks = heads, kv_heads, dim, window, sinks
        self.bias, self.scale = bias, scale
        self.bucket_of = None if bucket_of is None else torch.as_tensor(bucket_of, dtype=torch.int64, device=q.device)

    def parts(self):
        """(rows of q, rows of k, visible, buckets) of the sequences that have queries."""
        a = b = 0
        for lq, lk, f in zip(self.q_rows, self.k_rows, self.first):
            if lq:
                p = f + torch.arange(lq, device=self.q.device)
                buckets = None
                if self.bias is not None:
                    d = len(self.bucket_of) // 2
                    buckets = self.bucket_of[(torch.arange(lk, device=p.device)[None, :] - p[:, None]).clamp(-d, d) + d]
                yield slice(a, a + lq), slice(b, b + lk), visible(p, lk, self.window, self.sinks), buckets
            a, b = a + lq, b + lk

    def columns(self, h):
        g = h // (self.heads // self.kv_heads)
        return slice(h * self.dim, (h + 1) * self.dim), slice(g * self.dim, (g + 1) * self.dim)

    def scores(self, rows, keys, see, buckets, h):
        cq, ck = self.columns(h)
        s = self.scale * self.q[rows, cq].double() @ self.k[keys, ck].double().t().contiguous()
        if buckets is not None:
            s = s + self.bias[:, h].double()[buckets]
        return torch.where(see, s, -math.inf)

    def forward(self, step):
        """(out, lse, bound of out's error, bound of lse's): `step` is half a step of the inputs' type."""
        out = torch.zeros(self.q.shape, dtype=torch.float64, device=self.q.device)
        lse = torch.full((self.heads, len(self.q)), -math.inf, dtype=torch.float64, device=self.q.device)
        far, far_lse = torch.zeros_like(out), torch.zeros_like(lse)
        for rows, keys, see, buckets in self.parts():
            for h in range(self.heads):
                cq, ck = self.columns(h)
                if keys.stop == keys.start:
                    continue
                s = self.scores(rows, keys, see, buckets, h)
                total = torch.logsumexp(s, 1)
                p = torch.exp(s - torch.where(total == -math.inf, math.inf, total)[:, None])
                v = torch.where(torch.isfinite(self.v[keys, ck]), self.v[keys, ck], 0).double()
                out[rows, cq] = p @ v
                lse[h, rows] = total
                # A score is a sum of dim products in fp32, scaled, with the bias added and multiplied by log2 e: dim + 6 roundings of 2^-24 of its terms' sum.
                # The exponential's argument is the difference to the maximum (2 more of the scores), the function good to 2^-22.
                terms = abs(self.scale) * self.q[rows, cq].double().abs().nan_to_num(0, 0, 0) @ self.k[keys, ck].double().abs().nan_to_num(0, 0, 0).t().contiguous()
                if buckets is not None:
                    terms = terms + self.bias[:, h].double().abs().nan_to_num(0, 0, 0)[buckets]
                ds = 2 * (self.dim + 8) * 2.0 ** -24 * (torch.where(see, terms, 0).amax(1, keepdim=True) + 1) + 2.0 ** -22
                far_lse[h, rows] = ds[:, 0] + (len(p[0]) + 4) * 2.0 ** -24 + 2.0 ** -22 * total.abs().nan_to_num(0, 0, 0)
                # Weights are rounded once (fp16's smallest ones to 2^-25 of the largest), added up in fp32, the result rounded once.
                weights = p @ v.abs()
                far[rows, cq] = (step * (1 + step) + 2 * ds + (len(p[0]) + 4) * 2.0 ** -24) * weights + step * out[rows, cq].abs()
                if step < 2.0 ** -9:
                    top = torch.exp(torch.where(see, s, -math.inf).amax(1) - total).nan_to_num(0)
                    far[rows, cq] += 2.0 ** -25 * top[:, None] * (see.double() @ v.abs()) + 2.0 ** -25
        return out, lse, far, far_lse

    def backward(self, dout, out, lse, step):
        """Gradients from dout and what the forward pass left, and bounds of their errors: [(dq, far), (dk, far), (dv, far), (dbias, far)]."""
        dev = self.q.device
        dq, dk, dv = (torch.zeros(t.shape, dtype=torch.float64, device=dev) for t in (self.q, self.k, self.v))
        fq, fk, fv = (torch.zeros_like(t) for t in (dq, dk, dv))
        db = torch.zeros((1 if self.bias is None else len(self.bias), self.heads), dtype=torch.float64, device=dev)
        fb = torch.zeros_like(db)
        for rows, keys, see, buckets in self.parts():
            for h in range(self.heads):
                cq, ck = self.columns(h)
                if keys.stop == keys.start:
                    continue
                q, k, v = self.q[rows, cq].double(), self.k[keys, ck].double(), self.v[keys, ck].double()
                g, o, ls = dout[rows, cq].double(), out[rows, cq].double(), lse[h, rows].double()
                s = self.scores(rows, keys, see, buckets, h)
                p = torch.exp(s - torch.where(ls == -math.inf, math.inf, ls)[:, None])
                dp, delta = g @ v.t().contiguous(), (g * o).sum(1, keepdim=True)
                ds = p * (dp - delta)
                dq[rows, cq] = self.scale * ds @ k
                dk[keys, ck] += self.scale * ds.t().contiguous() @ q
                dv[keys, ck] += p.t().contiguous() @ g
                # fp32: the score's error as in forward(), dp's and delta's sums of dim products; then one rounding of P and of dS where they enter products
                terms = abs(self.scale) * q.abs() @ k.abs().t().contiguous()
                if buckets is not None:
                    terms = terms + self.bias[:, h].double().abs().nan_to_num(0, 0, 0)[buckets]
                es = 2 * (self.dim + 8) * 2.0 ** -24 * (terms + 1) + 2.0 ** -22 * (1 + ls.abs().nan_to_num(0, 0, 0)[:, None])
                size = g.abs() @ v.abs().t().contiguous() + (g * o).abs().sum(1, keepdim=True)
                eds = es * ds.abs() + (self.dim + 4) * 2.0 ** -24 * p * size
                ep = (es + step) * p
                erow = eds + step * ds.abs()
                if step < 2.0 ** -9:  # fp16: 2^15 P, off by 2^-25 where that is no normal number; dS likewise, or scaled so that its largest is 2^14 at least
                    ep = ep + 2.0 ** -40 * see
                    erow = erow + see * (2.0 ** -40 + 2.0 ** -39 * ds.abs().amax())
                n = 2.0 ** -24 * (len(q) + len(k))
                fq[rows, cq] = abs(self.scale) * (erow + n * ds.abs()) @ k.abs()
                fk[keys, ck] += abs(self.scale) * (erow + n * ds.abs()).t().contiguous() @ q.abs()
                fv[keys, ck] += (ep + n * p).t().contiguous() @ g.abs()
                if buckets is not None:
                    db[:, h] += torch.zeros(len(db), dtype=torch.float64, device=dev).index_add_(0, buckets.reshape(-1), ds.reshape(-1))
                    fb[:, h] += torch.zeros(len(db), dtype=torch.float64, device=dev).index_add_(0, buckets.reshape(-1), (eds + 1e-6 * ds.abs()).reshape(-1))
        tiny = 2.0 ** -25 if step < 2.0 ** -9 else 0.0  # half of fp16's smallest number
        return [(dq, fq + step * dq.abs() + tiny), (dk, fk + step * dk.abs() + tiny), (dv, fv + step * dv.abs() + tiny), (db, fb)]


def assert_near(got, want, far, what):
    """|got - want| <= far wherever want is finite, and the same infinities and NaN elsewhere."""
    got = got.double()
    fine = torch.isfinite(want)
    assert torch.equal(fine, torch.isfinite(got)), f"{what}: {int((fine != torch.isfinite(got)).sum())} values differ in being finite"
    assert torch.equal(got[~fine].isnan(), want[~fine].isnan()) and torch.equal(got[~fine].nan_to_num(0), want[~fine].nan_to_num(0)), f"{what}: infinities differ"
    off = torch.where(fine, (got - want).abs() - far, -1.0).nan_to_num(-1)
    assert bool((off <= 0).all()), f"{what}: off by up to {float(off.max()):.3e} beyond the bound at {int(off.argmax())} of {tuple(want.shape)}"
