"""Dropout, LayerNorm and low-rank adapters in 64 bits on the host: what the kernels are compared with."""
import numpy as np

# unit roundoff of a rounding to nearest (24, 8 and 11 significant bits), and half the spacing of the smallest numbers
ROUND = {"float32": (2.0 ** -24, 2.0 ** -150), "bfloat16": (2.0 ** -8, 2.0 ** -134), "float16": (2.0 ** -11, 2.0 ** -25)}


def philox(counter, key):
    """Philox4x32-10 of uint32 arrays counter[4], key[2]: four uint32 arrays."""
    c, k = [np.asarray(v, np.uint64) for v in counter], [int(v) for v in key]
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return [v.astype(np.uint32) for v in c]


def dropout_bits(rows, cols, seed, offset):
    """uint16 [rows][cols]: the bits that each element is decided by."""
    group = (cols + 7) // 8
    row, chunk = np.meshgrid(np.arange(rows), np.arange(group), indexing="ij")
    full = lambda v: np.full(row.shape, v, np.uint64)
    w = philox([chunk, row, full(offset & 0xFFFFFFFF), full(offset >> 32)], [seed & 0xFFFFFFFF, seed >> 32])
    halves = [h for v in w for h in (v & np.uint32(0xFFFF), v >> np.uint32(16))]
    return np.stack(halves, -1).reshape(rows, group * 8)[:, :cols].astype(np.uint16)


def dropout(x, drop):
    """x in 64 bits; drop = (p, seed, offset) or None."""
    if drop is None:
        return x
    p, seed, offset = drop
    below = int(np.rint(np.float32(p) * np.float32(65536)))
    if below == 65536:
        return np.zeros_like(x)
    return np.where(dropout_bits(*x.shape, seed, offset) < below, 0.0, x * (65536 / (65536 - below)))


def layernorm(t, gamma, beta, eps):
    """(out, mean, rstd) over the rows of t."""
    mean = t.mean(1)
    rstd = 1 / np.sqrt(((t - mean[:, None]) ** 2).mean(1) + eps)
    return (t - mean[:, None]) * rstd[:, None] * gamma + beta, mean, rstd


def layernorm_backward(dout, t, mean, rstd, gamma):
    """(dt, dgamma, dbeta)."""
    xhat = (t - mean[:, None]) * rstd[:, None]
    gy = dout * gamma
    dt = rstd[:, None] * (gy - gy.mean(1, keepdims=True) - xhat * (gy * xhat).mean(1, keepdims=True))
    return dt, (dout * xhat).sum(0), dout.sum(0)


def request_rows(lengths, of):
    """[(adapter or -1, slice of its rows)] of the requests."""
    starts = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)
    return [(a, slice(int(starts[i]), int(starts[i + 1]))) for i, a in enumerate(of)]


def project(x, w, bias, down, up, lengths, of, ranks, scales):
    """(out, low)."""
    out, low = x @ w.T + bias, np.zeros((x.shape[0], down.shape[1]))
    for a, rows in request_rows(lengths, of):
        if a >= 0:
            r = ranks[a]
            low[rows, :r] = x[rows] @ down[a, :r].T
            out[rows] += scales[a] * (low[rows, :r] @ up[a, :, :r].T)
    return out, low


def project_backward(dout, x, low, w, down, up, lengths, of, ranks, scales):
    """(dx, ddown, dup)."""
    dx, ddown, dup = dout @ w, np.zeros(down.shape), np.zeros(up.shape)
    for a, rows in request_rows(lengths, of):
        if a >= 0:
            r = ranks[a]
            g = scales[a] * (dout[rows] @ up[a, :, :r])
            dx[rows] += g @ down[a, :r]
            ddown[a, :r] += g.T @ x[rows]
            dup[a, :, :r] += scales[a] * (dout[rows].T @ low[rows, :r])
    return dx, ddown, dup
