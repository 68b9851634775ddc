"""CPU checks of the 64-bit forms that the operators' GPU tests compare with."""
import numpy as np

import plain64


def test_philox_known_answers():
    """The generator's published test vectors."""
    for counter, key, want in [
            ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
            ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
            ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))]:
        assert tuple(int(v) for v in plain64.philox(counter, key)) == want


def test_unit_roundoffs():
    import torch
    for name, (u, tiny) in plain64.ROUND.items():
        info = torch.finfo(getattr(torch, name))
        assert u == info.eps / 2 and tiny == info.tiny * info.eps / 2


def test_dropout_rate_and_factor():
    x = np.ones((257, 1003))
    for p in (0.1, 0.5):
        y = plain64.dropout(x, (p, 3, 5))
        n = x.size
        assert abs((y == 0).mean() - p) < 5 * np.sqrt(p * (1 - p) / n)   # five standard deviations
        assert abs(y.mean() - 1) < 5 * np.sqrt(p / (1 - p) / n)
    assert (plain64.dropout(x, (0.0, 3, 5)) == x).all() and (plain64.dropout(x, (1.0, 3, 5)) == 0).all()
    assert (plain64.dropout(x, (0.5, 3, 5)) != plain64.dropout(x, (0.5, 3, 6))).mean() > 0.4


def test_layernorm_gradient_against_differences():
    rng = np.random.default_rng(1)
    for rows, cols in [(3, 1), (2, 5), (4, 17)]:
        t, dout, gamma, beta = rng.normal(size=(rows, cols)), rng.normal(size=(rows, cols)), rng.normal(size=cols), rng.normal(size=cols)
        loss = lambda t, gamma, beta: (plain64.layernorm(t, gamma, beta, 1e-3)[0] * dout).sum()
        _, mean, rstd = plain64.layernorm(t, gamma, beta, 1e-3)
        grads = plain64.layernorm_backward(dout, t, mean, rstd, gamma)
        for i, (g, v) in enumerate(zip(grads, (t, gamma, beta))):
            args = [t, gamma, beta]
            for j in np.ndindex(v.shape):
                d = np.zeros_like(v)
                d[j] = 1e-6
                up, down = list(args), list(args)
                up[i], down[i] = v + d, v - d
                assert abs((loss(*up) - loss(*down)) / 2e-6 - g[j]) < 1e-6 * (1 + abs(g[j])) * 100


def test_project_gradient_against_differences():
    rng = np.random.default_rng(2)
    lengths, of, ranks, scales = [2, 0, 3, 1], [1, 0, -1, 1], [2, 3], [0.5, 2.0]
    x, w, bias, down, up, dout = (rng.normal(size=s) for s in [(6, 4), (5, 4), (5,), (2, 3, 4), (2, 5, 3), (6, 5)])
    loss = lambda x, down, up: (plain64.project(x, w, bias, down, up, lengths, of, ranks, scales)[0] * dout).sum()
    low = plain64.project(x, w, bias, down, up, lengths, of, ranks, scales)[1]
    grads = plain64.project_backward(dout, x, low, w, down, up, lengths, of, ranks, scales)
    for i, (g, v) in enumerate(zip(grads, (x, down, up))):
        for j in np.ndindex(v.shape):
            a, b = [[x, down, up] for _ in range(2)]
            a[i], b[i] = v.copy(), v.copy()
            a[i][j] += 1e-6
            b[i][j] -= 1e-6
            assert abs((loss(*a) - loss(*b)) / 2e-6 - g[j]) < 1e-7 * (1 + abs(g[j]))
