"""The gradient of attention over ragged sequences on the GPU against its definition in 64 bits."""
import pytest

from attention64 import assert_near
from gpu_util import say
from test_gpu_attention import CASES, CTX, Case, ctx  # noqa: F401

pytestmark = pytest.mark.gpu
NAMES = ("dq", "dk", "dv", "dbias")


def backward(c, out, lse, **more):
    return c.L.leann_attention_backward(c.ctx, c.plan, c.dout, c.q, c.k, c.v, out, lse, bias=c.bias, **more)


def check(c):
    out, lse = c.run()
    got = backward(c, out, lse)
    want = c.sequences().backward(c.dout, out, lse, c.step)
    for name, g, (w, far) in zip(NAMES, got, want):
        if g is None:
            assert name == "dbias" and c.bias is None
        else:
            assert_near(g, w, far, name)
    return got


@pytest.mark.parametrize("name", CASES)
def test_against_the_definition(ctx, name):  # noqa: F811
    say("attention backward", name)
    with Case(ctx, **CASES[name]) as c:
        check(c)


@pytest.mark.parametrize("distance", [1024, 603, 604])
@pytest.mark.parametrize("dim", [32, 64, 128])
def test_long_tables_of_biases_beside_short_sequences(ctx, dim, distance):  # noqa: F811
    """Tables go by the longest sequence, or the last position; a block that takes a whole short one has less room the more wavefronts it has."""
    say("attention backward, tables", dim, distance)
    with Case(ctx, [1100, 200, 100, 1], heads=2, dim=dim, buckets=64, distance=distance) as c:
        check(c)
    with Case(ctx, [200, 100], heads=2, dim=dim, buckets=64, distance=distance, first=[3000, 0]) as c:
        check(c)


@pytest.mark.parametrize("size", [1e-4, 300.0])
@pytest.mark.parametrize("dim", [32, 128])
def test_fp16_of_any_size(ctx, size, dim):  # noqa: F811
    """Gradients near the ends of fp16's range: weights of 1 / 2000 times 1e-4 below its normal numbers, dO V^T above its largest."""
    say("attention backward, fp16", size, dim)
    with Case(ctx, [2000, 5], heads=2, dim=dim, dtype="float16", buckets=32, distance=128, spread=1.0 if size < 1 else 2.5) as c:
        c.dout = c.dout.float().mul(size * 10).half()
        c.dout[1000:1010] *= 0.01
        check(c)


def test_slices_of_one_projection(ctx):  # noqa: F811
    import torch
    say("attention backward into slices")
    with Case(ctx, [70, 3, 150], heads=4, kv_heads=2, packed=True, pad=8) as c:
        out, lse = c.run()
        want = backward(c, out, lse)
        whole = torch.full((223, 4 * 128 + 8), 7.0, dtype=c.q.dtype, device="cuda:0")
        got = backward(c, out, lse, dq=whole[:, :256], dk=whole[:, 256:384], dv=whole[:, 384:512])
        for a, b in zip(got[:3], want[:3]):
            assert torch.equal(a, b)
        assert bool((whole[:, 512:] == 7).all())


def test_bits_repeat_and_sequences_are_apart(ctx):  # noqa: F811
    import torch
    say("attention backward, twice")
    with Case(ctx, [150, 40, 300], packed=True, buckets=32, distance=128) as c:
        out, lse = c.run()
        a, b = backward(c, out, lse), backward(c, out, lse)
        assert all(torch.equal(x, y) for x, y in zip(a, b))
        b = backward(c, out, lse, need_bias=False)
        assert b[3] is None and all(torch.equal(x, y) for x, y in zip(a[:3], b))
        c.dout[150:190] = float("nan")
        d = backward(c, out, lse)
        for x, y in zip(a[:3], d[:3]):
            assert torch.equal(x[:150], y[:150]) and torch.equal(x[190:], y[190:])


@pytest.mark.parametrize("window,sinks", [((30, 30), 0), ((64, 0), 3), ((-1, 0), 0), (None, 0)])
@pytest.mark.parametrize("what", ["q", "k", "v", "dout"])
def test_what_is_hidden_does_not_reach_a_row(ctx, window, sinks, what):  # noqa: F811
    import torch
    say("attention backward, infinities", window, what)
    with Case(ctx, [90, 150, 40], window=window, sinks=sinks, heads=2) as c:
        out, lse = c.run()
        clean = backward(c, out, lse)
        t = getattr(c, what)
        t[100, 5:70], t[239, 3] = float("nan"), float("inf")
        out, lse = c.run()
        dq, dk, dv, _ = backward(c, out, lse)
        meets_q, meets_k, nan_q, nan_k = (torch.zeros(280, dtype=torch.bool, device="cuda:0") for _ in range(4))
        for rows, keys, see, _ in c.sequences().parts():
            for i in (100, 239):
                if rows.start <= i < rows.stop:
                    if what in ("k", "v"):  # queries that see the key, and whatever those see
                        sees = see[:, i - keys.start]
                        meets_q[rows] |= sees
                        meets_k[rows] |= (see & sees[:, None]).any(0)
                    else:  # the query, and what it sees
                        meets_q[i] = True
                        meets_k[rows] |= see[i - rows.start]
                    if i == 100:
                        nan_q, nan_k = meets_q.clone(), meets_k.clone()
        assert torch.equal(dq[~meets_q], clean[0][~meets_q])
        assert torch.equal(dk[~meets_k], clean[1][~meets_k])
        assert torch.equal(dv[~meets_k], clean[2][~meets_k])
        # NaN reaches all that meets it; of the infinity a score may be -inf, which is a weight of 0
        assert bool((~torch.isfinite(dq[nan_q])).any(1).all())
        assert bool((~torch.isfinite(dk[nan_k])).any(1).all())


def test_biases_that_hide(ctx):  # noqa: F811
    import torch
    say("attention backward, hiding biases")
    with Case(ctx, [5, 200], buckets=32, distance=128, window=(20, 20)) as c:
        c.bias[3:9] = -float("inf")
        check(c)
        c.bias[:] = -float("inf")
        got = check(c)
        assert not any(g.any() for g in got)


def test_against_differences(ctx):  # noqa: F811
    """Along a random direction the loss changes as the gradients say: the forward pass's own outputs, from bfloat16 inputs that differ by whole steps."""
    import torch
    say("attention backward against differences")
    with Case(ctx, [40, 90, 7], heads=4, kv_heads=2, dim=32, buckets=16, distance=40, dtype="float16", window=(50, 20), sinks=2) as c:
        g = torch.Generator("cuda:0").manual_seed(5)
        out, lse = c.run()
        grads = backward(c, out, lse)
        for name, grad in zip(("q", "k", "v", "bias"), grads):
            x = getattr(c, name)
            old = x.clone()
            d = torch.sign(grad.float()) + (grad == 0)  # the steepest direction, where the change is largest against the roundings
            h = 2.0 ** -6
            loss = []
            for sign in (1, -1):
                x.copy_((old.float() + sign * h * d).to(x.dtype))
                moved = x.double() - old.double()
                o = c.sequences().forward(c.step)[0]  # in 64 bits, of the moved inputs
                near = c.run(keep=False)
                loss.append(((c.dout.double() * near.double()).sum(), (c.dout.double() * o).sum(), (grad.double() * moved).sum(), (c.dout.abs().double() * o.abs()).sum()))
            x.copy_(old)
            change, exact, said = (float(loss[0][i] - loss[1][i]) for i in range(3))
            # third-order terms: h^2 of a change; outputs are off by two half steps of fp16 of theirs
            assert abs(exact - said) <= 0.02 * abs(said), (name, exact, said)
            assert abs(change - said) <= 0.02 * abs(said) + 4 * c.step * float(loss[0][3]), (name, change, said)


def test_captured_and_replayed():
    """Forward and backward in one graph, while eager calls of the same inputs live; replays with new inputs."""
    import torch
    import paper_2506_08276_amd as L
    say("attention backward, captured")
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        own = L.leann_create(CTX, torch.zeros(640, device="cuda:0"), stream=stream.cuda_stream)
        with Case(own, [100, 2, 260], heads=2, buckets=32, distance=128, packed=True) as c:
            def step():
                out, lse = c.run()
                return (out, lse, *backward(c, out, lse))
            eager = step()
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                captured = step()
            for i in range(3):
                c.q.normal_()
                c.bias.normal_()
                graph.replay()
                stream.synchronize()
                for a, b in zip(captured, step()):
                    assert torch.equal(a, b), i
                torch.zeros(1000, device="cuda:0").sum().item()
            assert eager[0].shape == captured[0].shape
            del graph
        stream.synchronize()
        L.leann_destroy(own)


def test_a_workspace_that_grows_behind_a_capture():
    """A graph keeps the workspace that its capture met: a larger call, and what is allocated then, changes nothing in its replays."""
    import torch
    import paper_2506_08276_amd as L
    say("attention backward, a workspace that grows")
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        own = L.leann_create(CTX, torch.zeros(640, device="cuda:0"), stream=stream.cuda_stream)
        args = dict(buckets=32, distance=128)
        with Case(own, [3, 9], k_rows=[2500, 700], **args) as c, Case(own, [4000, 300], packed=True, **args) as large:
            def step(of):
                out, lse = of.run()
                return (out, lse, *backward(of, out, lse))
            eager = step(c)
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                captured = step(c)
            for i in range(3):
                other = step(large)
                rest = [torch.full((1 << 22,), float("nan"), device="cuda:0") for _ in range(4)]
                graph.replay()
                stream.synchronize()
                for a, b in zip(captured, eager):
                    assert torch.equal(a, b), i
                for a, b in zip(step(large), other):
                    assert torch.equal(a, b), i
                del rest
            del graph
        stream.synchronize()
        L.leann_destroy(own)


def test_refusals(ctx):  # noqa: F811
    import torch
    import paper_2506_08276_amd as L
    say("attention backward refusals")
    with Case(ctx, [20], packed=True) as c:
        out, lse = c.run()
        free = torch.empty((20, 256), dtype=c.q.dtype, device="cuda:0")
        for bad in (dict(dq=c.q), dict(dk=c.k), dict(dv=c.dout), dict(dq=out), dict(dq=free, dk=free), dict(dk=free, dv=free)):
            with pytest.raises(L.LeannError) as e:
                backward(c, out, lse, **bad)
            assert e.value.status == -1
        for bad in (lse[:3], lse.double(), lse.t()):
            with pytest.raises(AssertionError):
                backward(c, out, bad)
        with pytest.raises(AssertionError):
            backward(c, out[:19], lse)
        lib = L.load_library()
        rc = lib.leann_attention_backward(ctx, c.plan, *[v for t in (c.dout, c.q, c.k, c.v, out) for v in (t.data_ptr(), t.stride(0))], lse.data_ptr(), 1, 0.125, None,
                                          *[v for t in (torch.empty_like(free), torch.empty_like(free), torch.empty_like(free)) for v in (t.data_ptr(), 256)], free.data_ptr())
        assert rc == -1  # a gradient of no bias
