"""Attention over ragged sequences on the GPU against its definition in 64 bits."""
import numpy as np
import pytest

from attention64 import Sequences, assert_near
from gpu_util import say

pytestmark = pytest.mark.gpu
CTX = dict(layers=0, hidden=128, heads=2, ffn=128, vocab=1, max_pos=1)


@pytest.fixture(scope="module")
def ctx():
    import torch
    import paper_2506_08276_amd as L
    c = L.leann_create(CTX, torch.zeros(640, device="cuda:0"))
    yield c
    L.leann_destroy(c)


class Case:
    """Inputs and plan of one call."""

    def __init__(self, ctx, q_rows, k_rows=None, first=None, heads=4, kv_heads=None, dim=64, window=None, sinks=0, buckets=0, distance=0, both=True,
                 dtype="bfloat16", packed=False, pad=0, seed=0, spread=1.3):
        import torch
        import paper_2506_08276_amd as L
        self.L, self.ctx, self.torch = L, ctx, torch
        g = torch.Generator("cuda:0").manual_seed(seed)
        kv = heads if kv_heads is None else kv_heads
        dtype = getattr(torch, dtype)
        self.step = torch.finfo(dtype).eps / 2
        Tq, Tk = int(np.sum(q_rows)), int(np.sum(q_rows if k_rows is None else k_rows))
        make = lambda rows, cols: (spread * torch.randn((rows, cols), generator=g, device="cuda:0")).to(dtype)
        if packed:
            qkv = make(Tq, (heads + 2 * kv) * dim + pad)
            self.q, self.k, self.v = qkv[:, :heads * dim], qkv[:, heads * dim:(heads + kv) * dim], qkv[:, (heads + kv) * dim:(heads + 2 * kv) * dim]
        else:
            self.q, self.k, self.v = make(Tq, heads * dim + pad)[:, :heads * dim], make(Tk, kv * dim + pad)[:, :kv * dim], make(Tk, kv * dim + pad)[:, :kv * dim]
        self.dout = (0.1 * torch.randn((Tq, heads * dim), generator=g, device="cuda:0")).to(dtype)
        self.bias = torch.randn((buckets, heads), generator=g, device="cuda:0") if buckets else None
        self.table = L.leann_position_buckets(buckets, distance, both) if buckets else None
        self.args = dict(heads=heads, head_dim=dim, kv_heads=kv, first=first, window=window, sinks=sinks, bucket_of=self.table)
        self.q_rows, self.k_rows = q_rows, k_rows
        self.plan = L.leann_attention_create(ctx, q_rows, k_rows, **self.args)
        self.scale = dim ** -0.5

    def __enter__(self):
        return self

    def __exit__(self, *_):
        self.L.leann_attention_free(self.plan)

    def sequences(self):
        a = self.args
        return Sequences(self.q, self.k, self.v, self.q_rows, self.q_rows if self.k_rows is None else self.k_rows,
                         [0] * len(self.q_rows) if a["first"] is None else a["first"], a["heads"], a["kv_heads"], a["head_dim"],
                         (-1, -1) if a["window"] is None else a["window"], a["sinks"], self.bias, self.table, self.scale)

    def run(self, keep=True, out=None):
        return self.L.leann_attention(self.ctx, self.plan, self.q, self.k, self.v, bias=self.bias, keep=keep, out=out)

    def check(self):
        out, lse = self.run()
        want, want_lse, far, far_lse = self.sequences().forward(self.step)
        assert_near(out, want, far, "out")
        assert_near(lse, want_lse, far_lse, "lse")
        return out, lse


CASES = {
    "one token": dict(q_rows=[1], heads=1),
    "one query": dict(q_rows=[12], heads=12),
    "lengths around tiles": dict(q_rows=[0, 1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 0], packed=True),
    "fp16": dict(q_rows=[5, 130, 77], dtype="float16", packed=True),
    "shared key heads": dict(q_rows=[70, 3, 129], heads=6, kv_heads=2, packed=True, pad=8),
    "head size 32": dict(q_rows=[70, 3, 129], dim=32, dtype="float16"),
    "head size 40": dict(q_rows=[70, 3, 129], dim=40, packed=True),
    "head size 8": dict(q_rows=[17, 66], dim=8),
    "head size 96": dict(q_rows=[70, 3, 129], dim=96, heads=2, dtype="float16"),
    "head size 128": dict(q_rows=[70, 3, 129, 300], dim=128, heads=4, kv_heads=1, pad=8),
    "bias": dict(q_rows=[3, 64, 129, 300, 40], buckets=32, distance=128, packed=True),
    "bias, one direction": dict(q_rows=[3, 64, 129, 300], window=(-1, 0), buckets=16, distance=50, both=False, packed=True),
    "bias, far": dict(q_rows=[1500], heads=2, buckets=64, distance=1024),
    "bias, near": dict(q_rows=[700, 33], heads=2, buckets=8, distance=5, dtype="float16"),
    "window": dict(q_rows=[5, 64, 129, 500], window=(30, 30), packed=True),
    "window of one": dict(q_rows=[5, 64, 129], window=(0, 0)),
    "window and first tokens": dict(q_rows=[5, 64, 129, 700], window=(30, 17), sinks=4),
    "first tokens beyond a tile": dict(q_rows=[800, 90], window=(10, 0), sinks=70, buckets=32, distance=128),
    "nothing behind, nothing ahead": dict(q_rows=[200], window=(0, -1)),
    "few queries, long keys": dict(q_rows=[1, 3, 1, 16], k_rows=[5000, 1, 0, 777], heads=2, buckets=32, distance=128),
    "last queries": dict(q_rows=[1, 4, 1], k_rows=[3000, 4, 1], first=[2999, 0, 0], window=(100, 0), sinks=2, heads=2),
    "last queries, long": dict(q_rows=[1, 9], k_rows=[9000, 20000], first=[8999, 19991], heads=3, kv_heads=1, dim=128, dtype="float16"),
    "128 queries, keys in parts": dict(q_rows=[40, 130, 1], k_rows=[3000, 2100, 5], heads=2, buckets=32, distance=128),
    "keys in parts, some hidden": dict(q_rows=[200, 33], k_rows=[2500, 1700], first=[1500, 1667], window=(-1, 0), heads=4, kv_heads=2, dim=128, dtype="float16"),
    "keys in parts behind first ones": dict(q_rows=[150], k_rows=[4000], first=[3800], window=(2000, 0), sinks=70, heads=2, dim=32),
    "queries that see nothing": dict(q_rows=[40, 100], k_rows=[10, 0], first=[5, 0], window=(3, 3)),
    "long, split": dict(q_rows=[2000], heads=1),
    "long, first tokens, shared heads": dict(q_rows=[2500, 1300], heads=6, kv_heads=1, dim=32, window=(40, 40), sinks=3, dtype="float16", packed=True),
    "many short": dict(q_rows=[1 + i % 9 for i in range(700)], heads=3, packed=True),
}


@pytest.mark.parametrize("name", CASES)
def test_against_the_definition(ctx, name):
    say("attention", name)
    with Case(ctx, **CASES[name]) as c:
        c.check()


def test_scores_of_any_size(ctx):
    """One key's score far above the others, all far below zero, and a scale given."""
    say("attention, large scores")
    with Case(ctx, [70, 130], spread=8.0) as c:
        c.check()
        c.scale = 0.7
        out = c.L.leann_attention(ctx, c.plan, c.q, c.k, c.v, scale=0.7)
        want, _, far, _ = c.sequences().forward(c.step)
        assert_near(out, want, far, "out")
        c.scale = -0.05
        out = c.L.leann_attention(ctx, c.plan, c.q, c.k, c.v, scale=-0.05)
        want, _, far, _ = c.sequences().forward(c.step)
        assert_near(out, want, far, "out")


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_biases_that_hide(ctx, dtype):
    """A bias of -inf, and of fp32's lowest value, hides a key; a row that has no other sees nothing, or all alike."""
    import torch
    say("attention, hiding biases")
    with Case(ctx, [5, 200], buckets=32, distance=128, window=(20, 20), dtype=dtype) as c:
        c.bias[3:9] = -float("inf")
        c.check()
        c.bias[:] = -float("inf")
        out, lse = c.run()
        assert not out.any() and bool((lse == -float("inf")).all())
        c.bias[:] = torch.finfo(torch.float32).min
        out, _ = c.run()
        for rows, keys, see, _ in c.sequences().parts():  # the scores are lost against it: all that a query sees weighs the same, up to the roundings of weights and result
            v = c.v[keys].double()
            mean = see.double() @ v / see.sum(1, keepdim=True)
            assert_near(out[rows], mean, c.step * (see.double() @ v.abs() / see.sum(1, keepdim=True) * (1 + c.step) + mean.abs()) + 1e-6, "out")


@pytest.mark.parametrize("window,sinks", [((30, 30), 0), ((64, 0), 3), ((-1, 0), 0)])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_what_is_hidden_does_not_reach_a_query(ctx, window, sinks, value):
    import torch
    say("attention, infinities", window, value)
    with Case(ctx, [90, 150, 40], window=window, sinks=sinks, heads=2) as c:
        clean, _ = c.run()
        c.k[100], c.v[130, 5:70], c.v[239, 3] = value, value, value
        out, _ = c.run()
        s = c.sequences()
        reached = torch.zeros(len(out), dtype=torch.bool, device="cuda:0")
        for rows, keys, see, _ in s.parts():
            for j in (100, 130, 239):
                if keys.start <= j < keys.stop:
                    reached[rows] |= see[:, j - keys.start]
        assert torch.equal(out[~reached], clean[~reached])
        assert bool((~torch.isfinite(out[reached])).any(1).all())
        # an infinite value makes its own columns infinite or NaN, and no others
        only_v = torch.zeros_like(reached)
        for rows, keys, see, _ in s.parts():
            for j in (130, 239):
                if keys.start <= j < keys.stop:
                    only_v[rows] |= see[:, j - keys.start]
            if keys.start <= 100 < keys.stop:
                only_v[rows] &= ~see[:, 100 - keys.start]
        columns = torch.zeros(out.shape[1], dtype=torch.bool, device="cuda:0")
        columns[3] = columns[5:70] = True
        assert torch.equal(out[only_v][:, ~columns], clean[only_v][:, ~columns])


def test_rows_and_columns_around_stay(ctx):
    import torch
    say("attention into a slice")
    with Case(ctx, [70, 3], heads=2, packed=True, pad=16) as c:
        whole = torch.full((80, 160), 7.0, dtype=c.q.dtype, device="cuda:0")
        c.run(out=whole[2:75, 8:136])
        assert torch.equal(whole[2:75, 8:136], c.run(keep=False))
        whole[2:75, 8:136] = 7
        assert bool((whole == 7).all())


def test_bits_repeat_and_sequences_are_apart(ctx):
    """The same call gives the same bits; a sequence's do not depend on the others' values."""
    say("attention, twice")
    with Case(ctx, [150, 40, 300], packed=True, buckets=32, distance=128) as c:
        a, la = c.run()
        b, lb = c.run()
        assert c.torch.equal(a, b) and c.torch.equal(la, lb)
        c.q[150:190] = float("nan")
        d, _ = c.run()
        assert c.torch.equal(a[:150], d[:150]) and c.torch.equal(a[190:], d[190:])


def test_captured_and_replayed():
    """A context on a stream of its own, captured; replays with new inputs, other work between them."""
    import torch
    import paper_2506_08276_amd as L
    say("attention, captured")
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        own = L.leann_create(CTX, torch.zeros(640, device="cuda:0"), stream=stream.cuda_stream)
        with Case(own, [1, 2], k_rows=[4000, 3000], heads=2, buckets=32, distance=128) as c:
            out = torch.empty((3, 128), dtype=c.q.dtype, device="cuda:0")
            c.run(keep=False, out=out)
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                c.run(keep=False, out=out)
            for i in range(3):
                c.q.normal_()
                c.v.normal_()
                graph.replay()
                stream.synchronize()
                got = out.clone()
                assert torch.equal(got, c.run(keep=False)), i
                torch.zeros(1000, device="cuda:0").sum().item()
            del graph
        stream.synchronize()
        L.leann_destroy(own)


def test_offsets_beyond_32_bits(ctx):
    import torch
    say("attention over 2.3e9 elements of keys")
    rows = 3_000_000
    with Case(ctx, [2], k_rows=[128], heads=12) as small:
        far = torch.zeros((rows, 768), dtype=torch.bfloat16, device="cuda:0")
        k, v = far, far.clone()
        k[-128:], v[-128:] = small.k, small.v
        plan = small.L.leann_attention_create(ctx, [0, 2], [rows - 128, 128], heads=12, head_dim=64)
        assert torch.equal(small.L.leann_attention(ctx, plan, small.q, k, v), small.run(keep=False))
        small.L.leann_attention_free(plan)
        plan = small.L.leann_attention_create(ctx, [2], [rows], heads=12, head_dim=64)
        out = small.L.leann_attention(ctx, plan, small.q, k, v).double()  # rows - 128 keys with a score of 0 and a value of 0
        small.L.leann_attention_free(plan)
        want, lse, far_off, _ = small.sequences().forward(small.step)
        share = 1 / (1 + (rows - 128) * torch.exp(-lse))
        want = want.view(2, 12, 64) * share.t()[:, :, None]
        assert_near(out, want.reshape(2, 768), far_off.view(2, 12, 64).mul(share.t()[:, :, None]).reshape(2, 768) + 2.0 ** -20 * want.abs().reshape(2, 768), "out")


def test_refusals(ctx):
    import torch
    import paper_2506_08276_amd as L
    say("attention refusals")

    def refused(status, what, **changed):
        args = dict(q_rows=[4], heads=2, head_dim=64)
        args.update(changed)
        with pytest.raises(L.LeannError) as e:
            L.leann_attention_create(ctx, args.pop("q_rows"), args.pop("k_rows", None), **args)
        assert e.value.status == status, what

    for what, changed in {"length": dict(q_rows=[-1]), "keys": dict(k_rows=[-2]), "first": dict(first=[-1]), "window": dict(window=(-2, 0)),
                          "sinks": dict(sinks=-1), "bucket": dict(bucket_of=[0, -1, 0])}.items():
        refused(-1, what, **changed)
    for what, changed in {"heads": dict(heads=0), "share": dict(heads=3, kv_heads=2), "dim": dict(head_dim=60), "wide": dict(head_dim=136),
                          "far": dict(first=[1 << 30]), "distance": dict(bucket_of=np.zeros(2051, int)), "buckets": dict(bucket_of=[0, 4096, 0])}.items():
        refused(-4, what, **changed)
    with Case(ctx, [20], packed=True) as c:
        for bad in (c.q, c.k, c.v):
            with pytest.raises(L.LeannError):
                L.leann_attention(ctx, c.plan, c.q, c.k, c.v, out=bad)
        for scale in (float("inf"), float("nan"), 0.0, 1e-7, 2e6):
            with pytest.raises(L.LeannError):
                L.leann_attention(ctx, c.plan, c.q, c.k, c.v, scale=scale)
        wide = torch.zeros((20, 260), dtype=c.q.dtype, device="cuda:0")
        with pytest.raises(L.LeannError):
            L.leann_attention(ctx, c.plan, wide[:, :256], c.k, c.v)  # rows 260 elements apart
        with pytest.raises(L.LeannError):
            L.leann_attention(ctx, c.plan, wide.view(-1)[1:5121].view(20, 256), c.k, c.v)  # not aligned
        for bad in (c.q[:19], c.q.float(), c.q.half()):
            with pytest.raises(AssertionError):
                L.leann_attention(ctx, c.plan, bad, c.k, c.v)
        with pytest.raises(AssertionError):
            L.leann_attention(ctx, c.plan, c.q, c.k, c.v, bias=torch.zeros((4, 4), device="cuda:0"))
    for buckets, distance, both in ((1, 5, False), (3, 5, True), (32, 8, True), (32, 1025, True), (2, 4, True)):
        with pytest.raises(L.LeannError):
            L.leann_position_buckets(buckets, distance, both)
