"""quake_attention_shared on the GPU against plain 64-bit attention, element by element
within the bounds ref64_cache.shared_attention derives."""
import math

import pytest
import torch

import ref64_cache as ref
from gpu_util import say

pytestmark = pytest.mark.gpu
HALF = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def q():
    from paper_2412_00408_amd import quake
    return quake


def make(b, groups, sq, sp, skv, h, hk, d, dt, seed=0):
    """q, k, v, prefix_k, prefix_v"""
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + b * 31 + sq + skv + sp)

    def n(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(dt)
    x = [n(b, sq, h, d), n(b, skv, hk, d), n(b, skv, hk, d)]
    return x + ([n(groups, sp, hk, d), n(groups, sp, hk, d)] if sp else [None, None])


def within(name, got, want, bound, live=None):
    bad = ~((got.double() - want).abs() <= bound)
    if live is not None:
        bad &= live
    if bad.any():
        at = bad.nonzero()[0].tolist()
        raise AssertionError("%s: %d of %d out of bound, first at %s: %s for %s, bound %s" % (
            name, int(bad.sum()), bad.numel(), at, got[tuple(at)].item(), want[tuple(at)].item(),
            bound[tuple(at)].item()))


def check(name, o, w, want):
    say(name)
    torch.cuda.synchronize()
    within(name + " o", o, want[0], want[1], want[2][:, :, None, None])
    if w is not None:
        within(name + " weight", w, want[3], want[4])


def weights(x, seed=3):
    b, skv, hk = x[1].shape[:3]
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.rand((b, hk, skv), generator=g, device="cuda")


SHAPES = [
    # batch, groups, sq, sp, skv, heads, kv_heads, dim
    (1, 1, 1, 0, 1, 1, 1, 64),
    (1, 1, 1, 1, 1, 3, 1, 128),
    (4, 1, 1, 500, 64, 8, 2, 64),
    (2, 2, 1, 33, 31, 8, 8, 128),
    (12, 3, 1, 130, 65, 8, 1, 64),
    (6, 1, 1, 700, 40, 40, 1, 128),            # more than one tile of a sequence's heads
    (48, 1, 1, 1500, 70, 4, 2, 128),
    (40, 2, 1, 2100, 130, 6, 2, 64),
    (3, 1, 7, 50, 7, 5, 5, 64),
    (8, 2, 5, 333, 97, 10, 2, 128),
    (2, 1, 200, 100, 200, 4, 4, 64),
    (4, 2, 129, 257, 300, 4, 2, 128),
    (2, 1, 33, 0, 65, 6, 2, 128),
    (1, 1, 513, 0, 513, 3, 1, 64),
    (3, 3, 64, 640, 64, 2, 1, 64),
    (1, 1, 1, 9000, 20, 8, 1, 128),
    (130, 1, 1, 900, 5, 1, 1, 64),
    (5, 5, 40, 1000, 900, 8, 2, 64),
    (16, 1, 12, 1234, 48, 4, 1, 128),
]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dt", HALF, ids=["bf16", "f16"])
def test_shapes(q, shape, dt):
    x = make(*shape, dt)
    t = 1.0 / math.sqrt(shape[-1])
    for mode in (0, 1, 2, 3):
        w0 = weights(x)
        want = ref.shared_attention(*x, mode=mode, t=t, weight=w0)
        ws = q.attention_shared_workspace(x[0], x[1], x[3])
        o = q.quake_attention_shared(*x, mode=mode, workspace=ws)
        check("%s %s mode %d" % (shape, dt, mode), o, None, want)
        o = q.quake_attention_shared(*x, mode=mode)
        check("%s %s mode %d, no workspace" % (shape, dt, mode), o, None, want)
        w = w0.clone()
        o = q.quake_attention_shared(*x, weight=w, mode=mode,
                                     workspace=q.attention_shared_workspace(x[0], x[1], x[3], weigh=True))
        check("%s %s mode %d, weighed" % (shape, dt, mode), o, w, want)


@pytest.mark.parametrize("dt", HALF, ids=["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sq,skv", [(1, 700), (40, 700), (300, 300)])
def test_ragged_lengths_and_rows_left_alone(q, dt, d, sq, skv):
    b, groups, sp, h, hk = 8, 4, 130, 6, 2
    x = make(b, groups, sq, sp, skv, h, hk, d, dt, 1)
    # none, one, a few, all, more than the buffers hold, negative; fewer keys than queries
    kl = torch.tensor([0, 1, skv // 3, skv, skv + 50, -5, min(3, skv), 64], dtype=torch.int32, device="cuda")
    ql = torch.tensor([sq, 1, sq // 2, sq, sq + 9, sq, sq, 0], dtype=torch.int32, device="cuda")
    pl = torch.tensor([0, 1, sp + 3, 77], dtype=torch.int32, device="cuda")
    for i in range(b):                           # slots past the length: anything
        n = int(kl[i].clamp(0, skv))
        x[1][i, n:] = math.nan
        x[2][i, n:] = math.inf
        x[0][i, int(ql[i].clamp(0, sq)):] = math.nan
    for i in range(groups):
        n = int(pl[i].clamp(0, sp))
        x[3][i, n:] = math.inf
        x[4][i, n:] = math.nan
    lens = dict(prefix_lens=pl, q_lens=ql, kv_lens=kl)
    w0 = weights(x)
    want = ref.shared_attention(*x, t=0.1, weight=w0, **lens)
    for weigh in (False, True):
        for ws in (None, q.attention_shared_workspace(x[0], x[1], x[3], weigh=weigh)):
            if weigh and ws is None:
                continue
            o, w = torch.full_like(x[0], 7.0), w0.clone() if weigh else None
            got = q.quake_attention_shared(*x, o, weight=w, t=0.1, workspace=ws, **lens)
            assert got is o
            check("ragged %s" % ([sq, skv, d, weigh, ws is not None],), o, w, want)
            assert (o[~want[2]] == 7.0).all()
            assert (o[0][:ql[0]] == 0).all()     # no key: zeros
            for i in range(b if weigh else 0):   # slots behind a cache, and no query: as they were
                n = int(kl[i].clamp(0, skv)) if int(ql[i]) > 0 else 0
                assert torch.equal(w[i, :, n:], w0[i, :, n:])


def test_rows_without_keys(q):
    x = make(2, 2, 3, 0, 5, 4, 2, 64, torch.bfloat16, 2)
    w = torch.zeros((2, 2, 5), device="cuda")
    kl = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    ws = q.attention_shared_workspace(x[0], x[1], weigh=True)
    o = q.quake_attention_shared(*x, weight=w, kv_lens=kl, workspace=ws)
    assert (o[0] == 0).all() and (o[1, :2] == 0).all() and torch.equal(o[1, 2], x[2][1, 0].repeat_interleave(2, 0))
    assert torch.equal(w, torch.tensor([0.0, 2.0], device="cuda")[:, None, None].expand(2, 2, 5)
                       * (torch.arange(5, device="cuda") == 0))
    none = make(2, 1, 3, 7, 1, 4, 2, 64, torch.bfloat16, 2)      # no slots at all: the prefix alone
    want = ref.shared_attention(none[0], none[1][:, :0], none[2][:, :0], *none[3:])
    for ws in (None, q.attention_shared_workspace(none[0], none[1][:, :0], none[3])):
        o = q.quake_attention_shared(none[0], none[1][:, :0], none[2][:, :0], *none[3:], workspace=ws)
        check("no slots", o, None, want)
    w = torch.zeros((2, 2, 0), device="cuda")                    # nor any weight
    o = q.quake_attention_shared(none[0], none[1][:, :0], none[2][:, :0], *none[3:], weight=w)
    check("no slots, a weight", o, None, want)
    ws = torch.empty(4096, dtype=torch.uint8, device="cuda")     # no keys at all
    for sq in (3, 300):
        y = torch.randn((2, sq, 4, 64), device="cuda").to(torch.bfloat16)
        o = q.quake_attention_shared(y, none[1][:, :0], none[2][:, :0], weight=w, workspace=ws)
        assert (o == 0).all()


def test_scores_that_keep_rising_and_extreme_scores(q):
    for dt in HALF:
        for sq in (1, 40):
            x = make(20, 2, sq, 640, 320, 8, 2, 64, dt, 3)
            up = (torch.ones_like(x[0]) * 3).to(dt)
            for scale in (0.5, 4.0, -4.0):
                k = (x[1].float() * 0.1 + torch.linspace(-1, 1, 320, device="cuda")[None, :, None, None] * scale).to(dt)
                pk = (x[3].float() * 0.1 - torch.linspace(-1, 1, 640, device="cuda")[None, :, None, None] * scale).to(dt)
                for mode in (0, 2):
                    w = torch.zeros((20, 2, 320), device="cuda")
                    want = ref.shared_attention(up, k, x[2], pk, x[4], mode=mode, t=0.5)
                    ws = q.attention_shared_workspace(up, k, pk, weigh=True)
                    o = q.quake_attention_shared(up, k, x[2], pk, x[4], weight=w, mode=mode, t=0.5, workspace=ws)
                    check("ramp %s %s %s %d" % (dt, sq, scale, mode), o, w, want)


def test_strided_views(q):
    # a fused projection's q, k and v, heads outside the tokens, a prefix inside a larger cache,
    # a prefix that groups share, weights of a longer cache
    b, s, h, hk, d = 4, 50, 6, 2, 64
    g = torch.Generator(device="cuda").manual_seed(5)
    qkv = torch.randn((b, s, h + 2 * hk, d), generator=g, device="cuda").to(torch.bfloat16)
    big = torch.randn((2, 2, hk, 300, d), generator=g, device="cuda").to(torch.bfloat16)
    pk, pv = big[0].permute(0, 2, 1, 3)[:, 10:200], big[1].permute(0, 2, 1, 3)[:, 10:200]
    x = (qkv[:, :, :h], qkv[:, :, h:h + hk], qkv[:, :, h + hk:], pk, pv)
    want = ref.shared_attention(*x)
    out = torch.empty((b, h, s, d), dtype=torch.bfloat16, device="cuda").permute(0, 2, 1, 3)
    w = torch.zeros((hk, b, 200), device="cuda").permute(1, 0, 2)[..., :s]
    ws = q.attention_shared_workspace(x[0], x[1], pk, weigh=True)
    check("views", q.quake_attention_shared(*x, out, weight=w, workspace=ws), w, want)
    one = (x[0], x[1], x[2], pk[:1].expand(2, -1, -1, -1), pv[:1].expand(2, -1, -1, -1))
    want = ref.shared_attention(*one)
    for ws in (None, q.attention_shared_workspace(x[0], x[1], one[3])):
        check("expanded", q.quake_attention_shared(*one, workspace=ws), None, want)


def test_offsets_past_32_bits(q):
    # sequences and groups 2^31 elements apart in one buffer
    far, d = (1 << 31) + 64, 64
    x = make(3, 3, 1, 70, 40, 4, 1, d, torch.bfloat16, 6)
    buf = torch.empty(2 * far + 8192, dtype=torch.bfloat16, device="cuda")
    k = buf.as_strided((3, 40, 1, d), (far, d, d, 1))
    pk = buf[4096:].as_strided((3, 50, 1, d), (far, d, d, 1))
    k.copy_(x[1])
    pk.copy_(x[3][:, :50])
    w = torch.empty(2 * far + 64, dtype=torch.float32, device="cuda").as_strided((3, 1, 40), (far, 40, 1))
    w.zero_()
    want = ref.shared_attention(x[0], k, x[2], pk, x[4][:, :50])
    ws = q.attention_shared_workspace(x[0], k, pk, weigh=True)
    check("far apart", q.quake_attention_shared(x[0], k, x[2], pk, x[4][:, :50], weight=w, workspace=ws), w, want)


def test_long_prefix_and_long_cache(q):
    x = make(2, 1, 1, 100000, 30, 8, 1, 128, torch.bfloat16, 7)
    want = ref.shared_attention(*x, t=0.08)
    ws = q.attention_shared_workspace(x[0], x[1], x[3])
    check("100000 prefix keys", q.quake_attention_shared(*x, t=0.08, workspace=ws), None, want)
    x = make(1, 1, 1, 40, 100000, 8, 2, 64, torch.float16, 8)
    w = weights(x)
    want = ref.shared_attention(*x, t=0.08, weight=w)
    ws = q.attention_shared_workspace(x[0], x[1], x[3], weigh=True)
    check("100000 own keys", q.quake_attention_shared(*x, weight=w, t=0.08, workspace=ws), w, want)


def test_very_many_sequences(q):
    # more tiles than are joined in one launch: every sequence reads the prefix for itself
    b = 70000
    for sq, weigh in ((1, True), (1, False), (9, True)):
        x = make(b, 1, sq, 20, 10, 8, 4, 64, torch.bfloat16, 12)
        w = weights(x) if weigh else None
        w0 = w.clone() if weigh else None
        ws = q.attention_shared_workspace(x[0], x[1], x[3], weigh=weigh)
        o = q.quake_attention_shared(*x, weight=w, workspace=ws)
        for at in (slice(0, 3), slice(b // 2, b // 2 + 3), slice(b - 3, b)):
            want = ref.shared_attention(x[0][at], x[1][at], x[2][at], x[3], x[4], weight=w0[at] if weigh else None)
            check("many sequences %s %s %s" % (sq, weigh, at), o[at], w[at] if weigh else None, want)


def test_agrees_with_windowed_attention(q):
    # no prefix: the windowed operator with a window of the whole length; and a prefix is
    # what the same keys in front of every sequence's own would be
    x = make(6, 1, 9, 200, 100, 8, 2, 128, torch.bfloat16, 9)
    want = ref.shared_attention(*x, t=0.125)
    k = torch.cat([x[3].expand(6, -1, -1, -1), x[1]], 1)
    v = torch.cat([x[4].expand(6, -1, -1, -1), x[2]], 1)
    check("windowed", q.quake_attention_window(x[0], k, v, t=0.125), None, want)
    ws = q.attention_shared_workspace(x[0], x[1], x[3])
    check("shared", q.quake_attention_shared(*x, t=0.125, workspace=ws), None, want)


def test_weight_sums_to_the_rows(q):
    # every row spreads a weight of 1 over its keys
    for sq, skv in ((1, 900), (300, 300)):
        x = make(3, 1, sq, 0, skv, 8, 2, 64, torch.bfloat16, 10)
        w = torch.zeros((3, 2, skv), device="cuda")
        ws = q.attention_shared_workspace(x[0], x[1], weigh=True)
        for i in range(1, 4):
            q.quake_attention_shared(*x, weight=w, workspace=ws)
            total = w.double().sum(2)
            assert (total - i * 4 * sq).abs().max() <= i * 4 * sq * (skv + 4 * sq) * 2.0 ** -23


CALLS = [(2, 1, 1, 0, 900, 8, 2, 128), (24, 2, 1, 1500, 70, 8, 2, 64), (16, 1, 6, 900, 48, 4, 1, 128),
         (4, 2, 150, 300, 150, 8, 4, 128)]


@pytest.mark.parametrize("shape", CALLS, ids=str)
@pytest.mark.parametrize("weigh", [False, True])
def test_same_bits_every_time_on_other_streams_and_in_graphs(q, shape, weigh):
    x = make(*shape, torch.bfloat16, 11)
    ws = q.attention_shared_workspace(x[0], x[1], x[3], weigh=weigh)

    def call(o=None, ws=ws, **kw):
        w = torch.zeros(x[1].shape[0], x[1].shape[2], x[1].shape[1], device="cuda") if weigh else None
        o = q.quake_attention_shared(*x, o, weight=w, workspace=ws, **kw)
        return [o, w] if weigh else [o]
    want = call()
    for fill in (0, 0xFF):                         # a larger workspace full of anything
        big = torch.full(((0 if ws is None else ws.numel()) + 4096,), fill, dtype=torch.uint8, device="cuda")
        assert all(torch.equal(a, c) for a, c in zip(call(ws=big), want))
        assert (big[-4096:] == fill).all()
    torch.cuda.synchronize()
    got = []
    streams = [torch.cuda.Stream() for _ in range(3)]
    spaces = [None if ws is None else torch.empty_like(ws) for _ in streams]
    for _ in range(3):
        for s, w in zip(streams, spaces):
            with torch.cuda.stream(s):
                got.append(call(ws=w))
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for g in got for a, c in zip(g, want))
    graphs, outs = [], []                          # two graphs that share a workspace
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(call())
        graphs.append(graph)
    for i in range(3):
        for a, c in zip(x, make(*shape, torch.bfloat16, 20 + i)):
            if a is not None:
                a.copy_(c)
        want = call()
        for graph, o in zip(graphs, outs):
            for a in o:
                a.fill_(3.0)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, c) for a, c in zip(o, want)), i
