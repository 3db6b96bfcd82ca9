"""quake_attention_window on the GPU against plain 64-bit attention, element by
element within the bound ref64.window_attention derives."""
import math

import pytest
import torch

import ref64
from gpu_util import say

pytestmark = pytest.mark.gpu
HALF = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def q():
    from paper_2412_00408_amd import quake
    return quake


def make(b, sq, skv, h, hk, d, dt, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + b * 31 + sq + skv)

    def n(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(dt)
    return n(b, sq, h, d), n(b, skv, hk, d), n(b, skv, hk, d)


def check(name, o, ref, what="o"):
    want, bound, written = ref
    say(name)
    torch.cuda.synchronize()
    off = (o.double() - want).abs()
    bad = ~(off <= bound) & written[:, :, None, None]
    if bad.any():
        at = bad.nonzero()[0].tolist()
        raise AssertionError("%s: %d of %d %s out of bound, first at %s: %s for %s, bound %s" % (
            name, int(bad.sum()), bad.numel(), what, at, o[tuple(at)].item(), want[tuple(at)].item(),
            bound[tuple(at)].item()))


SHAPES = [
    # batch, sq, skv, heads, kv_heads, dim, window, sinks
    (1, 1, 1, 1, 1, 64, 1, 0),
    (1, 1, 1, 3, 1, 128, 5, 2),
    (1, 1, 300, 8, 2, 64, 256, 4),
    (2, 1, 33, 8, 8, 128, 32, 1),
    (2, 1, 4097, 8, 1, 128, 1000, 5),
    (1, 1, 5000, 40, 1, 64, 4096, 0),          # more than one tile of heads
    (3, 7, 7, 5, 5, 64, 3, 1),
    (2, 33, 65, 6, 2, 128, 16, 40),            # sinks longer than the window
    (1, 200, 200, 4, 4, 64, 2 ** 31 - 1, 0),   # causal
    (1, 129, 129, 4, 2, 128, 129, 0),          # window of the whole length
    (2, 130, 1111, 10, 2, 128, 200, 33),
    (1, 513, 513, 3, 1, 64, 64, 0),
    (1, 64, 640, 2, 1, 64, 100, 2 ** 31 - 1),  # every key a sink
    (2, 257, 700, 6, 3, 128, 1, 0),            # itself alone
    (1, 1500, 1500, 4, 1, 128, 700, 7),
    (1, 160, 3000, 2, 2, 64, 2500, 3),         # rows that share tiles, keys split
    (1, 100, 9000, 1, 1, 128, 9000, 0),
    (1, 97, 600, 1, 1, 64, 500, 100),
]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dt", HALF, ids=["bf16", "f16"])
def test_shapes(q, shape, dt):
    b, sq, skv, h, hk, d, window, sinks = shape
    x = make(b, sq, skv, h, hk, d, dt)
    t = 1.0 / math.sqrt(d)
    for mode in (0, 1, 2, 3):
        ref = ref64.window_attention(*x, window, sinks, mode, t)
        ws = q.attention_window_workspace(x[0], x[1], window, sinks)
        o = q.quake_attention_window(*x, window=window, sinks=sinks, mode=mode, workspace=ws)
        check("%s %s mode %d" % (shape, dt, mode), o, ref)
        if ws is not None:
            o = q.quake_attention_window(*x, window=window, sinks=sinks, mode=mode)
            check("%s %s mode %d unsplit" % (shape, dt, mode), o, ref)


@pytest.mark.parametrize("dt", HALF, ids=["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sq,skv", [(1, 700), (40, 700), (300, 300)])
def test_ragged_lengths_and_rows_left_alone(q, dt, d, sq, skv):
    b, h, hk, window, sinks = 7, 6, 2, 100, 3
    x = make(b, sq, skv, h, hk, d, dt, 1)
    # none, one, a few, all, more than the buffers hold, negative; fewer keys than queries
    kl = torch.tensor([0, 1, skv // 3, skv, skv + 50, -5, min(3, skv)], dtype=torch.int32, device="cuda")
    ql = torch.tensor([sq, 1, sq // 2, sq, sq + 9, sq, sq], dtype=torch.int32, device="cuda")
    for i in range(b):                           # keys past the length: anything
        n = int(kl[i].clamp(0, skv))
        x[1][i, n:] = math.nan
        x[2][i, n:] = math.inf
    ref = ref64.window_attention(*x, window, sinks, 2, 0.1, ql, kl)
    for ws in (None, q.attention_window_workspace(x[0], x[1], window, sinks)):
        o = torch.full_like(x[0], 7.0)
        got = q.quake_attention_window(*x, o, window=window, sinks=sinks, q_lens=ql, kv_lens=kl,
                                       t=0.1, workspace=ws)
        assert got is o
        check("ragged %s" % ([b, sq, skv, d, ws is not None],), o, ref)
        assert (o[~ref[2]] == 7.0).all()
        assert (o[0][:ql[0]] == 0).all()         # no key: zeros


def test_keys_outside_the_window_are_not_read(q):
    x = make(1, 1, 900, 4, 2, 64, torch.bfloat16, 2)
    ref = ref64.window_attention(*x, 100, 5, 2, 0.125)
    x[1][:, 5:800] = math.nan
    x[2][:, 5:800] = math.nan
    check("evicted keys", q.quake_attention_window(*x, window=100, sinks=5, t=0.125), ref)


def test_scores_that_keep_rising_and_extreme_scores(q):
    # the running exponent is raised block after block, and falls far behind
    for dt in HALF:
        x = make(1, 40, 640, 4, 2, 64, dt, 3)
        ramp = torch.linspace(-1, 1, 640, device="cuda")[None, :, None, None]
        up = (torch.ones_like(x[0][..., :1]) * 3).to(dt).expand_as(x[0]).contiguous()
        for scale in (0.5, 4.0, -4.0):
            k = (x[1].float() * 0.1 + ramp * scale).to(dt)
            for mode in (0, 2):
                ref = ref64.window_attention(up, k, x[2], 600, 4, mode, 0.5)
                check("ramp %s %s %d" % (dt, scale, mode), q.quake_attention_window(
                    up, k, x[2], window=600, sinks=4, mode=mode, t=0.5), ref)


def test_equal_scores_give_the_mean(q):
    x = make(1, 70, 70, 4, 4, 128, torch.bfloat16, 4)
    z = torch.zeros_like(x[1])
    ref = ref64.window_attention(x[0], z, x[2], 64, 0, 2, 1.0)
    check("mean", q.quake_attention_window(x[0], z, x[2], window=64, t=1.0), ref)


def test_strided_views(q):
    # a fused projection's q, k and v; caches with the heads outside the tokens
    b, s, h, hk, d = 2, 150, 6, 2, 64
    g = torch.Generator(device="cuda").manual_seed(5)
    qkv = torch.randn((b, s, h + 2 * hk, d), generator=g, device="cuda").to(torch.bfloat16)
    x = (qkv[:, :, :h], qkv[:, :, h:h + hk], qkv[:, :, h + hk:])
    ref = ref64.window_attention(*x, 50, 3, 2, 0.125)
    out = torch.empty((b, h, s, d), dtype=torch.bfloat16, device="cuda").permute(0, 2, 1, 3)
    check("fused qkv", q.quake_attention_window(*x, out, window=50, sinks=3), ref)
    k = x[1].permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    v = x[2].permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    check("heads first", q.quake_attention_window(x[0], k, v, window=50, sinks=3), ref)
    one = k[:1].expand(b, -1, -1, -1)               # a prompt that all sequences share
    ref = ref64.window_attention(x[0], one, v, 50, 3, 2, 0.125)
    check("expanded", q.quake_attention_window(x[0], one, v, window=50, sinks=3), ref)


def test_offsets_past_32_bits(q):
    # sequences 2^31 elements apart in one cache buffer
    far, d = (1 << 31) + 64, 64
    buf = torch.empty(2 * far + 4096, dtype=torch.bfloat16, device="cuda")
    k = buf.as_strided((3, 64, 1, d), (far, d, d, 1))[:, :40]
    v = torch.empty_like(buf).as_strided((3, 64, 1, d), (far, d, d, 1))[:, :40]
    x = make(3, 1, 40, 4, 1, d, torch.bfloat16, 6)
    k.copy_(x[1])
    v.copy_(x[2])
    ref = ref64.window_attention(*x, 30, 2, 2, 0.125)
    check("far apart", q.quake_attention_window(x[0], k, v, window=30, sinks=2), ref)


def test_long_cache_token(q):
    x = make(1, 1, 200000, 8, 1, 128, torch.bfloat16, 7)
    ref = ref64.window_attention(*x, 2 ** 31 - 1, 0, 2, 0.08)
    ws = q.attention_window_workspace(x[0], x[1], 2 ** 31 - 1)
    assert ws is not None
    check("200000 keys", q.quake_attention_window(*x, t=0.08, workspace=ws), ref)


def test_no_keys_and_more_queries_than_keys(q):
    for sq in (1, 40, 200):
        x = make(2, sq, 8, 6, 2, 64, torch.float16, 10)
        o = q.quake_attention_window(x[0], x[1][:, :0], x[2][:, :0], window=5)
        assert (o == 0).all()
        ref = ref64.window_attention(*x, 5, 1, 2, 0.125)
        o = q.quake_attention_window(*x, window=5, sinks=1)
        check("sq %d over 8 keys" % sq, o, ref)
        if sq > 8:
            assert (o[:, :sq - 8] == 0).all()
    with pytest.raises(q.QuakeError):                # rows of the output on one another
        x = make(2, 3, 8, 4, 2, 64, torch.float16, 11)
        q.quake_attention_window(*x, x[0][:, :, :1].clone().expand(2, 3, 4, 64), window=5)


def test_same_bits_every_time_on_another_stream_and_in_a_graph(q):
    for sq in (1, 200):
        x = make(2, sq, 900, 8, 2, 128, torch.bfloat16, 8)
        ws = q.attention_window_workspace(x[0], x[1], 500, 4)
        kw = dict(window=500, sinks=4, workspace=ws)
        want = q.quake_attention_window(*x, **kw)
        o = torch.zeros_like(want)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            q.quake_attention_window(*x, o, **kw)
        side.synchronize()
        assert torch.equal(o, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            q.quake_attention_window(*x, o, **kw)
        for i in range(4):
            y = make(2, sq, 900, 8, 2, 128, torch.bfloat16, 20 + i)
            for a, c in zip(x, y):
                a.copy_(c)
            o.fill_(3.0)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, q.quake_attention_window(*x, **kw)), i


def test_agrees_with_attention(q):
    # window of the whole length: causal attention of quake_attention, up to the
    # factor that the two take their exponentials against
    x = make(1, 300, 300, 4, 4, 64, torch.bfloat16, 9)
    a = q.quake_attention(*(i[0].transpose(0, 1).contiguous() for i in x[:2]),
                          x[2][0].permute(1, 2, 0).contiguous(), mode=0, causal=True)
    o = q.quake_attention_window(*x, mode=0)
    ref = ref64.window_attention(*x, 2 ** 31 - 1, 0, 0, 0.125)
    check("window", o, ref)
    check("attention", a.transpose(0, 1)[None], ref)


# From 96 rows a key head on, the sequences repeated until workgroups of 32 rows outnumber
# the compute units, and long walks of few rows: the form with 128 rows a workgroup.
def repeats(shape):
    b, sq, _, h, hk = shape[:5]
    return 1 + 256 // (b * hk * -(-sq * (h // hk) // 32))


LARGE = [s for s in SHAPES if s[1] * s[3] // s[4] >= 96] + [
    (1, 130, 200, 4, 4, 128, 2 ** 31 - 1, 0),
    (1, 100, 9000, 8, 8, 64, 9000, 0),         # 32 workgroups share a tile's keys
    (1, 128, 9000, 8, 8, 128, 8500, 9),
]


@pytest.mark.parametrize("shape", LARGE, ids=str)
@pytest.mark.parametrize("dt", HALF, ids=["bf16", "f16"])
def test_many_rows(q, shape, dt):
    b, sq, skv, h, hk, d, window, sinks = shape
    one = make(b, sq, skv, h, hk, d, dt, 11)
    n = 1 if hk * skv > 50000 else repeats(shape)
    x = [a.repeat(n, 1, 1, 1) for a in one]
    t = 1.0 / math.sqrt(d)
    for mode in (0, 1, 2, 3):
        ref = ref64.window_attention(*one, window, sinks, mode, t)
        for ws in (None, q.attention_window_workspace(x[0], x[1], window, sinks)):
            o = q.quake_attention_window(*x, window=window, sinks=sinks, mode=mode, workspace=ws)
            check("many rows %s %s mode %d %s" % (shape, dt, mode, ws is not None), o[:b], ref)
            assert torch.equal(o.view(n, -1), o[:b].reshape(1, -1).expand(n, -1))


def test_many_rows_with_scores_that_keep_rising_and_ragged_lengths(q):
    for dt in HALF:
        x = make(32, 70, 640, 8, 4, 64, dt, 12)      # 640 workgroups of 32 rows
        ramp = torch.linspace(-1, 1, 640, device="cuda")[None, :, None, None]
        up = (torch.ones_like(x[0]) * 3).to(dt)
        kl = torch.arange(0, 640, 20, dtype=torch.int32, device="cuda")
        ql = torch.arange(70, 6, -2, dtype=torch.int32, device="cuda")
        for scale in (0.5, 4.0, -4.0):
            k = (x[1].float() * 0.1 + ramp * scale).to(dt)
            for lens in ((None, None), (ql, kl)):
                ref = ref64.window_attention(up, k, x[2], 600, 4, 2, 0.5, *lens)
                o = torch.full_like(x[0], 7.0)
                q.quake_attention_window(up, k, x[2], o, window=600, sinks=4, t=0.5, q_lens=lens[0],
                                         kv_lens=lens[1])
                check("many rows, ramp %s %s %s" % (dt, scale, lens[0] is not None), o, ref)
                assert (o[~ref[2]] == 7.0).all()


def test_many_rows_same_bits_in_a_graph(q):
    x = make(6, 200, 900, 8, 2, 128, torch.bfloat16, 13)   # 300 workgroups of 32 rows
    ws = q.attention_window_workspace(x[0], x[1], 500, 4)
    assert ws is not None
    eager = q.quake_attention_window(*x, window=500, sinks=4, workspace=ws)
    o = torch.empty_like(eager)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        q.quake_attention_window(*x, o, window=500, sinks=4, workspace=ws)
    for _ in range(4):
        o.zero_()
        graph.replay()
        again = q.quake_attention_window(*x, window=500, sinks=4, workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(o, eager) and torch.equal(again, eager)
