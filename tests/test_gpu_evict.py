"""quake_cache_evict on the GPU against the choice by whole numbers and a plain copy, bit
for bit; and a run of the cache operators together."""
import math

import pytest
import torch

import ref64_cache as ref
from gpu_util import say
from test_gpu_shared import check, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q():
    from paper_2412_00408_amd import quake
    return quake


def cache(b, skv, hk, d, dt, seed, kind="spread"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    k, v = (torch.randn((b, skv, hk, d), generator=g, device="cuda").to(dt) for _ in range(2))
    w = torch.randn((b, hk, skv), generator=g, device="cuda")
    if kind == "spread":
        w = (w * 3).exp_()
    elif kind == "ties":
        w = (w * 2).round_()                      # -0 and 0 among them
    elif kind == "one":
        w.fill_(0.25)
    elif kind == "odd":
        w = torch.where(w > 1.5, math.inf, torch.where(w < -1.5, -math.inf, w))
        w = w.masked_fill(torch.rand(w.shape, generator=g, device="cuda") < 0.3, math.nan)
    elif kind == "rising":
        w = torch.arange(skv, device="cuda").float().expand(b, hk, skv).contiguous()
    elif kind == "falling":
        w = -torch.arange(skv, device="cuda").float().expand(b, hk, skv).contiguous()
    elif kind == "tiny":                          # denormal, next to one another
        w = torch.randint(0, 50, w.shape, generator=g, device="cuda", dtype=torch.int32).view(torch.float32)
    return k, v, w


def same(name, got, want):
    say(name)
    torch.cuda.synchronize()
    for what, a, c in zip(("k", "v", "weight", "lens", "kept", "evicted"), got, want):
        if a is None:
            continue
        a = a.cpu()
        bits = {2: torch.int16, 4: torch.int32}[a.element_size()]
        assert torch.equal(a.contiguous().view(bits), c.contiguous().view(bits)), (name, what)


def both(q, name, k, v, w, budget, sinks, recent, lens, extra=5):
    """Into another cache, then in place."""
    b, skv, hk, d = k.shape
    size = budget + extra
    out = [torch.full((b, size, hk, d), 7.0, dtype=k.dtype, device="cuda") for _ in range(2)]
    out += [torch.full((b, hk, size), 9.0, device="cuda"), torch.full((b,), -9, dtype=torch.int32, device="cuda")]
    want = ref.evict(k, v, w, budget, sinks, recent, lens, *out[:3])
    kept, evicted = q.quake_cache_evict(k, v, w, budget, sinks, recent, kv_lens=lens, out=out)
    same(name + " into another", out + [kept, evicted], want)
    if budget > skv:
        return
    want = ref.evict(k, v, w, budget, sinks, recent, lens, k, v, w)
    kept, evicted = q.quake_cache_evict(k, v, w, budget, sinks, recent, kv_lens=lens)
    same(name + " in place", [k, v, w, lens, kept, evicted], want)


SHAPES = [
    # batch, slots, key heads, dim, budget, sinks, recent
    (1, 2, 1, 8, 1, 0, 0),
    (1, 2, 1, 64, 1, 1, 0),
    (2, 64, 3, 64, 63, 4, 8),
    (2, 65, 1, 128, 64, 0, 64),
    (3, 300, 2, 64, 100, 1, 16),
    (1, 1000, 2, 80, 999, 3, 5),
    (2, 1025, 4, 128, 400, 200, 200),           # nothing chosen by weight
    (1, 5000, 1, 256, 700, 33, 0),
    (4, 2500, 8, 64, 2048, 4, 128),
    (40, 300, 8, 128, 111, 2, 31),              # as many rows as workgroups fill the GPU
    (1, 40, 1, 64, 100, 5, 7),                  # a budget beyond the slots
    (1, 70, 2, 4096, 33, 1, 1),
]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_shapes(q, shape, dt):
    b, skv, hk, d, budget, sinks, recent = shape
    for kind in ("spread", "ties"):
        both(q, "%s %s %s" % (shape, dt, kind), *cache(b, skv, hk, d, dt, 1, kind), budget, sinks, recent, None)


@pytest.mark.parametrize("kind", ["spread", "ties", "one", "odd", "rising", "falling", "tiny"])
def test_weights_of_all_kinds_and_ragged_lengths(q, kind):
    b, skv, hk, d = 7, 900, 2, 64
    lens = torch.tensor([900, 0, 1, 200, 201, 5000, -3], dtype=torch.int32, device="cuda")
    both(q, kind, *cache(b, skv, hk, d, torch.float16, 2, kind), 200, 3, 20, lens.clone())
    both(q, kind + ", no sinks", *cache(b, skv, hk, d, torch.float16, 3, kind), 200, 0, 0, lens.clone())


def test_long_rows(q):
    for kind in ("spread", "one", "rising"):
        k, v, w = cache(1, 200000, 1, 64, torch.bfloat16, 4, kind)
        both(q, "200000 " + kind, k, v, w, 4096, 4, 1000, None)
    both(q, "a large budget", *cache(1, 100000, 1, 64, torch.bfloat16, 5), 99000, 0, 0, None)


def test_evicting_again_changes_nothing(q):
    k, v, w = cache(2, 600, 2, 64, torch.bfloat16, 6)
    lens = torch.tensor([600, 500], dtype=torch.int32, device="cuda")
    q.quake_cache_evict(k, v, w, 300, 2, 50, kv_lens=lens)
    was = [a.clone() for a in (k, v, w, lens)]
    kept, evicted = q.quake_cache_evict(k, v, w, 300, 2, 50, kv_lens=lens)
    assert all(torch.equal(a, c) for a, c in zip((k, v, w, lens), was))
    assert (evicted == 0).all() and torch.equal(kept, torch.arange(300, device="cuda").int().expand(2, 2, 300))


def test_views(q):
    # heads first, K and V interleaved in one cache, a part of a longer one
    g = torch.Generator(device="cuda").manual_seed(7)
    for what in ("heads first", "interleaved", "part"):
        b, skv, hk, d = 3, 400, 2, 64
        shape, order = {"heads first": ((2, b, hk, skv, d), (0, 1, 3, 2, 4)),
                        "interleaved": ((b, skv, 2, hk, d), (2, 0, 1, 3, 4)),
                        "part": ((2, b, skv + 60, hk + 1, d), (0, 1, 2, 3, 4))}[what]
        kv = torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)
        before = kv.clone()
        k, v = kv.permute(order)[:, :, :skv, :hk]
        w = torch.randn((hk, b, skv + 3), generator=g, device="cuda").permute(1, 0, 2)[..., :skv]
        lens = torch.tensor([400, 399, 90], dtype=torch.int32, device="cuda")
        both(q, what, k, v, w, 100, 2, 10, lens)
        if what == "part":
            assert torch.equal(kv[:, :, skv:], before[:, :, skv:])
            assert torch.equal(kv[..., hk:, :], before[..., hk:, :])


def test_offsets_past_32_bits(q):
    far, d = (1 << 31) + 64, 64
    buf = torch.empty(2 * far + 8192, dtype=torch.bfloat16, device="cuda")
    k = buf.as_strided((3, 50, 1, d), (far, d, d, 1))
    v = buf[4096:].as_strided((3, 50, 1, d), (far, d, d, 1))
    x = cache(3, 50, 1, d, torch.bfloat16, 8)
    k.copy_(x[0])
    v.copy_(x[1])
    both(q, "far apart", k, v, x[2], 20, 1, 5, None)


def test_very_many_rows(q):
    b, hk = 1 << 18, 4
    k, v, w = cache(b, 12, hk, 8, torch.bfloat16, 11, "ties")
    lens = torch.randint(0, 13, (b,), dtype=torch.int32, device="cuda")
    out = [torch.zeros((b, 8, hk, 8), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    out += [torch.zeros((b, hk, 8), device="cuda"), torch.zeros(b, dtype=torch.int32, device="cuda")]
    kept, evicted = q.quake_cache_evict(k, v, w, 6, 1, 2, kv_lens=lens, out=out)
    torch.cuda.synchronize()
    for at in (slice(0, 40), slice(b // 2, b // 2 + 40), slice(b - 40, b)):
        zero = [torch.zeros_like(a[at]) for a in out[:3]]
        want = ref.evict(k[at], v[at], w[at], 6, 1, 2, lens[at], *zero)
        same("many rows %s" % at, [a[at] for a in out] + [kept[at], evicted[at]], want)
    part = slice(b - 40, b)
    want = ref.evict(k[part], v[part], w[part], 6, 1, 2, lens[part], k[part], v[part], w[part])
    kept, evicted = q.quake_cache_evict(k, v, w, 6, 1, 2, kv_lens=lens)
    same("many rows in place", [a[part] for a in (k, v, w, lens, kept, evicted)], want)
    with pytest.raises(q.QuakeError):                # 2^20 rows are the most
        y = torch.empty((1 << 18, 1, 5, 8), dtype=torch.bfloat16, device="cuda")
        q.quake_cache_evict(y, y.clone(), torch.empty((1 << 18, 5, 1), device="cuda"), 1)


def test_no_slots_and_no_sequences(q):
    e = torch.empty((2, 0, 1, 64), dtype=torch.bfloat16, device="cuda")
    out = [torch.ones((2, 8, 1, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    out += [torch.ones((2, 1, 8), device="cuda"), torch.ones(2, dtype=torch.int32, device="cuda")]
    kept, evicted = q.quake_cache_evict(e, e.clone(), torch.empty((2, 1, 0), device="cuda"), 5, out=out)
    assert (kept == -1).all() and (evicted == 0).all() and (out[2] == 0).all() and (out[3] == 0).all()
    assert (out[0] == 1).all()
    z = torch.empty((0, 5, 1, 64), dtype=torch.bfloat16, device="cuda")
    kept, evicted = q.quake_cache_evict(z, z, torch.empty((0, 1, 5), device="cuda"), 3)
    assert kept.shape == (0, 1, 3) and evicted.shape == (0,)


def test_streams_and_graphs(q):
    x = cache(4, 700, 2, 128, torch.bfloat16, 9)
    lens = torch.tensor([700, 650, 300, 40], dtype=torch.int32, device="cuda")
    want = ref.evict(*x, 256, 4, 32, lens, *x)
    for s in (torch.cuda.Stream(), torch.cuda.Stream()):
        y, ln = [a.clone() for a in x], lens.clone()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            kept, evicted = q.quake_cache_evict(*y, 256, 4, 32, kv_lens=ln)
        s.synchronize()
        same("stream", y + [ln, kept, evicted], want)
    y, ln = [a.clone() for a in x], lens.clone()
    kept, evicted = (torch.empty(n, dtype=torch.int32, device="cuda") for n in ((4, 2, 256), (4,)))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        q.quake_cache_evict(*y, 256, 4, 32, kv_lens=ln, kept=kept, evicted=evicted)
    for i in range(4):
        new = cache(4, 700, 2, 128, torch.bfloat16, 30 + i, "ties")
        for a, c in zip(y, new):
            a.copy_(c)
        ln.copy_(lens)
        graph.replay()
        torch.cuda.synchronize()
        same("graph %d" % i, y + [ln, kept, evicted], ref.evict(*new, 256, 4, 32, lens, *new))


def test_decoding_over_a_shared_prefix_with_a_bounded_cache(q):
    """As they are used: prompts, then tokens one by one; the caches are cut when full. The
    whole against 64-bit attention over the keys that are left at each step."""
    b, groups, sp, h, hk, d, slots, budget = 6, 2, 150, 8, 2, 64, 96, 60
    g = torch.Generator(device="cuda").manual_seed(10)
    n = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    pk, pv = n(groups, sp, hk, d), n(groups, sp, hk, d)
    k, v = (torch.zeros((b, slots, hk, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    w = torch.zeros((b, hk, slots), device="cuda")
    lens = torch.tensor([70, 96, 40, 61, 1, 90], dtype=torch.int32, device="cuda")
    for i, m in enumerate(lens.tolist()):
        k[i, :m], v[i, :m] = n(m, hk, d), n(m, hk, d)
    x = n(b, slots, h, d)
    lost = torch.zeros(b, dtype=torch.int32, device="cuda")
    for step in range(80):
        if step:
            x = n(b, 1, h, d)
            at = torch.arange(b, device="cuda")
            k[at, lens.long()], v[at, lens.long()] = n(b, hk, d), n(b, hk, d)
            lens += 1
        q_lens = lens if step == 0 else None
        want = ref.shared_attention(x, k, v, pk, pv, q_lens=q_lens, kv_lens=lens, weight=w)
        ws = q.attention_shared_workspace(x, k, pk, weigh=True)
        o = q.quake_attention_shared(x, k, v, pk, pv, weight=w, q_lens=q_lens, kv_lens=lens, workspace=ws)
        check("step %d" % step, o, w, want)
        if int(lens.max()) == slots:
            want = ref.evict(k, v, w, budget, 4, 8, lens, k, v, w)
            kept, evicted = q.quake_cache_evict(k, v, w, budget, 4, 8, kv_lens=lens)
            same("evict at %d" % step, [k, v, w, lens, kept, evicted], want)
            lost += evicted
    assert (lost > 0).all()
