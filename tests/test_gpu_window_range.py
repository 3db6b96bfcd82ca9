"""quake_attention_window where its probabilities or scores are far apart: scores up
to the stated |t q.k| of 1e6, and binary16 rows whose sink takes the row max while
thousands of keys lie far below it. Scores are sums of two products that binary32
holds exactly, so the references below need no bound for them."""
import math

import numpy as np
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


def attend(s, v, mode, t, seen, dt):
    """(o, bound) of scores s [rows, keys] (exact) and values v [keys, dim], float64.

    y = s c0 with the binary32 c0 that the library folds. A probability is off by ARG
    + FEW (and the mode's jump) of itself, then rounded to dt by half a step (twice
    where a later max rescales it); binary16's steps are at least 2^-24, against a
    largest probability of the row of at least 2^6 at any time. The quotient's both
    sides carry that; sums of n terms 2^-24 n, the result half a step."""
    c0 = float(np.float32(t / ref64.LN2)) if mode == 0 else float(np.float32(t / ref64.LN2 * 2.0 ** 23)) / 2.0 ** 23
    y = (s * c0).masked_fill(~seen, -math.inf)
    p = ref64.real_exp2(y - torch.ceil(y.amax(-1, keepdim=True)), mode)
    total = p.sum(-1, keepdim=True)
    o = p @ v / total
    eps, n = torch.finfo(dt).eps, seen.sum(-1, keepdim=True).double()
    e = p * (ref64.ARG + ref64.FEW + ref64.jump(mode) + eps)
    if dt == torch.float16:
        e = e + 2 * 2.0 ** -25 / 2.0 ** 6 * p.amax(-1, keepdim=True) * seen
    # sum p' v / sum p' - o = sum (p' - p) (v - o) / sum p'
    dev = (e @ v.abs() + e.sum(-1, keepdim=True) * o.abs()) / (total - e.sum(-1, keepdim=True))
    mean = p @ v.abs() / total
    bound = 1.01 * dev + (n + 8) * 2.0 ** -24 * (mean + o.abs()) + o.abs() * eps / 2
    return o, 1.01 * bound + (2.0 ** -25 if dt == torch.float16 else 2.0 ** -126)


def check(name, o, want, bound):
    say(name)
    torch.cuda.synchronize()
    off = (o.double() - want).abs()
    bad = ~(off <= bound)
    if bad.any():
        at = tuple(bad.nonzero()[0].tolist())
        raise AssertionError("%s: %d of %d out of bound, first at %s: %s for %s, bound %s" % (
            name, int(bad.sum()), bad.numel(), at, o[at].item(), want[at].item(), bound[at].item()))


def both(q, name, qq, k, v, dt, mode, t, window, sinks=0):
    """One key head and sequence, repeated until 128 rows share a workgroup where they
    are many; with a workspace and without."""
    sq, skv = qq.shape[0], k.shape[0]
    pos = torch.arange(sq, device="cuda")[:, None] + skv - sq
    j = torch.arange(skv, device="cuda")[None]
    seen = (j <= pos) & ((j > pos - window) | (j < sinks))
    want, bound = attend(qq.double() @ k.double().T.contiguous(), v.double(), mode, t, seen, dt)
    for b in (1, 300) if sq >= 96 else (1,):
        x = [a[None, :, None].expand(b, -1, -1, -1).contiguous() for a in (qq, k, v)]
        for ws in (None, q.attention_window_workspace(x[0], x[1], window, sinks)):
            o = q.quake_attention_window(*x, window=window, sinks=sinks, mode=mode, t=t, workspace=ws)
            check("%s %s mode %d b %d %s" % (name, dt, mode, b, ws is not None), o[0, :, 0], want, bound)
            assert torch.equal(o, o[:1].expand_as(o))


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


@pytest.mark.parametrize("dt", HALF, ids=["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sq", [1, 120])
def test_scores_up_to_the_stated_bound(q, dt, d, sq):
    skv, t = 600, 0.125
    g = gen(d + sq)
    fine = torch.randint(-128, 128, (skv,), generator=g, device="cuda").float() / 2   # t s: 8 either way
    v = torch.randn((skv, d), generator=g, device="cuda").to(dt)
    qq = torch.zeros((sq, d), device="cuda")
    qq[:, 0], qq[:, 1] = 2048.0, 1.0                 # t q.k = 256 k_0 + k_1 / 8
    ramp = torch.arange(skv, device="cuda") // 60    # 0 .. 9
    # about 999424 = 256 * 3904 all over, or the row max rising to that from far below
    for name, base in (("high", torch.full((skv,), 3904.0, device="cuda")),
                       ("low", torch.full((skv,), -3904.0, device="cuda")),
                       ("last", torch.where(ramp < 9, -3904.0, 3904.0)),
                       ("first", torch.where(ramp > 0, -3904.0, 3904.0)),
                       ("rising", (ramp.float() - 5.0) * 768.0)):
        k = torch.zeros((skv, d), device="cuda")
        k[:, 0], k[:, 1] = base, fine
        for mode in (0, 1, 2, 3):
            both(q, "scores " + name, qq.to(dt), k.to(dt), v, dt, mode, t, 10 ** 6)


@pytest.mark.parametrize("far", [10.0, 15.5, 18.0, 20.0])
@pytest.mark.parametrize("sq", [1, 120])
def test_binary16_sinks_far_above_the_other_keys(q, far, sq):
    # all keys but the first `far` base-2 units below it, about, where binary16
    # probabilities relative to the largest are subnormal from 2^-14 on; in the values the
    # sink is 0 (the others are all there is), 1 (their mean is exactly that), or random
    skv, d, dt = 9000, 64, torch.float16
    g = gen(int(far * 2) + sq)
    fine = torch.randint(-32, 33, (skv,), generator=g, device="cuda").float() / 64
    qq = torch.zeros((sq, d), device="cuda")
    qq[:, 0] = 1.0
    for last in (False, True):                       # the largest key first, or the newest ones
        k = torch.zeros((skv, d), device="cuda")
        k[:, 0] = fine - far * ref64.LN2
        if last:
            k[skv - sq:, 0] = fine[skv - sq:] / 8
        else:
            k[0, 0] = 0.0
        v = torch.randn((skv, d), generator=g, device="cuda")
        v[:, 0] = 1.0
        v[:, 1] = 1.0
        v[(slice(skv - sq, skv) if last else slice(0, 1)), 1] = 0.0
        for mode in (0, 1, 2, 3):
            both(q, "sink %s %s" % (far, last), qq.to(dt), k.to(dt), v.to(dt), dt, mode, 1.0, 8700, 1)


@pytest.mark.parametrize("far", [20.3, 22.6, 25.4])
@pytest.mark.parametrize("sq", [1, 120])
def test_binary16_keys_of_one_weight_far_below_their_sink(q, far, sq):
    # the same probability in every key, so that its rounding does not average out: held
    # against a largest one of 1 it would be off by up to half of itself, or lost
    skv, d, dt = 9000, 64, torch.float16
    qq = torch.zeros((sq, d), device="cuda")
    qq[:, 0] = 1.0
    k = torch.zeros((skv, d), device="cuda")
    k[1:, 0] = -far * ref64.LN2
    v = torch.ones((skv, d), device="cuda")
    v[0, 1:] = 0.0
    for mode in (0, 1, 2, 3):
        both(q, "one weight %s" % far, qq.to(dt), k.to(dt), v.to(dt), dt, mode, 1.0, 8700, 1)


@pytest.mark.parametrize("dt", HALF, ids=["bf16", "f16"])
def test_many_rows_that_could_be_split_without_a_workspace(q, dt):
    # 128 rows of each of 4 key heads over 9000 keys: 16 workgroups of 32 rows, each
    # walking all of them where the call has no workspace
    g = gen(3)
    x = [torch.randn(s, generator=g, device="cuda").to(dt)
         for s in ((1, 64, 8, 64), (1, 9000, 4, 64), (1, 9000, 4, 64))]
    want, bound, _ = ref64.window_attention(*x, 8000, 5, 2, 0.125)
    for ws in (None, q.attention_window_workspace(x[0], x[1], 8000, 5)):
        o = q.quake_attention_window(*x, window=8000, sinks=5, t=0.125, workspace=ws)
        check("unsplit %s %s" % (dt, ws is None), o, want, bound)
