"""Workloads of libquake's decoding operators as a user's program calls them:
attention over a key/value cache with a sliding window and sink tokens, drawing
the next token from LM-head logits, and distillation from a teacher's top logits.

A case is a dict of plain values with a "kind":

  window   batch, sq, skv, heads, kv_heads, dim, window, sinks, dtype, mode, ragged
           (sequences of different lengths in one padded batch)
  sample   rows, cols, dtype, mode, filters (text: which of k, p, m the rows use),
           masked (share of forbidden words), greedy (share of rows at temperature 0)
  distill  rows, cols, topk, dtype, mode, t, padded (short teacher lists), fused
           (loss and gradient in one call, or the loss first and its gradient later)

`run` computes a case through the library where `own` is true, else in plain
torch operations. `exact` is the definition in 64 bits, with QuAKE's exponential
as the real function of Eq. 2 and Eq. 6 (2^i times the polynomial of the fraction).
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
LN2 = math.log(2.0)
Q2M = tuple(map(float.fromhex, ("0x1.594830p-2", "-0x1.124f86p-6", "0x1.5cd076p-1")))


def listed() -> list[dict]:
    return [
        # the smallest call: one new token of one conversation, launch latency
        dict(name="window_decode_bf16_1x300", kind="window", batch=1, sq=1, skv=300, heads=8,
             kv_heads=2, dim=64, window=256, sinks=4, dtype="bf16", mode="quake2", ragged=False),
        # one decode step of a full batch over long caches: the cache's bytes
        dict(name="window_decode_bf16_64x8192", kind="window", batch=64, sq=1, skv=8192, heads=32,
             kv_heads=8, dim=128, window=4096, sinks=4, dtype="bf16", mode="quake2", ragged=True),
        # prefill of one long prompt, the largest product
        dict(name="window_prefill_bf16_16384", kind="window", batch=1, sq=16384, skv=16384,
             heads=32, kv_heads=8, dim=128, window=4096, sinks=4, dtype="bf16", mode="quake2",
             ragged=False),
        # prefill of a padded batch of short prompts, no sinks, a head of its own per key head
        dict(name="window_prefill_f16_4x1001", kind="window", batch=4, sq=1001, skv=1001, heads=16,
             kv_heads=16, dim=64, window=256, sinks=0, dtype="f16", mode="exact", ragged=True),
        # a few tokens per sequence against its cache: checking drafted tokens
        dict(name="window_chunk_f16_8x37", kind="window", batch=8, sq=37, skv=6000, heads=40,
             kv_heads=8, dim=128, window=2000, sinks=16, dtype="f16", mode="quake1", ragged=True),
        # next words of a batch of 64 over a 128256-word vocabulary, the usual filters together
        dict(name="sample_f32_64x128256_kp", kind="sample", rows=64, cols=128256, dtype="f32",
             mode="quake2", filters="kp", masked=0.0, greedy=0.0),
        # nucleus sampling over an odd vocabulary for a large batch
        dict(name="sample_bf16_256x50257_p", kind="sample", rows=256, cols=50257, dtype="bf16",
             mode="quake2m", filters="p", masked=0.0, greedy=0.0),
        # one conversation, no filter
        dict(name="sample_f32_1x32000", kind="sample", rows=1, cols=32000, dtype="f32",
             mode="quake2", filters="", masked=0.0, greedy=0.0),
        # constrained decoding: half the words forbidden, min-p, some rows greedy
        dict(name="sample_f16_32x128256_m", kind="sample", rows=32, cols=128256, dtype="f16",
             mode="quake1", filters="m", masked=0.5, greedy=0.25),
        # a training step's loss over 2048 tokens, the largest distillation
        dict(name="distill_bf16_2048x128256", kind="distill", rows=2048, cols=128256, topk=64,
             dtype="bf16", mode="quake2", t=0.5, padded=False, fused=True),
        # few tokens, binary32 logits, short lists padded, the gradient asked for later
        dict(name="distill_f32_37x50257", kind="distill", rows=37, cols=50257, topk=100,
             dtype="f32", mode="quake2", t=1.0, padded=True, fused=False),
        # a smaller vocabulary of odd length (rows that are not 16-byte aligned)
        dict(name="distill_f16_512x32001", kind="distill", rows=512, cols=32001, topk=20,
             dtype="f16", mode="exact", t=0.5, padded=True, fused=True),
    ]


def _log(rng, lo: int, hi: int) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case: dict) -> float:
    w = work(case)
    return w["bytes"] / 8e12 + w["flops"] / 2.5e15


def draw(rng) -> dict:
    mode = rng.choice(["quake2", "quake2", "quake1", "quake2m"])
    kind = rng.choice(["window", "window", "sample", "sample", "distill"])
    most = max(_cost(c) for c in listed() if c["kind"] == kind)
    while True:
        if kind == "window":
            kv = rng.choice([1, 2, 4, 8, 16])
            step = rng.choice(["one", "few", "all"])
            skv = _log(rng, 16, 16384)
            case = dict(kind=kind, batch=_log(rng, 1, 64),
                        sq=1 if step == "one" else min(skv, _log(rng, 2, 64)) if step == "few" else skv,
                        skv=skv, heads=kv * rng.choice([1, 2, 4, 5, 8]), kv_heads=kv,
                        dim=rng.choice([64, 128]), window=_log(rng, 16, 8192),
                        sinks=rng.choice([0, 1, 4, 33, 128]), dtype=rng.choice(["bf16", "f16"]),
                        mode=rng.choice([mode, "exact"]), ragged=rng.random() < 0.6)
            if case["batch"] * skv * kv * case["dim"] > 1 << 29:
                continue
        elif kind == "sample":
            case = dict(kind=kind, rows=_log(rng, 1, 256), cols=_log(rng, 64, 131072),
                        dtype=rng.choice(["f32", "f16", "bf16"]), mode=mode,
                        filters=rng.choice(["", "k", "p", "m", "kp", "kpm"]),
                        masked=rng.choice([0.0, 0.0, 0.9]), greedy=rng.choice([0.0, 0.2]))
        else:
            cols = _log(rng, 512, 131072)
            case = dict(kind=kind, rows=_log(rng, 1, 4096), cols=cols, topk=min(cols, _log(rng, 1, 256)),
                        dtype=rng.choice(["f32", "f16", "bf16"]), mode=rng.choice([mode, "exact"]),
                        t=rng.choice([0.5, 1.0]), padded=rng.random() < 0.5, fused=rng.random() < 0.6)
        if _cost(case) <= most:
            return case


# ---------------------------------------------------------------- inputs

def _lengths(case: dict) -> tuple[list[int], list[int]]:
    """Query and key lengths of the sequences of a window case (its own, whatever
    the seed): a batch padded to the longest, or all as long as the buffers."""
    b, sq, skv = case["batch"], case["sq"], case["skv"]
    if not case["ragged"]:
        return [sq] * b, [skv] * b
    r = random.Random(b * 1000003 + skv)
    kv = [skv] + [max(1, int(skv * r.uniform(0.1, 1.0))) for _ in range(b - 1)]
    if sq == skv:                                    # whole prompts: every key has its query
        return list(kv), kv
    return [min(n, sq if i == 0 else r.randint(1, sq)) for i, n in enumerate(kv)], kv


def _gen(seed: int) -> torch.Generator:
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(shape, std, dtype, g):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(std).to(dtype)


def _uniform(n, lo, hi, g):
    return torch.rand(n, generator=g, device="cuda").mul_(hi - lo).add_(lo)


def _window_inputs(c: dict, g) -> dict:
    dt, b, d = DTYPES[c["dtype"]], c["batch"], c["dim"]
    st = dict(q=_normal((b, c["sq"], c["heads"], d), 1.0, dt, g),
              k=_normal((b, c["skv"], c["kv_heads"], d), 1.0, dt, g),
              v=_normal((b, c["skv"], c["kv_heads"], d), 1.0, dt, g),
              o=torch.zeros((b, c["sq"], c["heads"], d), dtype=dt, device="cuda"))
    st["k"][:, :c["sinks"]] *= 1.5                   # first tokens draw attention
    ql, kl = _lengths(c)
    at = torch.randperm(b, generator=g, device="cuda")
    st["q_lens"] = torch.tensor(ql, dtype=torch.int32, device="cuda")[at]
    st["kv_lens"] = torch.tensor(kl, dtype=torch.int32, device="cuda")[at]
    return st


def _logits(rows, cols, dtype, g):
    x = torch.randn((rows, cols), generator=g, device="cuda").mul_(2.5)
    top = torch.randint(cols, (rows, 16), generator=g, device="cuda")    # a few likely words
    x.scatter_(1, top, torch.randn((rows, 16), generator=g, device="cuda").mul_(2.0).add_(14.0))
    return x.to(dtype)


def _sample_inputs(c: dict, g) -> dict:
    n = c["rows"]
    x = _logits(n, c["cols"], DTYPES[c["dtype"]], g)
    if c["masked"]:
        x.masked_fill_(torch.rand((n, c["cols"]), generator=g, device="cuda") < c["masked"], -math.inf)
    temp = _uniform(n, 0.5, 1.3, g)
    temp.masked_fill_(torch.rand(n, generator=g, device="cuda") < c["greedy"], 0.0)
    k = torch.randint(1, 101, (n,), generator=g, device="cuda", dtype=torch.int32)
    p, m = _uniform(n, 0.5, 0.98, g), _uniform(n, 0.001, 0.1, g)
    return dict(x=x, u=torch.rand(n, generator=g, device="cuda"), temperature=temp,
                top_k=k if "k" in c["filters"] else None, top_p=p if "p" in c["filters"] else None,
                min_p=m if "m" in c["filters"] else None)


def _distill_inputs(c: dict, g) -> dict:
    n, k = c["rows"], c["topk"]
    x = _logits(n, c["cols"], DTYPES[c["dtype"]], g)
    teacher = torch.randn(x.shape, generator=g, device="cuda").add_(x)
    y, idx = torch.topk(teacher, k, dim=1)
    idx = idx.int()
    if c["padded"]:                                  # lists of different lengths, -1 behind them
        kept = torch.randint(0, k + 1, (n, 1), generator=g, device="cuda")
        idx.masked_fill_(torch.arange(k, device="cuda") >= kept, -1)
    # the mean over the rows; binary16 gradients under a loss scale, as they are trained
    weight = _uniform(n, 0.5, 1.5, g).mul_((1024.0 if c["dtype"] == "f16" else 1.0) / n)
    weight.masked_fill_(torch.rand(n, generator=g, device="cuda") < 0.05, 0.0)   # prompt tokens
    return dict(x=x, idx=idx, y=y, weight=weight)


def _inputs(case: dict, seed: int) -> dict:
    make = dict(window=_window_inputs, sample=_sample_inputs, distill=_distill_inputs)[case["kind"]]
    return make(case, _gen(seed))


def prepare(case: dict, seed: int) -> dict:
    st = dict(case=case, **_inputs(case, seed))
    if own:
        from paper_2412_00408_amd import quake as q
        if case["kind"] == "window":
            st["workspace"] = q.attention_window_workspace(st["q"], st["k"], case["window"], case["sinks"])
        elif case["kind"] == "sample":
            st["workspace"] = q.sample_workspace(st["x"])
        else:
            st["workspace"] = q.distill_workspace(st["x"])
    return st


# ---------------------------------------------------------------- plain forms

def _pow2(l: torch.Tensor, mode: str) -> torch.Tensor:
    """The exponential of `mode` from its binary32 argument l = (y + 127) 2^23
    (base-2 exponent y): Eq. 3's integer, then Eq. 2 or Algorithm 1 on its bits."""
    if mode == "exact":
        return torch.exp2(l.double().div_(8388608.0).sub_(127.0)).float()
    z = l.clamp(0.0, 2139095040.0).to(torch.int32)
    if mode == "quake1":
        return z.view(torch.float32)
    a = ((z & 0x7FFFFF) | 0x3F800000).view(torch.float32)
    if mode == "quake2":
        y = (a.double().square().add_(2.0)).float() * (1.0 / 3.0)
    else:
        y = ((a.double() * Q2M[0] + Q2M[1]).float().double() * a.double() + Q2M[2]).float()
        y = torch.where(a == 1.0, a, y)
    return ((z & -8388608) | (y.view(torch.int32) & 0x7FFFFF)).view(torch.float32)


def _c0(t):
    """2^23 t / ln2 rounded to binary32, as a binary64 number."""
    return torch.as_tensor(t / LN2 * 8388608.0, dtype=torch.float64).float().double()


def _window_scores(st, i0, n, wide):
    """Scores [batch, kv head, query, group, key] of queries i0 .. i0 + n - 1, -inf where
    hidden, and the values [batch, kv head, key, dim] of the keys they may see."""
    c = st["case"]
    b, hk, d, w, sinks = c["batch"], c["kv_heads"], c["dim"], c["window"], c["sinks"]
    grp = c["heads"] // hk
    i = torch.arange(i0, i0 + n, device="cuda")
    pos = (st["kv_lens"] - st["q_lens"])[:, None] + i                             # [b, n]
    first = (pos[:, :1] - w + 1).clamp(min=0)
    band = first + torch.arange(min(c["skv"], w + n), device="cuda")              # [b, m]
    keys = torch.cat([torch.arange(min(sinks, c["skv"]), device="cuda").expand(b, -1), band], 1)
    again = (torch.arange(keys.shape[1], device="cuda") >= min(sinks, c["skv"])) & (keys < sinks)
    at = keys.clamp(max=c["skv"] - 1)[:, :, None, None].expand(-1, -1, hk, d)
    kk = st["k"].gather(1, at).to(wide).permute(0, 2, 3, 1).contiguous()          # [b, hk, d, m]
    vv = st["v"].gather(1, at).to(wide).permute(0, 2, 1, 3).contiguous()
    q = st["q"][:, i0:i0 + n].to(wide).view(b, n, hk, grp, d).permute(0, 2, 1, 3, 4).reshape(b, hk, n * grp, d)
    s = torch.matmul(q, kk).view(b, hk, n, grp, -1)
    j = keys[:, None, :]
    seen = (j <= pos[:, :, None]) & ((j > pos[:, :, None] - w) | (j < sinks)) & ~again[:, None, :]
    return s.masked_fill_(~seen[:, None, :, None, :], -math.inf), vv


def _window_blocks(st, wide, weigh):
    c = st["case"]
    b, sq, grp = c["batch"], c["sq"], c["heads"] // c["kv_heads"]
    o = torch.zeros(st["q"].shape, dtype=wide, device="cuda")
    step = max(1, min(sq, 512, (1 << 28) // (b * c["heads"] * min(c["skv"], c["window"] + 512))))
    for i0 in range(0, sq, step):
        n = min(step, sq - i0)
        s, vv = _window_scores(st, i0, n, wide)
        p = weigh(s)
        p = p / p.sum(-1, keepdim=True).clamp(min=1e-300 if wide == torch.float64 else 1e-38)
        part = torch.matmul(p.view(b, c["kv_heads"], n * grp, -1), vv).view(b, c["kv_heads"], n, grp, -1)
        o[:, i0:i0 + n] = part.permute(0, 2, 1, 3, 4).reshape(b, n, c["heads"], -1)
    late = torch.arange(sq, device="cuda")[None, :] >= st["q_lens"][:, None]
    return o.masked_fill_(late[:, :, None, None], 0.0)


def _row_exponent(top, t):
    """The whole number of binary digits that the row's largest entry is held against."""
    m = torch.ceil(top * (t / LN2))
    return torch.where(torch.isfinite(m), m, torch.zeros_like(m))


def _window_plain(st):
    t, mode = 1.0 / math.sqrt(st["case"]["dim"]), st["case"]["mode"]
    c0 = float(_c0(t))

    def weigh(s):
        top = _row_exponent(s.amax(-1, keepdim=True), t)
        hidden = s == -math.inf
        return _pow2(s.mul_(c0).add_((127.0 - top) * 8388608.0), mode).masked_fill_(hidden, 0.0)
    return _window_blocks(st, torch.float32, weigh).to(st["q"].dtype)


def _times(share: torch.Tensor, mass: torch.Tensor) -> torch.Tensor:
    """floor(share * mass) for share in [0, 1] cut to 24 binary digits, mass below 2^62."""
    f = (share.double() * 16777216.0).long()
    return f * (mass >> 24) + ((f * (mass & 0xFFFFFF)) >> 24)


def _sample_plain(st):
    x = st["x"].float()
    rows, cols = x.shape
    m = x.amax(1, keepdim=True)
    temp = st["temperature"][:, None]
    l = ((x - m).double() * _c0(1.0 / temp.double()).to(x.device)).add_(1065353216.0).float()
    l = torch.where(temp > 0, l, torch.full_like(l, 0.0)).masked_fill_(x == m, 1065353216.0)
    w = _pow2(l, st["case"]["mode"]).masked_fill_(x == -math.inf, 0.0)
    order = torch.sort(w, dim=1, descending=True, stable=True)
    mass = (order.values.double() * 2.0 ** 40).long()                # whole numbers: sums are exact
    rank = torch.arange(cols, device=x.device)
    keep = (mass > 0) & ((temp > 0) | (rank == 0))                   # greedy: the first of the largest
    if st["top_k"] is not None:
        keep &= rank < st["top_k"][:, None]
    if st["top_p"] is not None:
        live = mass.masked_fill(~keep, 0)
        before = live.cumsum(1) - live
        keep &= (before < _times(st["top_p"][:, None], live.sum(1, keepdim=True))) | (rank == 0)
    if st["min_p"] is not None:
        keep &= mass >= _times(st["min_p"][:, None], mass[:, :1])
    mass = torch.zeros_like(mass).scatter_(1, order.indices, mass.masked_fill(~keep, 0))
    upto = mass.cumsum(1)
    all_ = upto[:, -1:]
    token = (upto <= _times(st["u"][:, None], all_)).sum(1)          # the first one past u
    none = all_[:, 0] == 0
    token = token.clamp(max=cols - 1)
    prob = mass.gather(1, token[:, None])[:, 0].double() / all_[:, 0].clamp(min=1).double()
    return token.masked_fill(none, -1).int(), prob.float()


def _distill_plain(st):
    c = st["case"]
    x, idx, y = st["x"], st["idx"].long(), st["y"]
    t, mode, c0 = c["t"], c["mode"], float(_c0(c["t"]))
    live = idx >= 0
    y = y.masked_fill(~live, -math.inf)
    my = _row_exponent(y.amax(1, keepdim=True), t)
    p = _pow2((y.double() * c0 + (127.0 - my) * 8388608.0).float(), mode).masked_fill_(~live, 0.0).double()
    sy = p.sum(1, keepdim=True)
    p = p / sy.clamp(min=1e-300)
    loss = torch.empty(c["rows"], device="cuda")
    grad = torch.empty_like(x)
    step = max(1, (1 << 27) // c["cols"])
    for r in range(0, c["rows"], step):
        s = slice(r, r + step)
        xr = x[s].double()
        mx = _row_exponent(xr.amax(1, keepdim=True), t)
        e = _pow2((xr * c0 + (127.0 - mx) * 8388608.0).float(), mode)
        sx = e.sum(1, keepdim=True, dtype=torch.float64)
        at = idx[s].clamp(min=0)
        logp = y[s].double() * (t / LN2) - my[s] - torch.log2(sy[s])
        logq = xr.gather(1, at) * (t / LN2) - mx - torch.log2(sx)
        loss[s] = torch.where(p[s] > 0, p[s] * (logp - logq), 0.0).sum(1).mul(LN2).float()
        g = (e.double() / sx) * live[s].any(1, keepdim=True)
        g.scatter_add_(1, at, -p[s])
        grad[s] = (g * (st["weight"][s, None].double() * t)).to(x.dtype)
    return dict(loss=loss, grad=grad)


def run(st: dict):
    c = st["case"]
    if own:
        from paper_2412_00408_amd import quake as q
        if c["kind"] == "window":
            lens = dict(q_lens=st["q_lens"], kv_lens=st["kv_lens"]) if c["ragged"] else {}
            return q.quake_attention_window(st["q"], st["k"], st["v"], st["o"], window=c["window"],
                                            sinks=c["sinks"], mode=c["mode"],
                                            workspace=st["workspace"], **lens)
        if c["kind"] == "sample":
            return q.quake_sample(st["x"], st["u"], temperature=st["temperature"],
                                  top_k=st["top_k"], top_p=st["top_p"], min_p=st["min_p"],
                                  mode=c["mode"], workspace=st["workspace"])
        args = dict(t=c["t"], mode=c["mode"], workspace=st["workspace"])
        if c["fused"]:
            loss, _, grad = q.quake_distill(st["x"], st["idx"], st["y"], weight=st["weight"],
                                            grad=True, **args)
        else:
            loss, stats, _ = q.quake_distill(st["x"], st["idx"], st["y"], **args)
            grad = q.quake_distill_grad(st["x"], st["idx"], st["y"], stats, weight=st["weight"],
                                        t=c["t"], mode=c["mode"])
        return dict(loss=loss, grad=grad)
    return dict(window=_window_plain, sample=_sample_plain, distill=_distill_plain)[c["kind"]](st)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case: dict) -> dict:
    e = BYTES[case["dtype"]]
    if case["kind"] == "sample":                     # each logit once
        n = case["rows"] * case["cols"]
        return dict(bytes=e * n + 8 * case["rows"], flops=8 * n)
    if case["kind"] == "distill":                    # the logits once in, their gradient once out
        n = case["rows"] * case["cols"]
        return dict(bytes=2 * e * n + 8 * case["rows"] * (case["topk"] + 1), flops=12 * n)
    w, sinks = case["window"], case["sinks"]
    queries = keys = pairs = 0
    for ql, kl in zip(*_lengths(case)):
        queries += ql
        first = kl - ql                              # position of the first query
        low = max(0, first - w + 1)
        keys += kl - low + min(sinks, low)

        def below(n):                                # sum of min(x, cap) for x = 1 .. n
            cap = w + sinks
            return n * (n + 1) // 2 if n <= cap else cap * (cap + 1) // 2 + (n - cap) * cap
        pairs += below(kl) - below(first)
    d = case["dim"]
    return dict(bytes=2 * e * d * (queries * case["heads"] + keys * case["kv_heads"]),
                flops=4 * d * case["heads"] * pairs)


# ---------------------------------------------------------------- the same in 64 bits

def _real(v: torch.Tensor, mode: str) -> torch.Tensor:
    """2^v with the exponential of `mode`, v in float64 (base-2 exponent)."""
    if mode == "exact":
        return torch.exp2(v)
    dead = v == -math.inf
    v = v.clamp(-1000.0, 1000.0)
    i = torch.floor(v)
    a = 1.0 + (v - i)
    if mode == "quake2":
        a = (a * a + 2.0) / 3.0
    elif mode == "quake2m":
        a = torch.where(a == 1.0, a, (Q2M[0] * a + Q2M[1]) * a + Q2M[2])
    return torch.exp2(i).mul_(a).masked_fill_(dead, 0.0)


def _exact_window(a, case):
    t = 1.0 / math.sqrt(case["dim"])

    def weigh(s):
        y = s * (t / LN2)
        top = torch.ceil(y.amax(-1, keepdim=True))
        return _real(y - torch.where(top == -math.inf, 0.0, top), case["mode"])
    return _window_blocks(dict(case=case, **a), torch.float64, weigh)


def _exact_distill(a, case):
    t, mode = case["t"], case["mode"]
    loss = torch.empty(case["rows"], dtype=torch.float64, device="cuda")
    grad = torch.empty(a["x"].shape, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 26) // case["cols"])
    for r in range(0, case["rows"], step):
        s = slice(r, r + step)
        x, idx = a["x"][s].double() * (t / LN2), a["idx"][s].long()
        y = (a["y"][s].double() * (t / LN2)).masked_fill(idx < 0, -math.inf)
        x = x - torch.ceil(x.amax(1, keepdim=True))
        y = y - torch.ceil(y.amax(1, keepdim=True)).clamp(min=-1e9)
        q, p = _real(x, mode), _real(y, mode)
        sq, sp = q.sum(1, keepdim=True), p.sum(1, keepdim=True)
        p = torch.where(sp > 0, p / sp, 0.0)
        gap = (y - torch.log2(sp)) - (x - torch.log2(sq)).gather(1, idx.clamp(min=0))
        loss[s] = torch.where(p > 0, p * gap, 0.0).sum(1) * LN2
        g = torch.where(sp > 0, q / sq, 0.0)
        g.scatter_add_(1, idx.clamp(min=0), -p)
        grad[s] = g * (a["weight"][s, None].double() * t)
    return dict(loss=loss, grad=grad)


def _exact_sample(a, case):
    """The probability of the drawn word among the words kept; the word itself is
    a whole number, given by the plain form."""
    x = a["x"].double()
    m, temp = x.amax(1, keepdim=True), a["temperature"][:, None].double()
    w = _real(torch.where(x == m, 0.0, (x - m) / (temp.clamp(min=1e-30) * LN2)), case["mode"])
    w.masked_fill_(x == -math.inf, 0.0)
    rank = torch.arange(x.shape[1], device="cuda")
    p, at = torch.sort(w, dim=1, descending=True, stable=True)
    p.masked_fill_((temp <= 0) & (rank > 0), 0.0)
    if a["top_k"] is not None:
        p.masked_fill_(rank >= a["top_k"][:, None], 0.0)
    if a["top_p"] is not None:
        cut = p.cumsum(1) - p >= a["top_p"][:, None].double() * p.sum(1, keepdim=True)
        p.masked_fill_(cut, 0.0)
    if a["min_p"] is not None:
        p.masked_fill_(p < a["min_p"][:, None].double(), 0.0)
    p = torch.zeros_like(p).scatter_(1, at, p)
    upto = p.cumsum(1)
    word = (upto <= a["u"][:, None].double() * upto[:, -1:]).sum(1, keepdim=True)
    return None, (p.gather(1, word.clamp(max=x.shape[1] - 1)) / upto[:, -1:].clamp(min=1e-300))[:, 0]


def exact(case: dict, seed: int):
    a = _inputs(case, seed)
    if case["kind"] == "window":
        return _exact_window(a, case)
    if case["kind"] == "distill":
        return _exact_distill(a, case)
    return _exact_sample(a, case)
