"""Workloads of libquake's cache operators as a user's program calls them: attention
for a batch that shares a long prefix, the attention weight that the keys of a cache
gather, and eviction of the keys that gathered least.

A case is a dict of plain values with a "kind":

  attend  batch, groups (of sequences that share a prefix), sq, sp (tokens of a prefix, 0:
          none), skv (slots of a sequence's own cache), heads, kv_heads, dim, dtype, mode,
          ragged (lengths of their own in padded buffers), weigh (the keys' weight is gathered)
  evict   batch, skv, kv_heads, dim, budget, sinks, recent, dtype, ragged (some sequences
          within the budget)

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


def _attend(name, batch, groups, sq, sp, skv, heads, kv_heads, dim, dtype, mode, ragged, weigh):
    return dict(name=name, kind="attend", batch=batch, groups=groups, sq=sq, sp=sp, skv=skv, heads=heads,
                kv_heads=kv_heads, dim=dim, dtype=dtype, mode=mode, ragged=ragged, weigh=weigh)


def _evict(name, batch, skv, kv_heads, dim, budget, sinks, recent, dtype, ragged):
    return dict(name=name, kind="evict", batch=batch, skv=skv, kv_heads=kv_heads, dim=dim, budget=budget,
                sinks=sinks, recent=recent, dtype=dtype, ragged=ragged)


def listed() -> list[dict]:
    return [
        # the smallest call: four answers to one short prompt, launch latency
        _attend("shared_bf16_4x500", 4, 1, 1, 500, 64, 8, 2, 64, "bf16", "quake2", False, False),
        # one decode step of 64 conversations under one system prompt
        _attend("shared_bf16_64x8192", 64, 1, 1, 8192, 1024, 32, 8, 128, "bf16", "quake2", True, False),
        # 256 samples of one long document, the largest product of single tokens
        _attend("shared_bf16_256x32768", 256, 1, 1, 32768, 512, 32, 8, 128, "bf16", "quake2", True, False),
        # eight prompts with eight answers each, prompts of odd lengths, a head per key head
        _attend("shared_f16_8x8x3001", 64, 8, 1, 3001, 300, 16, 16, 64, "f16", "exact", True, False),
        # drafted tokens checked against a shared prompt
        _attend("shared_f16_16x5x10007", 16, 1, 5, 10007, 700, 40, 8, 128, "f16", "quake1", True, False),
        # the users' own prompts behind one system prompt
        _attend("shared_prompts_bf16_8x600", 8, 1, 600, 4096, 600, 32, 8, 128, "bf16", "quake2", True, False),
        # one decode step over bounded caches, with the weight that eviction goes by
        _attend("weigh_bf16_32x4096", 32, 1, 1, 0, 4096, 32, 8, 128, "bf16", "quake2", True, True),
        # a prompt whose keys gather their first weight
        _attend("weigh_prompt_bf16_4096", 1, 1, 4096, 0, 4096, 32, 8, 128, "bf16", "quake2", False, True),
        # both: a shared prefix that stays, and the sequences' own keys weighed
        _attend("weigh_shared_f16_24x6000", 24, 1, 1, 6000, 1500, 16, 4, 64, "f16", "quake2m", True, True),
        # a prompt's cache cut to the size that decoding goes on with
        _evict("evict_bf16_1x16384", 1, 16384, 8, 128, 2048, 4, 256, "bf16", False),
        # a batch whose caches are full, the most bytes
        _evict("evict_bf16_64x2560", 64, 2560, 8, 128, 2048, 4, 128, "bf16", True),
        # a small cache
        _evict("evict_f16_2x300", 2, 300, 2, 64, 100, 1, 16, "f16", False),
    ]


def _log(rng, lo: int, hi: int) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case: dict) -> float:
    w = work(case)
    return w["bytes"] / 8e12 + w["flops"] / 2.5e15


def draw(rng) -> dict:
    kind = rng.choice(["attend", "attend", "attend", "evict"])
    most = max(_cost(c) for c in listed() if c["kind"] == kind)
    while True:
        kv = rng.choice([1, 2, 4, 8, 16])
        if kind == "evict":
            skv = _log(rng, 16, 40000)
            budget = max(2, int(skv * rng.uniform(0.05, 0.95)))
            sinks = rng.choice([0, 1, 4, 33])
            case = dict(kind=kind, batch=_log(rng, 1, 128), skv=skv, kv_heads=kv, dim=rng.choice([64, 80, 128, 256]),
                        budget=budget, sinks=min(sinks, budget // 2), recent=int(budget * rng.choice([0.0, 0.1, 0.5])),
                        dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), ragged=rng.random() < 0.5)
        else:
            groups = rng.choice([1, 1, 1, 2, 5])
            step = rng.choice(["one", "one", "few", "all"])
            weigh = rng.random() < 0.4
            sp = 0 if weigh and rng.random() < 0.5 else _log(rng, 16, 32768)
            skv = _log(rng, 4, 1500 if step == "all" else 6000)
            sq = 1 if step == "one" else min(skv, _log(rng, 2, 32)) if step == "few" else skv
            case = dict(kind=kind, batch=groups * _log(rng, 1, 200 // groups), groups=groups, sq=sq, sp=sp, skv=skv,
                        heads=kv * rng.choice([1, 2, 4, 5, 8]), kv_heads=kv, dim=rng.choice([64, 128]),
                        dtype=rng.choice(["bf16", "f16"]), mode=rng.choice(["quake2", "quake2", "quake1", "quake2m", "exact"]),
                        ragged=rng.random() < 0.6, weigh=weigh)
            if case["batch"] * sq * case["heads"] * (sp + skv) > 1 << 29:
                continue
        if _cost(case) <= most:
            return case


# ---------------------------------------------------------------- inputs

def _lengths(c: dict) -> tuple[list[int], list[int], list[int]]:
    """Query, key and prefix lengths of a case's sequences and groups (its own, whatever
    the seed): batches padded to the longest, or all as long as the buffers."""
    b, g = c["batch"], c.get("groups", 1)
    sq, sp, skv = c.get("sq", 1), c.get("sp", 0), c["skv"]
    if not c["ragged"]:
        return [sq] * b, [skv] * b, [sp] * g
    r = random.Random(b * 1000003 + skv)
    low = 0.6 if c["kind"] == "evict" else 0.1
    kv = [skv] + [max(1, int(skv * r.uniform(low, 1.0))) for _ in range(b - 1)]
    pre = [sp] + [int(sp * r.uniform(0.5, 1.0)) for _ in range(g - 1)]
    if sq == skv:                                    # whole prompts: every key has its query
        return list(kv), kv, pre
    return [min(n, sq if i == 0 else r.randint(1, sq)) for i, n in enumerate(kv)], kv, pre


def _normal(shape, std, dtype, g):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(std).to(dtype)


def _int32(v, order=None):
    t = torch.tensor(v, dtype=torch.int32, device="cuda")
    return t if order is None else t[order]


def _inputs(c: dict, seed: int) -> dict:
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt, b, hk, d, skv = DTYPES[c["dtype"]], c["batch"], c["kv_heads"], c["dim"], c["skv"]
    ql, kl, pl = _lengths(c)
    order = torch.randperm(b, generator=g, device="cuda")
    st = dict(k=_normal((b, skv, hk, d), 1.0, dt, g), v=_normal((b, skv, hk, d), 1.0, dt, g),
              kv_lens=_int32(kl, order))
    slots = torch.arange(skv, device="cuda")
    if c["kind"] == "evict":
        # a few keys gathered most of the weight; the newest ones none yet, which are equal
        w = torch.randn((b, hk, skv), generator=g, device="cuda").mul_(2.0).exp_().mul_(16.0 / skv)
        st["weight"] = w.masked_fill_(slots >= st["kv_lens"][:, None, None] - 2, 0.0)
        size = c["budget"] + 64                      # the cache that goes on, with room for new tokens
        st["out"] = [torch.zeros((b, size, hk, d), dtype=dt, device="cuda") for _ in range(2)]
        st["out"] += [torch.zeros((b, hk, size), device="cuda"), torch.zeros(b, dtype=torch.int32, device="cuda")]
        return st
    st["q"] = _normal((b, c["sq"], c["heads"], d), 1.0, dt, g)
    st["o"] = torch.zeros_like(st["q"])
    st["q_lens"] = _int32(ql, order)
    st["prefix_lens"] = _int32(pl)
    st["pk"] = st["pv"] = st["weight"] = None
    if c["sp"]:
        st["pk"] = _normal((c["groups"], c["sp"], hk, d), 1.0, dt, g)
        st["pv"] = _normal((c["groups"], c["sp"], hk, d), 1.0, dt, g)
        st["pk"][:, :4] *= 1.5                       # first tokens draw attention
    if c["weigh"]:                                   # as it stands after some steps
        st["weight"] = torch.rand((b, hk, skv), generator=g, device="cuda").mul_(8.0 / skv)
    return st


def prepare(case: dict, seed: int) -> dict:
    st = dict(case=case, **_inputs(case, seed))
    if own and case["kind"] == "attend":
        from paper_2412_00408_amd import quake as q
        st["workspace"] = q.attention_shared_workspace(st["q"], st["k"], st["pk"], weigh=case["weigh"])
    return st


# ---------------------------------------------------------------- plain forms

def _pow2(l: torch.Tensor, mode: str) -> torch.Tensor:
    """The exponential of `mode` from its binary32 argument l = (y + 127) 2^23
    (base-2 exponent y): Eq. 3's integer, then Eq. 2 or Algorithm 1 on its bits."""
    if mode == "exact":
        return torch.exp2(l.double().div_(8388608.0).sub_(127.0)).float()
    z = l.clamp_(0.0, 2139095040.0).to(torch.int32)
    if mode == "quake1":
        return z.view(torch.float32)
    a = ((z & 0x7FFFFF) | 0x3F800000).view(torch.float32)
    if mode == "quake2":
        y = (a.double().square().add_(2.0)).float() * (1.0 / 3.0)
    else:
        y = ((a.double() * Q2M[0] + Q2M[1]).float().double() * a.double() + Q2M[2]).float()
        y = torch.where(a == 1.0, a, y)
    return ((z & -8388608) | (y.view(torch.int32) & 0x7FFFFF)).view(torch.float32)


def _attend_plain(st):
    """Rows [key head, query and head of the group] of every sequence; the prefix's scores are
    one product for all sequences of a group."""
    c = st["case"]
    b, sq, hk, d, skv, ng = c["batch"], c["sq"], c["kv_heads"], c["dim"], c["skv"], c["groups"]
    grp, n = c["heads"] // hk, b // ng
    t, mode = 1.0 / math.sqrt(d), c["mode"]
    late = torch.arange(sq, device="cuda") >= st["q_lens"][:, None]                       # [b, sq]
    q = st["q"].float().view(b, sq, hk, grp, d).permute(0, 2, 1, 3, 4).reshape(b, hk, sq * grp, d)
    k = st["k"].float().permute(0, 2, 3, 1).contiguous()
    v = st["v"].float().permute(0, 2, 1, 3).contiguous()
    pos = (st["kv_lens"] - st["q_lens"])[:, None] + torch.arange(sq, device="cuda")
    seen = (torch.arange(skv, device="cuda") <= pos[..., None]) & ~late[..., None]        # [b, sq, skv]
    s = torch.matmul(q, k).view(b, hk, sq, grp, skv)
    s.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    s = s.view(b, hk, sq * grp, skv)
    top = s.amax(-1, keepdim=True)
    if st["pk"] is not None:
        pk = st["pk"].float().permute(0, 2, 3, 1).contiguous()                            # [ng, hk, d, sp]
        pv = st["pv"].float().permute(0, 2, 1, 3).contiguous()
        rows = q.view(ng, n, hk, sq * grp, d).transpose(1, 2).reshape(ng, hk, n * sq * grp, d)
        far = torch.arange(c["sp"], device="cuda") >= st["prefix_lens"][:, None]
        ps = torch.matmul(rows, pk).masked_fill_(far[:, None, None, :], -math.inf)

        def back(x):                                 # rows of a group to rows of its sequences
            return x.view(ng, hk, n, sq * grp, -1).transpose(1, 2).reshape(b, hk, sq * grp, -1)
        top = torch.maximum(top, back(ps.amax(-1, keepdim=True)))
    m = torch.ceil(top * (t / LN2))
    m = torch.where(torch.isfinite(m), m, torch.zeros_like(m))
    c0 = float(torch.tensor(t / LN2 * 8388608.0, dtype=torch.float64).float())
    c1 = (127.0 - m) * 8388608.0
    p = _pow2(s.mul_(c0).add_(c1), mode).masked_fill_(~seen[:, None, :, None, :].expand(b, hk, sq, grp, skv)
                                                      .reshape(b, hk, sq * grp, skv), 0.0)
    total = p.sum(-1, keepdim=True, dtype=torch.float64)
    o = torch.matmul(p, v)
    if st["pk"] is not None:
        pc1 = c1.view(ng, n, hk, sq * grp, 1).transpose(1, 2).reshape(ng, hk, n * sq * grp, 1)
        pp = _pow2(ps.mul_(c0).add_(pc1), mode).masked_fill_(far[:, None, None, :], 0.0)
        total = total + back(pp.sum(-1, keepdim=True, dtype=torch.float64))
        o = o + back(torch.matmul(pp, pv))
    inv = torch.where(total > 0, 1.0 / total, 0.0).float()
    o = (o * inv).view(b, hk, sq, grp, d).permute(0, 2, 1, 3, 4).reshape(b, sq, hk * grp, d)
    st["o"].copy_(torch.where(late[:, :, None, None], st["o"].float(), o))
    if st["weight"] is None:
        return st["o"]
    st["weight"].add_((p * inv).sum(2, dtype=torch.float64).float())
    return dict(o=st["o"], weight=st["weight"])


def _evict_plain(st):
    c = st["case"]
    b, hk, skv, budget = c["batch"], c["kv_heads"], c["skv"], c["budget"]
    lens = st["kv_lens"].long()[:, None, None]
    slot = torch.arange(skv, device="cuda")
    w = st["weight"].masked_fill((slot < c["sinks"]) | (slot >= lens - c["recent"]), math.inf)
    w = w.masked_fill(slot >= lens, -math.inf)
    best = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :budget]     # equal ones: the first
    place = torch.arange(budget, device="cuda")
    stay = lens <= budget
    best = torch.where(stay, place, torch.sort(best, dim=-1).values)
    live = place < lens
    new = lens.clamp(max=budget)
    ko, vo, wo, lo = st["out"]
    at = best.clamp(max=skv - 1).transpose(1, 2)[..., None].expand(-1, -1, -1, c["dim"])  # [b, budget, hk, dim]
    there = live.expand(b, hk, budget).transpose(1, 2)[..., None]
    for x, y in ((st["k"], ko), (st["v"], vo)):
        y[:, :budget] = torch.where(there, x.gather(1, at), y[:, :budget])
    wo.zero_()
    wo[..., :budget] = torch.where(live, st["weight"].gather(2, best.clamp(max=skv - 1)), 0.0)
    lo.copy_(new[:, 0, 0])
    kept = torch.where(live, best, -1).expand(b, hk, budget).int()
    return dict(k=ko, v=vo, weight=wo, lens=lo, kept=kept, evicted=(lens - new)[:, 0, 0].int())


def run(st: dict):
    c = st["case"]
    if own:
        from paper_2412_00408_amd import quake as q
        if c["kind"] == "evict":
            kept, evicted = q.quake_cache_evict(st["k"], st["v"], st["weight"], c["budget"], sinks=c["sinks"],
                                                recent=c["recent"], kv_lens=st["kv_lens"], out=st["out"])
            k, v, weight, lens = st["out"]
            return dict(k=k, v=v, weight=weight, lens=lens, kept=kept, evicted=evicted)
        lens = dict(q_lens=st["q_lens"], kv_lens=st["kv_lens"]) if c["ragged"] else {}
        if c["ragged"] and st["pk"] is not None:
            lens["prefix_lens"] = st["prefix_lens"]
        o = q.quake_attention_shared(st["q"], st["k"], st["v"], st["pk"], st["pv"], st["o"], weight=st["weight"],
                                     mode=c["mode"], workspace=st["workspace"], **lens)
        return o if st["weight"] is None else dict(o=o, weight=st["weight"])
    return _evict_plain(st) if c["kind"] == "evict" else _attend_plain(st)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case: dict) -> dict:
    e, d, hk = BYTES[case["dtype"]], case["dim"], case["kv_heads"]
    ql, kl, pl = _lengths(case)
    if case["kind"] == "evict":                      # the weights, the kept rows in and out
        kept = sum(min(n, case["budget"]) for n in kl)
        return dict(bytes=hk * (4 * sum(kl) + kept * (4 * d * e + 8)), flops=hk * sum(kl))
    # a sequence's lengths go to any group: the mean prefix
    pairs = sum(a * sum(pl) / len(pl) + a * (2 * b - a + 1) / 2 for a, b in zip(ql, kl))
    keys = sum(kl) + sum(pl)
    io = 2 * e * d * (sum(ql) * case["heads"] + keys * hk) + (8 * hk * sum(kl) if case["weigh"] else 0)
    return dict(bytes=io, flops=int(4 * d * case["heads"] * pairs))


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


def _exact_attend(a, c):
    """Sequence by sequence and key head by key head, over the keys it has."""
    hk, d, grp = c["kv_heads"], c["dim"], c["heads"] // c["kv_heads"]
    scale = 1.0 / math.sqrt(d) / LN2
    ql, kl, pl = a["q_lens"].tolist(), a["kv_lens"].tolist(), a["prefix_lens"].tolist()
    o = torch.zeros(a["q"].shape, dtype=torch.float64, device="cuda")
    weight = a["weight"].double() if c["weigh"] else None
    per = c["batch"] // c["groups"]
    for b in range(c["batch"]):
        g, nq, nk = b // per, ql[b], kl[b]
        np_ = pl[g] if c["sp"] else 0
        if b % per == 0 and c["sp"]:
            pk, pv = (a[x][g, :np_].double().transpose(0, 1).contiguous() for x in ("pk", "pv"))
        k = a["k"][b, :nk].double().transpose(0, 1).contiguous()
        v = a["v"][b, :nk].double().transpose(0, 1).contiguous()
        q = a["q"][b, :nq].double().view(nq, hk, grp, d).transpose(0, 1).reshape(hk, nq * grp, d)
        y = torch.matmul(q, k.transpose(1, 2)).view(hk, nq, grp, nk) * scale
        hidden = torch.arange(nk, device="cuda")[None, :] > (nk - nq + torch.arange(nq, device="cuda"))[:, None]
        y = y.masked_fill(hidden[None, :, None, :], -math.inf).view(hk, nq * grp, nk)
        if np_:
            y = torch.cat([torch.matmul(q, pk.transpose(1, 2)) * scale, y], 2)
        p = _real(y - torch.ceil(y.amax(2, keepdim=True)), c["mode"])
        p = p / p.sum(2, keepdim=True)
        r = torch.matmul(p[:, :, np_:], v)
        if np_:
            r = r + torch.matmul(p[:, :, :np_], pv)
        o[b, :nq] = r.view(hk, nq, grp, d).transpose(0, 1).reshape(nq, hk * grp, d)
        if weight is not None:
            weight[b, :, :nk] += p[:, :, np_:].sum(1)
    return o if weight is None else dict(o=o, weight=weight)


def _exact_evict(a, c):
    """A slot stays if fewer than the budget's share are ahead of it."""
    budget, sinks, recent = c["budget"], c["sinks"], c["recent"]
    out = [x.double() for x in a["out"][:3]]
    for b, n in enumerate(a["kv_lens"].tolist()):
        for h in range(c["kv_heads"]):
            keep = torch.ones(n, dtype=torch.bool, device="cuda")
            if n > budget:
                w = a["weight"][b, h, sinks:n - recent].double()
                keep[sinks:n - recent] = False
                rank = torch.argsort(-w, stable=True)[:budget - sinks - recent]
                keep[sinks + rank] = True
            at = keep.nonzero()[:, 0]
            for x, y in zip((a["k"], a["v"]), out):
                y[b, :at.numel(), h] = x[b, at, h].double()
            out[2][b, h, :at.numel()] = a["weight"][b, h, at].double()
    return dict(k=out[0], v=out[1], weight=out[2], lens=None, kept=None, evicted=None)


def exact(case: dict, seed: int):
    a = _inputs(case, seed)
    return _exact_evict(a, case) if case["kind"] == "evict" else _exact_attend(a, case)
