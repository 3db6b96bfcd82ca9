"""Plain 64-bit references of attention over a shared prefix with the weight that keys
gather, and of eviction by it, with the error bounds that binary32 arithmetic allows."""
from __future__ import annotations

import math

import numpy as np
import torch

from ref64 import ARG, FEW, LN2, jump, real_exp2


def lengths(lens, n, most, dev):
    return [most] * n if lens is None else lens.clamp(0, most).tolist()


def shared_attention(q, k, v, pk=None, pv=None, mode=2, t=0.125, prefix_lens=None, q_lens=None,
                     kv_lens=None, weight=None):
    """(o, bound, written, weight, weight's bound) in float64; dense scores, so small sizes
    only. Keys behind the lengths may hold anything.

    The bound of o is that of ref64.window_attention, over the prefix's keys and the
    sequence's own. A weight is a sum of quotients p / S of positive numbers: with `off` the
    relative error of an exponential (the score's, the argument's rounding, three more), p and
    S are off by `off` each, QuAKE2M's by its jump each, S by (keys + 8) 2^-24 and the sum over
    the rows by (rows + 8) 2^-24; the reciprocal, the product and the addition to what was
    there round once each. An exponential below the least normal number, 2^-126 against 2^M,
    may be 0 instead: M is at most the row's largest argument rounded up, so S is at least
    1/2, and the row's part of a weight is then off by at most 2^-125."""
    dt, dev = q.dtype, q.device
    b, sq, h, d = q.shape
    skv, hk = k.shape[1:3]
    grp, groups = h // hk, 1 if pk is None else pk.shape[0]
    sp = 0 if pk is None else pk.shape[1]
    pl = lengths(prefix_lens, groups, sp, dev)
    ql, kl = lengths(q_lens, b, sq, dev), lengths(kv_lens, b, skv, dev)
    o = torch.zeros(q.shape, dtype=torch.float64, device=dev)
    bound = torch.zeros_like(o)
    written = torch.zeros((b, sq), dtype=torch.bool, device=dev)
    w = torch.zeros((b, hk, skv), dtype=torch.float64, device=dev) if weight is None else weight.double()
    wb = torch.zeros_like(w)
    eps = torch.finfo(dt).eps
    for i in range(b):
        g, n, m = i // (b // groups), ql[i], kl[i]
        written[i, :n] = True
        if n == 0:
            continue
        np_ = pl[g]
        pos = m - n + torch.arange(n, device=dev)
        seen = torch.arange(m, device=dev) <= pos[:, None]
        seen = torch.cat([torch.ones((n, np_), dtype=torch.bool, device=dev), seen], 1)
        cols = lambda x, px, c: torch.cat(([px[g, :np_, c]] if np_ else []) + [x[i, :m, c]]).double()  # noqa: E731
        for c in range(h):
            kk, vv = cols(k, pk, c // grp), cols(v, pv, c // grp)
            none = ~seen.any(0)
            kk, vv = kk.masked_fill(none[:, None], 0.0), vv.masked_fill(none[:, None], 0.0)
            qq = q[i, :n, c].double()
            kt = kk.t().contiguous()
            y = torch.matmul(qq, kt) * (t / LN2)
            y = y.masked_fill(~seen, -math.inf)
            keys = seen.sum(1, keepdim=True)
            if y.shape[1] == 0:
                bound[i, :n, c] = 2.0 ** -126
                continue
            off = torch.matmul(qq.abs(), kt.abs()).masked_fill(~seen, 0.0).amax(1, keepdim=True)
            off = off * (t / LN2 * (d + 1) * 2.0 ** -24) + ARG + FEW
            top = torch.ceil(y.amax(1, keepdim=True))
            p = real_exp2(y - torch.where(top == -math.inf, 0.0, top), mode)
            s = p.sum(1, keepdim=True)
            inv = torch.where(s > 0, 1.0 / s, 0.0)
            r = torch.matmul(p, vv) * inv
            mean = torch.matmul(p, vv.abs()) * inv
            rel = 2 * off + 2 * jump(mode) + eps / 2 + 2 * (keys + 8) * 2.0 ** -24
            o[i, :n, c] = r
            e = 1.01 * (mean * rel + 2 * r.abs() * eps / 2)
            if dt == torch.float16:
                e = e + torch.matmul(seen.double(), vv.abs()) * 2.0 ** -25 * 2 * inv.clamp(max=2.0) + 2.0 ** -25
            bound[i, :n, c] = e + 2.0 ** -126
            share = p * inv
            w[i, c // grp, :m] += share[:, np_:].sum(0)
            few = 2 * off + 2 * jump(mode) + (keys + n * grp + 24) * 2.0 ** -24
            wb[i, c // grp, :m] += 1.01 * (share * few)[:, np_:].sum(0) + n * 2.0 ** -125
    return o, bound, written, w, wb + (w.abs() + wb) * 2.0 ** -23 + 2.0 ** -126


def evict_row(weight, n, budget, sinks, recent):
    """The kept slots of a row of float32 weights with n keys, by whole numbers."""
    if n <= budget:
        return list(range(n))
    w = np.asarray(weight[:n], np.float32)
    bits = np.where(w == 0, np.float32(0.0), w).view(np.int32).astype(np.int64)
    order = np.where(np.isnan(w), -(1 << 40), np.where(bits < 0, -(bits & 0x7FFFFFFF), bits))
    mid = sorted(range(sinks, n - recent), key=lambda j: (-order[j], j))[:budget - sinks - recent]
    return sorted(list(range(sinks)) + mid + list(range(n - recent, n)))


def evict(k, v, weight, budget, sinks, recent, lens, k_out, v_out, weight_out):
    """(k_out, v_out, weight_out, lens, kept, evicted) as a call leaves them, on the CPU."""
    k, v, weight = k.cpu(), v.cpu(), weight.cpu()
    ko, vo, wo = k_out.cpu().clone(), v_out.cpu().clone(), weight_out.cpu().clone()
    b, skv, hk = k.shape[:3]
    ln = [skv] * b if lens is None else lens.clamp(0, skv).tolist()
    kept = torch.full((b, hk, budget), -1, dtype=torch.int32)
    for i in range(b):
        for h in range(hk):
            at = torch.tensor(evict_row(weight[i, h].numpy(), ln[i], budget, sinks, recent), dtype=torch.long)
            n = at.numel()
            kept[i, h, :n] = at.int()
            ko[i, :n, h] = k[i, at, h]
            vo[i, :n, h] = v[i, at, h]
            x = weight[i, h, at]
            wo[i, h] = 0.0
            wo[i, h, :n] = x
    new = torch.tensor([min(n, budget) for n in ln], dtype=torch.int32)
    return ko, vo, wo, new, kept, torch.tensor([max(n - budget, 0) for n in ln], dtype=torch.int32)
