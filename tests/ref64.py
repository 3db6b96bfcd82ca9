"""Plain 64-bit references of the windowed attention, the sampler and the
distillation loss, with QuAKE's exponential as the real function of Eq. 2 and
Eq. 6, and the error bounds that the binary32 arithmetic of each operator allows."""
from __future__ import annotations

import math

import numpy as np
import torch

LN2 = math.log(2.0)
NAMES = {0: "exact", 1: "quake1", 2: "quake2", 3: "quake2m"}
Q2M = tuple(map(float.fromhex, ("0x1.594830p-2", "-0x1.124f86p-6", "0x1.5cd076p-1")))

# Relative error of an exponential whose argument l = (y + 127) 2^23 is off by one
# rounding: l < 136 * 2^23 < 2^31 rounds by at most 64 units of 2^23, l's
# truncation loses one more: 65 * 2^-23 < 2^-16.9 base-2 units; the exponentials
# change by at most ln2 (exact), 1 (first order), 0.71 (refined) of a change of y.
# The refined result has three binary32 roundings more. QuAKE2M jumps at whole y by
# at most 0.18 % + 0.18 %.
ARG = 65 * 2.0 ** -23
FEW = 2.0 ** -21


def jump(mode: int) -> float:
    return 3.6e-3 if mode == 3 else 0.0


def real_exp2(v: torch.Tensor, mode: int) -> torch.Tensor:
    """2^v with the exponential of `mode`, v in float64."""
    if mode == 0:
        return torch.exp2(v)
    dead = v == -math.inf
    v = v.clamp(-1000.0, 1000.0)
    i = torch.floor(v)
    a = 1.0 + (v - i)
    if mode == 2:
        a = (a * a + 2.0) / 3.0
    elif mode == 3:
        a = torch.where(a == 1.0, a, (Q2M[0] * a + Q2M[1]) * a + Q2M[2])
    return (torch.exp2(i) * a).masked_fill(dead, 0.0)


def window_attention(q, k, v, window, sinks, mode, t, q_lens=None, kv_lens=None):
    """(o, bound, written): the outputs in float64, how far a right kernel's may be,
    and which rows a call writes. Any device; dense scores, so small sizes only.

    The bound: a score is off by (dim + 1) 2^-24 sum |q_d k_d|, times t/ln2 in base-2
    units, an exponential then by that plus ARG relative (both sides of the
    quotient: twice), its 16-bit rounding by half a step (binary16: at least 2^-25
    against a sum of at least 1/2), the products and sums by (keys + 8) 2^-24 each,
    the result by half a step of its format. The sum is of the rounded p too: with
    p' = p (1 + e), sum p' v / sum p' - o = sum p' e' (v - o) / sum p', so the rounding
    costs half a step of mean |v| + |o|, not of mean |v| alone."""
    dt = q.dtype
    b, sq, h, d = q.shape
    skv, hk = k.shape[1], k.shape[2]
    dev = q.device
    ql = torch.full((b,), sq, device=dev) if q_lens is None else q_lens.clamp(0, sq).long()
    kl = torch.full((b,), skv, device=dev) if kv_lens is None else kv_lens.clamp(0, skv).long()
    i = torch.arange(sq, device=dev)
    j = torch.arange(skv, device=dev)
    pos = (kl - ql)[:, None] + i                                          # [b, sq]
    seen = (j <= pos[..., None]) & ((j > pos[..., None] - window) | (j < sinks))
    seen &= (j < kl[:, None])[:, None, :]
    o = torch.zeros(q.shape, dtype=torch.float64, device=dev)
    bound = torch.zeros_like(o)
    eps = torch.finfo(dt).eps
    for n in range(h):
        kk = k[:, :, n // (h // hk)].double().transpose(1, 2).contiguous()
        vv = v[:, :, n // (h // hk)].double().contiguous()
        # keys that no query of the sequence sees may hold anything
        none = ~seen.any(1)
        kk = kk.masked_fill(none[:, None, :], 0.0)
        vv = vv.masked_fill(none[:, :, None], 0.0)
        qq = q[:, :, n].double().contiguous()
        y = torch.matmul(qq, kk) * (t / LN2)
        y = y.masked_fill(~seen, -math.inf)
        off = torch.matmul(qq.abs(), kk.abs()).masked_fill(~seen, 0.0).amax(-1, keepdim=True)
        off = off * (t / LN2 * (d + 1) * 2.0 ** -24) + ARG + FEW
        top = torch.ceil(y.amax(-1, keepdim=True))
        p = real_exp2(y - torch.where(top == -math.inf, 0.0, top), mode)
        s = p.sum(-1, keepdim=True)
        keys = seen.sum(-1, keepdim=True)
        inv = torch.where(s > 0, 1.0 / s, 0.0)
        o[:, :, n] = torch.matmul(p, vv) * inv
        mean = torch.matmul(p, vv.abs()) * inv
        rel = 2 * off + 2 * jump(mode) + eps / 2 + 2 * (keys + 8) * 2.0 ** -24
        bound[:, :, n] = 1.01 * (mean * rel + 2 * o[:, :, n].abs() * eps / 2)
        if dt == torch.float16:
            bound[:, :, n] += torch.matmul(seen.double(), vv.abs()) * (2.0 ** -25) * 2 * inv.clamp(max=2.0)
            bound[:, :, n] += 2.0 ** -25
        else:
            bound[:, :, n] += 2.0 ** -126
    return o, bound, (i < ql[:, None])


# ---------------------------------------------------------------- sampling

def weights(x: np.ndarray, temperature: float, mode: int) -> np.ndarray:
    """The weights' binary32 bits (uint32) of one row (float32, NaN as -inf)."""
    x = np.where(np.isnan(x), np.float32(-np.inf), x).astype(np.float32)
    m = x.max()
    if m == -np.inf:
        return np.zeros(x.shape, np.uint32)
    one = np.uint32(0x3F800000)
    if not temperature > 0:
        return np.where(x == m, one, np.uint32(0))
    with np.errstate(all="ignore"):
        c0 = np.float32(1.0 / float(np.float32(temperature)) / LN2 * (8388608.0 if mode else 1.0))
        d = (x - m).astype(np.float32)
        # one rounding: the product is exact in binary64
        l = (d.astype(np.float64) * np.float64(c0) + (1065353216.0 if mode else 0.0)).astype(np.float32)
        if mode == 0:
            w = np.exp2(l.astype(np.float64)).astype(np.float32).view(np.uint32)
        else:
            z = np.nan_to_num(np.clip(l, 0.0, 2139095040.0)).astype(np.int64).astype(np.uint32)
            a = ((z & np.uint32(0x7FFFFF)) | one).view(np.float32).astype(np.float64)
            if mode == 1:
                w = z
            else:
                if mode == 2:
                    y = (a * a + 2.0).astype(np.float32) * np.float32(1.0 / 3.0)
                else:
                    y = ((a * Q2M[0] + Q2M[1]).astype(np.float32).astype(np.float64) * a
                         + Q2M[2]).astype(np.float32)
                    y = np.where(a == 1.0, np.float32(1.0), y)
                w = (z & np.uint32(0xFF800000)) | (y.astype(np.float32).view(np.uint32) & np.uint32(0x7FFFFF))
    w = np.where(x == m, one, w)
    return np.where(x == -np.inf, np.uint32(0), w).astype(np.uint32)


def fraction(v: float) -> int:
    v = np.float32(v)
    return 0 if not v > 0 else int(min(float(v), 1.0) * 16777216.0)


def sample_row(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, mode=2):
    """(token, prob, upto): the definition of quake_sample in whole numbers; upto:
    running kept mass over the vocabulary, as Python-exact int64."""
    w = weights(x, temperature, mode)
    mass = np.array([int(v) for v in np.floor(w.view(np.float32).astype(np.float64) * 2.0 ** 40)], dtype=np.int64)
    n = len(w)
    order = np.lexsort((np.arange(n), -w.astype(np.int64)))
    keep = np.ones(n, bool)
    greedy = not temperature > 0
    k = 1 if greedy else top_k if 0 < top_k < n else n
    keep[order[k:]] = False
    if top_p < 1.0:
        ranked = np.where(keep, mass, 0)[order]
        before = np.cumsum(ranked) - ranked
        goal = max(fraction(top_p) * int(ranked.sum()) >> 24, 1)
        keep[order[before >= goal]] = False
    keep &= mass >= max((fraction(min_p) << 40) >> 24, 1)
    kept = np.where(keep, mass, 0)
    upto = np.cumsum(kept)
    if upto[-1] == 0:
        return -1, 0.0, upto
    f = min(fraction(u), (1 << 24) - 1)
    token = int(np.argmax(upto > (f * int(upto[-1]) >> 24)))
    return token, float(np.float32(float(kept[token]) / float(upto[-1]))), upto


# ---------------------------------------------------------------- distillation

def distill(x, idx, y, mode, t, weight=None):
    """(loss, grad, loss_bound, grad_bound) in float64. grad: weight t (q - P).

    Bounds: every exponential is off by e = ARG + FEW + the mode's jump, sums by
    e, too (and 2^-24 where kept in binary32), so q and p by 2 e and 2^-22; the loss
    by 2 e for both logarithms, 3 e of the entries' gaps, and its own rounding; the
    gradient's result by half a step of its format."""
    cols = x.shape[1]
    live = (idx >= 0) & (idx < cols)
    at = torch.where(live, idx, 0).long()
    xs = x.double() * (t / LN2)
    ys = (y.double() * (t / LN2)).masked_fill(~live, -math.inf)

    def shift(v):
        top = torch.ceil(v.amax(1, keepdim=True)) if v.shape[1] else v.new_full((v.shape[0], 1), -math.inf)
        return v - torch.where(torch.isfinite(top), top, 0.0)
    xs, ys = shift(xs), shift(ys)
    q, p = real_exp2(xs, mode), real_exp2(ys, mode)
    sq, sp = q.sum(1, keepdim=True), p.sum(1, keepdim=True)
    p = torch.where(sp > 0, p / sp, 0.0)
    q = torch.where(sq > 0, q / sq, 0.0)
    gap = (ys - torch.log2(sp)) - (xs - torch.log2(sq)).gather(1, at)
    terms = torch.where(p > 0, p * gap, 0.0)
    loss = terms.sum(1) * LN2
    e = ARG + FEW + jump(mode)
    # c0's own rounding moves every base-2 argument by 2^-24 of it
    arg = (x.double().masked_fill(x == -math.inf, 0).abs().amax(1) +
           (y.double().masked_fill(~live | (y == -math.inf), 0).abs().amax(1) if y.shape[1] else 0)) * (t / LN2)
    c = arg * 2.0 ** -23
    lb = 2 * e + c + (3 * e + c) * terms.abs().sum(1) + 2.0 ** -23 * loss.abs() + 1e-7
    w = torch.ones_like(loss) if weight is None else weight.double()
    big = torch.zeros_like(q).scatter_add_(1, at, p)
    has = (sp > 0).double()
    grad = (q * has - big) * (w * t)[:, None]
    eps = torch.finfo(x.dtype).eps
    tiny = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -126, torch.float32: 2.0 ** -126}[x.dtype]
    gb = (q + big) * (2 * e + c[:, None] + 2.0 ** -21) * (w * t).abs()[:, None] + grad.abs() * eps / 2 + tiny
    return loss, grad, lb, 1.01 * gb
