"""What the binding of the cache operators refuses of device tensors before any launch, by
its own messages (ValueError, TypeError) and by the library's answer (QuakeError)."""
import pytest
import torch

from test_gpu_evict import q  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu


def zeros(*shape, dt=torch.bfloat16):
    return torch.zeros(shape, dtype=dt, device="cuda")


def lens(n, dt=torch.int32):
    return torch.ones(n, dtype=dt, device="cuda")


def ints(t, n):
    """n int32 in the first bytes of t"""
    return t.view(-1).view(torch.int32)[:n]


def floats(t, *shape):
    """float32 in the first bytes of t"""
    return t.view(-1).view(torch.float32)[:torch.Size(shape).numel()].view(shape)


def shared_cases():
    x, k, v = zeros(4, 3, 4, 64), zeros(4, 10, 2, 64), zeros(4, 10, 2, 64)
    pk, pv, w = zeros(2, 6, 2, 64), zeros(2, 6, 2, 64), zeros(4, 2, 10, dt=torch.float32)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    ok = dict(q=x, k=k, v=v, prefix_k=pk, prefix_v=pv, weight=w, workspace=ws)
    o = torch.empty_like(x)
    long = zeros(4, 20, 8, 64)                   # whose bytes other operands are laid into
    val, typ = ValueError, TypeError
    return ok, [
        (dict(q=x[0]), val, "q needs"), (dict(k=k[0]), val, "k needs"), (dict(v=v[0]), val, "v needs"),
        (dict(q=x.cpu()), val, "device tensors, q"), (dict(v=v.cpu()), val, "device tensors, v"),
        (dict(q=x.double()), typ, "q must be"), (dict(k=k.half()), typ, "same dtype"), (dict(v=v.half()), typ, "same dtype"),
        (dict(v=v[:, :5]), val, "k and v must be"), (dict(k=k[:2], v=v[:2]), val, "k and v must be"),
        (dict(k=k[..., :32], v=v[..., :32]), val, "k and v must be"),
        (dict(k=zeros(4, 10, 3, 64), v=zeros(4, 10, 3, 64)), val, "multiple of kv_heads"),
        (dict(k=zeros(4, 10, 0, 64), v=zeros(4, 10, 0, 64)), val, "multiple of kv_heads"),
        (dict(prefix_k=None), val, "needs prefix_k and prefix_v"), (dict(prefix_v=None), val, "needs prefix_k and prefix_v"),
        (dict(prefix_k=None, prefix_v=None, prefix_lens=lens(1)), val, "needs prefix_k and prefix_v"),
        (dict(prefix_k=pk[0]), val, "must be .groups"), (dict(prefix_v=pv[:, :5]), val, "must be .groups"),
        (dict(prefix_k=zeros(2, 6, 4, 64), prefix_v=zeros(2, 6, 4, 64)), val, "must be .groups"),
        (dict(prefix_k=zeros(3, 6, 2, 64), prefix_v=zeros(3, 6, 2, 64)), val, "multiple of the prefix's groups"),
        (dict(prefix_k=zeros(0, 6, 2, 64), prefix_v=zeros(0, 6, 2, 64)), val, "multiple of the prefix's groups"),
        (dict(prefix_k=pk.half()), typ, "prefix_k must be"), (dict(prefix_v=pv.cpu()), val, "device tensors, prefix_v"),
        (dict(prefix_v=zeros(2, 6, 64, 2).transpose(2, 3)), val, "prefix_v must have a contiguous"),
        (dict(q=zeros(4, 3, 64, 4).transpose(2, 3)), val, "q, k, v and o must have a contiguous"),
        (dict(v=zeros(4, 10, 64, 2).transpose(2, 3)), val, "q, k, v and o must have a contiguous"),
        (dict(o=zeros(4, 3, 64, 4).transpose(2, 3)), val, "q, k, v and o must have a contiguous"),
        (dict(o=o[:, :2]), val, "o must have shape"), (dict(o=o.half()), typ, "o must be"),
        (dict(o=x), val, "o must not overlap q"),
        (dict(o=long[:, 9:12, :4], k=long[:, :10, :2]), val, "o must not overlap k"),
        (dict(o=long[:, 9:12, :4], v=long[:, :10, :2]), val, "o must not overlap v"),
        (dict(o=long[:, 5:8, :4], prefix_k=long[:2, :6, :2]), val, "o must not overlap prefix_k"),
        (dict(o=long[:, 5:8, :4], prefix_v=long[:2, :6, :2]), val, "o must not overlap prefix_v"),
        (dict(o=o, prefix_lens=ints(o, 2)), val, "o must not overlap prefix_lens"),
        (dict(o=o, q_lens=ints(o, 4)), val, "o must not overlap q_lens"),
        (dict(o=o, kv_lens=ints(o, 4)), val, "o must not overlap kv_lens"),
        (dict(weight=w[:, :, :9]), val, "weight must have shape"), (dict(weight=w.double()), typ, "weight must be"),
        (dict(weight=zeros(4, 10, 2, dt=torch.float32).transpose(1, 2)), val, "weight must have a contiguous"),
        (dict(weight=w.cpu()), val, "device tensors, weight"),
        (dict(workspace=None), val, "a weight needs a workspace"),
        (dict(o=o, weight=floats(o, 4, 2, 10)), val, "weight must not overlap o"),
        (dict(weight=floats(x, 4, 2, 10)), val, "weight must not overlap q"),
        (dict(weight=floats(k, 4, 2, 10)), val, "weight must not overlap k"),
        (dict(weight=floats(v, 4, 2, 10)), val, "weight must not overlap v"),
        (dict(weight=floats(pk, 4, 2, 10)), val, "weight must not overlap prefix_k"),
        (dict(weight=floats(pv, 4, 2, 10)), val, "weight must not overlap prefix_v"),
        (dict(prefix_lens=ints(w, 2)), val, "weight must not overlap prefix_lens"),
        (dict(q_lens=ints(w, 4)), val, "weight must not overlap q_lens"),
        (dict(kv_lens=ints(w, 4)), val, "weight must not overlap kv_lens"),
        (dict(prefix_lens=lens(4)), val, "prefix_lens must have shape"), (dict(q_lens=lens(3)), val, "q_lens must have shape"),
        (dict(kv_lens=lens(8)[::2]), val, "kv_lens must be contiguous"), (dict(kv_lens=lens(4, torch.int64)), typ, "kv_lens must be"),
        (dict(q_lens=lens(4).cpu()), val, "device tensors, q_lens"),
        (dict(workspace=ws.cpu()), val, "workspace must be"), (dict(workspace=ws[::2]), val, "workspace must be"),
        (dict(mode=7), (KeyError, ValueError), None),
        # the library's own
        (dict(workspace=ws[:16]), None, None), (dict(workspace=ws[8:]), None, None),
        (dict(workspace=long.view(-1).view(torch.uint8), k=long[:, :10, :2]), None, None),
        (dict(o=zeros(1, 3, 4, 64).expand(4, -1, -1, -1)), None, None), (dict(t=0.0), None, None),
        (dict(weight=zeros(4, 1, 10, dt=torch.float32).expand(-1, 2, -1)), None, None),
        (dict(q=zeros(4, 3, 4, 72)[..., 4:68]), None, None),
    ]


def test_shared_refusals(q):  # noqa: F811
    ok, bad = shared_cases()
    q.quake_attention_shared(**ok)
    torch.cuda.synchronize()
    ok["weight"].zero_()
    for kw, error, text in bad:
        with pytest.raises(error or q.QuakeError, match=text):
            q.quake_attention_shared(**dict(ok, **kw))
            pytest.fail("taken: %s %s" % (sorted(kw), text))
    torch.cuda.synchronize()
    assert (ok["weight"] == 0).all()
    for dt, d in ((torch.float32, 64), (torch.bfloat16, 96)):    # formats and head dims the library does not have
        with pytest.raises(q.QuakeError):
            q.quake_attention_shared(*(zeros(1, 1, 1, d, dt=dt) for _ in range(3)))


def evict_cases():
    k, v, w = zeros(3, 10, 2, 64), zeros(3, 10, 2, 64), zeros(3, 2, 10, dt=torch.float32)
    ko, vo, wo, lo = zeros(3, 7, 2, 64), zeros(3, 7, 2, 64), zeros(3, 2, 7, dt=torch.float32), lens(3)
    ok = dict(k=k, v=v, weight=w, budget=5, kv_lens=lens(3), out=(ko, vo, wo, lo))
    val, typ = ValueError, TypeError
    return ok, [
        (dict(k=k[0]), val, "k needs"), (dict(k=k.cpu()), val, "device tensors, k"), (dict(k=k.long()), typ, "k must be"),
        (dict(v=v[:, :9]), val, "v must have shape"), (dict(v=v.half()), typ, "v must be"),
        (dict(weight=w[:, :, :9]), val, "weight must have shape"), (dict(weight=w.half()), typ, "weight must be"),
        (dict(weight=zeros(3, 10, 2, dt=torch.float32).transpose(1, 2)), val, "weight must have a contiguous"),
        (dict(kv_lens=lens(2)), val, "kv_lens must have shape"), (dict(kv_lens=lens(3, torch.int64)), typ, "kv_lens must be"),
        (dict(kv_lens=lens(6)[::2]), val, "kv_lens must be contiguous"),
        (dict(out=(ko, vo)), val, "out must be"), (dict(out=(ko, vo, wo, lo, lo)), val, "out must be"),
        (dict(out=(ko[0], vo, wo)), val, "out's k needs"), (dict(out=(ko, vo[:, :6], wo)), val, "out's v must have shape"),
        (dict(out=(ko[:2], vo[:2], wo)), val, "out's k must have shape"), (dict(out=(ko, vo.half(), wo)), typ, "out's v must be"),
        (dict(out=(ko, vo, wo[:, :, :6])), val, "out's weight must have shape"),
        (dict(out=(ko, vo, wo.double())), typ, "out's weight must be"),
        (dict(out=(ko, vo, zeros(3, 7, 2, dt=torch.float32).transpose(1, 2))), val, "out's weight must have a contiguous"),
        (dict(out=(ko, vo, wo, lens(2))), val, "out's kv_lens must have shape"),
        (dict(out=(ko, vo, wo, lens(3, torch.int64))), typ, "out's kv_lens must be"),
        (dict(out=(zeros(3, 7, 64, 2).transpose(2, 3), vo, wo)), val, "keys and values must have a contiguous"),
        (dict(v=zeros(3, 10, 64, 2).transpose(2, 3)), val, "keys and values must have a contiguous"),
        (dict(kept=zeros(3, 2, 4, dt=torch.int32)), val, "kept must have shape"),
        (dict(kept=zeros(3, 2, 5, dt=torch.int64)), typ, "kept must be"),
        (dict(kept=zeros(3, 5, 2, dt=torch.int32).transpose(1, 2)), val, "kept must be contiguous"),
        (dict(evicted=zeros(2, dt=torch.int32)), val, "evicted must have shape"),
        (dict(evicted=zeros(6, dt=torch.int32)[::2]), val, "evicted must be contiguous"),
        # the library's own
        (dict(budget=0), None, None), (dict(budget=-2), None, None), (dict(budget=8), None, None),
        (dict(sinks=-1), None, None), (dict(sinks=3, recent=3), None, None), (dict(recent=6), None, None),
        (dict(out=(k, zeros(3, 10, 2, 64), zeros(3, 2, 10, dt=torch.float32))), None, None), (dict(out=(ko, ko, wo)), None, None), (dict(out=(ko, vo, floats(ko, 3, 2, 7))), None, None),
        (dict(out=(k[:, 1:8], vo, wo)), None, None), (dict(out=(ko, vo, w[:, :, 1:8])), None, None),
        (dict(out=None, v=k), None, None), (dict(out=(zeros(1, 7, 2, 64).expand(3, -1, -1, -1), vo, wo)), None, None),
        (dict(kept=ints(ko, 30).view(3, 2, 5)), None, None), (dict(kept=ints(w, 30).view(3, 2, 5)), None, None),
        (dict(evicted=ints(vo, 3)), None, None), (dict(evicted=lo), None, None), (dict(out=(ko, vo, wo, ints(k, 3))), None, None),
        (dict(k=zeros(3, 10, 2, 4), v=zeros(3, 10, 2, 4), out=(zeros(3, 7, 2, 4), zeros(3, 7, 2, 4), wo)), None, None),
    ]


def test_evict_refusals(q):  # noqa: F811
    ok, bad = evict_cases()
    kept, evicted = q.quake_cache_evict(**ok)
    torch.cuda.synchronize()
    assert (kept[..., 0] == 0).all() and (kept[..., 1:] == -1).all() and (evicted == 0).all()
    for a in ok["out"]:
        a.fill_(7)
    for kw, error, text in bad:
        with pytest.raises(error or q.QuakeError, match=text):
            q.quake_cache_evict(**dict(ok, **kw))
            pytest.fail("taken: %s %s" % (sorted(kw), text))
    torch.cuda.synchronize()
    assert all((a == 7).all() for a in ok["out"])
