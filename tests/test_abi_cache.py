"""Refusals of quake_attention_shared and quake_cache_evict (CPU: every call below returns
before a HIP call or a launch), their sizes and the binding's own checks."""
import ctypes
import math

import pytest
import torch

from test_abi_decode import A, BIG, caller, q  # noqa: F401 (q: the fixture)

AT = {n: A + (i + 1 << 22) for i, n in enumerate(
    ("q", "pk", "pv", "k", "v", "o", "w", "pl", "ql", "kl", "ko", "vo", "wo", "lo", "kept", "ev"))}


def only(names):
    return {n: AT[n] for n in names.split()}


def shared_strides(**kw):
    s = dict(q=(1024, 256, 64), pk=(6400, 64, 64), pv=(6400, 64, 64), k=(12800, 128, 64), v=(12800, 128, 64),
             o=(1024, 256, 64), w=(200, 100))
    s.update(kw)
    return (ctypes.c_int64 * 20)(*(i for n in ("q", "pk", "pv", "k", "v", "o", "w") for i in s[n]))


SHARED = "q pk pv k v o w pl ql kl batch groups sq sp skv heads kv dim st dt mode t ws nws stream"


def shared(q, **kw):
    return caller(q.lib.quake_attention_shared,
                  dict(only("q pk pv k v o"), w=None, pl=None, ql=None, kl=None, batch=2, groups=1, sq=4, sp=50,
                       skv=100, heads=4, kv=2, dim=64, st=shared_strides(), dt=2, mode=2, t=0.125, ws=None,
                       nws=0, stream=None, **kw), SHARED)


@pytest.mark.parametrize("bad", [
    dict(batch=-2), dict(groups=0), dict(groups=-1), dict(groups=3), dict(batch=3, groups=2), dict(sq=-1),
    dict(sp=-1), dict(skv=-1), dict(heads=0), dict(kv=0), dict(kv=3), dict(dim=32), dict(dim=65), dict(t=0.0),
    dict(t=-1.0), dict(t=math.nan), dict(t=math.inf), dict(t=3e38), dict(q=None), dict(pk=None), dict(pv=None),
    dict(k=None), dict(v=None), dict(o=None), dict(st=None), dict(q=A + 8), dict(pk=A + 2), dict(pv=A + 8),
    dict(k=A + 2), dict(v=A + 4), dict(o=A + 8), dict(w=A + 2), dict(pl=A + 1), dict(ql=A + 2), dict(kl=A + 3),
    dict(ws=A + 4), dict(nws=-1), dict(st=shared_strides(q=(1024, 60, 64))),
    dict(st=shared_strides(k=(64, -64, 64))), dict(st=shared_strides(k=(64, (1 << 24) + 8, 64))),
    dict(st=shared_strides(pk=(0, (1 << 24) + 8, 64))), dict(st=shared_strides(pv=(0, 4, 64))),
    dict(st=shared_strides(o=(1024, 256, 0))), dict(st=shared_strides(o=(0, 256, 64))),
    dict(st=shared_strides(o=(1024, 128, 64))), dict(st=shared_strides(q=(BIG, 256, 64))),
    dict(w=AT["w"]), dict(w=AT["w"], ws=A, nws=8), dict(skv=1 << 30, sp=1), dict(sp=(1 << 30) + 1),
    dict(sq=(1 << 24) + 1), dict(batch=1 << 30), dict(heads=1 << 20, kv=1 << 20),
    dict(batch=1 << 20, sq=1 << 11)], ids=str)
def test_shared_refusals(q, bad):
    assert shared(q)(**bad) == q.EINVAL


def test_shared_weight_refusals(q):
    need = q._size("quake_attention_shared_workspace_size", 2, 1, 4, 50, 100, 4, 2, 64, 1)
    assert need > 0 and need % 16 == 0
    call = shared(q)
    ok = dict(w=AT["w"], ws=A, nws=need)
    assert call(**ok, batch=0) == q.OK
    for bad in (dict(nws=need - 1), dict(st=shared_strides(w=(200, 99))), dict(st=shared_strides(w=(100, 100))),
                dict(st=shared_strides(w=(-200, 100))), dict(st=shared_strides(w=(BIG, 100))), dict(ws=None)):
        assert call(**dict(ok, **bad)) == q.EINVAL, bad
    # 2^24 tiles of 128 slots
    for size in ((1 << 14, 1, 1, 0, 1 << 20, 64, 64, 64, 1), (1 << 10, 1, 1, 0, 1 << 22, 1, 1, 64, 1)):
        with pytest.raises(q.QuakeError):
            q._size("quake_attention_shared_workspace_size", *size)


def test_shared_workspace_sizes(q):
    name = "quake_attention_shared_workspace_size"
    for weigh in (0, 1):
        assert q._size(name, 0, 1, 1, 0, 8, 4, 4, 64, weigh) == 0
        assert q._size(name, 2, 1, 0, 100, 8, 4, 4, 64, weigh) == 0
        assert q._size(name, 2, 1, 1, 0, 0, 4, 4, 64, weigh) == 0          # no keys at all
        assert q._size(name, 2, 1, 200, 0, 0, 4, 4, 64, weigh) == 0
        assert q._size(name, 1, 1, 1, 5, 0, 4, 4, 64, weigh) == 0
        for size in ((64, 1, 1, 8192, 1024, 32, 8, 128), (5, 5, 7, 300, 0, 8, 1, 64), (1, 1, 1, 1 << 20, 9, 128, 1, 128),
                     (1 << 20, 1, 1, 64, 64, 1, 1, 64), (3, 1, 500, 1, 500, 7, 7, 64), (1, 1, 1, 1 << 29, 1 << 29, 1, 1, 64)):
            assert q._size(name, *size, weigh) % 16 == 0
    assert q._size(name, 4, 1, 1, 500, 64, 8, 2, 64, 0) == 0               # brief: no second launch


def test_shared_formats_modes_and_empty_calls(q):
    call = shared(q)
    assert call(dt=0) == q.EDTYPE and call(dt=7) == q.EDTYPE and call(mode=4) == q.EMODE
    none = dict(q=None, pk=None, pv=None, k=None, v=None, o=None)
    assert call(batch=0, **none) == q.OK and call(sq=0, **none) == q.OK


@pytest.mark.parametrize("name,size", [("q", 2 * 2048), ("o", 2 * 2048), ("pk", 2 * 50 * 128), ("pv", 2 * 50 * 128),
                                       ("k", 2 * 25600), ("v", 2 * 25600), ("w", 4 * 400), ("pl", 4), ("ql", 8),
                                       ("kl", 8)])
def test_shared_workspaces_apart(q, name, size):
    need = q._size("quake_attention_shared_workspace_size", 2, 1, 4, 50, 100, 4, 2, 64, 1)
    call = shared(q)
    kw = dict(only("w pl ql kl"), st=shared_strides(pk=(0, 128, 64), pv=(0, 128, 64)))
    at = AT[name]
    for ws in {at, at - need + 16, (at + size - 1) & ~15, (at + size // 2) & ~15}:
        assert call(**kw, ws=ws, nws=need) == q.EINVAL, (name, hex(ws))


def evict_strides(**kw):
    s = dict(k=(12800, 128, 64), v=(12800, 128, 64), ko=(7680, 128, 64), vo=(7680, 128, 64), w=(200, 100),
             wo=(120, 60))
    s.update(kw)
    return (ctypes.c_int64 * 16)(*(i for n in ("k", "v", "ko", "vo", "w", "wo") for i in s[n]))


EVICT = "k v w kl ko vo wo lo kept ev batch skv slots kv dim st budget sinks recent dt stream"


def evict(q):
    return caller(q.lib.quake_cache_evict,
                  dict(only("k v w kl ko vo wo lo kept ev"), batch=2, skv=100, slots=60, kv=2, dim=64,
                       st=evict_strides(), budget=50, sinks=4, recent=10, dt=2, stream=None), EVICT)


IN_PLACE = dict(ko=AT["k"], vo=AT["v"], wo=AT["w"], lo=AT["kl"], slots=100,
                st=evict_strides(ko=(12800, 128, 64), vo=(12800, 128, 64), wo=(200, 100)))


@pytest.mark.parametrize("bad", [
    dict(batch=-1), dict(skv=-1), dict(kv=0), dict(dim=0), dict(dim=4), dict(dim=4104), dict(slots=49),
    dict(budget=0), dict(budget=-3), dict(budget=61), dict(sinks=-1), dict(recent=-1), dict(sinks=51),
    dict(sinks=20, recent=31), dict(k=None), dict(v=None), dict(w=None), dict(ko=None), dict(vo=None),
    dict(wo=None), dict(kept=None), dict(ev=None), dict(st=None), dict(k=A + 8), dict(v=A + 2), dict(ko=A + 8),
    dict(vo=A + 4), dict(w=A + 2), dict(wo=A + 1), dict(kl=A + 2), dict(lo=A + 1), dict(kept=A + 2),
    dict(ev=A + 3), dict(batch=1 << 21), dict(batch=1 << 12, kv=1 << 12), dict(skv=(1 << 30) + 1),
    dict(slots=(1 << 30) + 1), dict(st=evict_strides(k=(12800, 4, 64))), dict(st=evict_strides(v=(-64, 128, 64))),
    dict(st=evict_strides(ko=(7680, 64, 64))), dict(st=evict_strides(vo=(7680, 128, 0))),
    dict(st=evict_strides(w=(-1, 100))), dict(st=evict_strides(wo=(60, 60))), dict(st=evict_strides(k=(BIG, 128, 64))),
    dict(st=evict_strides(wo=(BIG, 60))),
    # an output that meets another operand
    dict(ko=AT["k"]), dict(vo=AT["v"]), dict(wo=AT["w"]), dict(ko=AT["v"]), dict(vo=AT["k"] + 16),
    dict(ko=AT["vo"]), dict(ko=AT["vo"] + 64), dict(wo=AT["ko"]), dict(wo=AT["w"] + 4), dict(kept=AT["k"]),
    dict(kept=AT["w"]), dict(kept=AT["vo"]), dict(kept=AT["kl"]), dict(kept=AT["ev"]), dict(ev=AT["wo"]),
    dict(ev=AT["kl"] + 4), dict(ev=AT["lo"]), dict(lo=AT["kl"] + 4), dict(lo=AT["ko"]), dict(lo=AT["k"] + 16),
    dict(kl=AT["ko"]), dict(kl=AT["kept"]),
    # in place in part, or with other slots or strides
    dict(IN_PLACE, ko=AT["ko"]), dict(IN_PLACE, vo=AT["vo"]), dict(IN_PLACE, wo=AT["wo"]),
    dict(IN_PLACE, slots=99), dict(IN_PLACE, st=evict_strides(ko=(12800, 128, 64), vo=(12800, 128, 64), wo=(240, 100))),
    dict(IN_PLACE, st=evict_strides(ko=(25600, 128, 64), vo=(12800, 128, 64), wo=(200, 100))),
    dict(IN_PLACE, v=AT["k"], vo=AT["k"]), dict(IN_PLACE, v=AT["k"] + 64, vo=AT["k"] + 64)], ids=str)
def test_evict_refusals(q, bad):
    assert evict(q)(**bad) == q.EINVAL


def test_evict_formats_and_empty_calls(q):
    call = evict(q)
    assert call(dt=3) == q.EDTYPE and call(dt=-1) == q.EDTYPE
    assert call(batch=0, k=None, v=None, w=None, ko=None, vo=None, wo=None, kept=None, ev=None) == q.OK


def test_binding_refuses(q):
    x = torch.zeros(1, 2, 2, 64, dtype=torch.bfloat16)
    w = torch.zeros(1, 2, 2)
    with pytest.raises(ValueError):
        q.quake_attention_shared(x, x, x)
    with pytest.raises(ValueError):
        q.quake_cache_evict(x, x, w, 1)
    for args in ((-1, 1, 1, 0, 8, 4, 4, 64, 0), (2, 1, 1, 0, 8, 4, 3, 64, 0), (2, 1, 1, 0, 8, 4, 4, 96, 0)):
        with pytest.raises(q.QuakeError):
            q._size("quake_attention_shared_workspace_size", *args)
    assert q.lib.quake_attention_shared_workspace_size(1, 1, 1, 0, 8, 4, 4, 64, 0, None) == q.EINVAL
