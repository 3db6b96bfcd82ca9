"""Refusals of quake_attention_window, quake_sample and quake_distill (CPU: every
call below returns before a HIP call or a launch), their workspace sizes and the
binding's own checks."""
import ctypes
import math
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x10000                      # 16-byte aligned, never dereferenced
BIG = 1 << 62


@pytest.fixture(scope="module")
def q():
    if not os.path.exists(os.path.join(ROOT, "paper_2412_00408_amd", "libquake.so")):
        pytest.fail("libquake.so is not built; run python -m paper_2412_00408_amd.build")
    from paper_2412_00408_amd import quake
    return quake


def caller(fn, defaults, names):
    def call(**kw):
        a = dict(defaults, **kw)
        return fn(*(a[n] for n in names.split()))
    return call


def strides(**kw):
    s = dict(q=(64, 64, 64), k=(6400, 64, 64), v=(6400, 64, 64), o=(64, 64, 64))
    s.update(kw)
    return (ctypes.c_int64 * 12)(*s["q"], *s["k"], *s["v"], *s["o"])


WINDOW = "q k v o ql kl batch sq skv heads kv dim st window sinks dt mode t ws nws stream"


def window(q):
    return caller(q.lib.quake_attention_window,
                  dict(q=A, k=A, v=A, o=A, ql=None, kl=None, batch=2, sq=4, skv=100, heads=4, kv=2,
                       dim=64, st=strides(), window=10, sinks=2, dt=2, mode=2, t=0.125, ws=None,
                       nws=0, stream=None), WINDOW)


@pytest.mark.parametrize("bad", [
    dict(batch=-1), dict(sq=-1), dict(skv=-1), dict(heads=0), dict(kv=0), dict(kv=3), dict(dim=32),
    dict(dim=65), dict(window=0), dict(window=-4), dict(window=1 << 31), dict(sinks=-1),
    dict(sinks=1 << 31), dict(t=0.0), dict(t=-1.0), dict(t=math.nan), dict(t=math.inf), dict(t=3e38),
    dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(st=None), dict(q=A + 8),
    dict(k=A + 2), dict(v=A + 4), dict(o=A + 8), dict(ql=A + 2), dict(kl=A + 1), dict(ws=A + 4),
    dict(nws=-1), dict(st=strides(q=(64, 60, 64))), dict(st=strides(k=(64, -64, 64))),
    dict(st=strides(k=(64, (1 << 24) + 8, 64))), dict(st=strides(v=(64, (1 << 24) + 8, 64))),
    dict(st=strides(o=(-8, 64, 64))), dict(st=strides(v=(4, 64, 64))),
    dict(st=strides(o=(64, 64, 3))), dict(st=strides(o=(64, 64, 0))), dict(st=strides(o=(0, 64, 64))),
    dict(st=strides(o=(64, 56, 64))), dict(st=strides(q=(BIG, 64, 64))), dict(skv=(1 << 30) + 1),
    dict(sq=(1 << 24) + 1), dict(batch=1 << 30), dict(heads=1 << 20, kv=1 << 20)], ids=str)
def test_window_refusals(q, bad):
    assert window(q)(**bad) == q.EINVAL


def test_window_formats_modes_and_empty_calls(q):
    call = window(q)
    assert call(dt=0) == q.EDTYPE and call(dt=7) == q.EDTYPE and call(mode=4) == q.EMODE
    assert call(batch=0, q=None, k=None, v=None, o=None) == q.OK
    assert call(sq=0, q=None, o=None) == q.OK
    # strides of sizes of one are never used
    one = strides(q=(3, -5, 64), o=(1, 1, 64), k=(7, 64, -1), v=(-9, 64, 2))
    assert call(batch=1, sq=1, kv=1, heads=1, st=one, ws=A, nws=-1) == q.EINVAL   # the workspace
    # a workspace that is too small
    n = q._size("quake_attention_window_workspace_size", 1, 1, 5000, 8, 1, 64, 5000, 0)
    assert n > 0
    st = strides(q=(512, 512, 64), o=(512, 512, 64))
    assert call(batch=1, sq=1, skv=5000, heads=8, kv=1, window=5000, st=st, ws=A, nws=n - 1) == q.EINVAL


def test_workspace_sizes(q):
    size = q._size
    w = "quake_attention_window_workspace_size"
    assert size(w, 64, 1, 8192, 32, 8, 128, 4096, 4) == 0          # fills the GPU without splits
    assert size(w, 0, 1, 100, 4, 4, 64, 10, 0) == 0
    assert size(w, 1, 1, 40, 4, 4, 64, 2 ** 31 - 1, 2 ** 31 - 1) == 0
    for args in ((1, 1, 10, 4, 3, 64, 10, 0), (1, 1, 10, 4, 4, 96, 10, 0), (1, 1, 10, 4, 4, 64, 0, 0)):
        with pytest.raises(q.QuakeError):
            size(w, *args)
    assert q.lib.quake_attention_window_workspace_size(1, 1, 10, 4, 4, 64, 10, 0, None) == q.EINVAL
    for fn in ("quake_sample_workspace_size", "quake_distill_workspace_size"):
        assert size(fn, 0, 1000) == 0 and size(fn, 4, 0) == 0
        assert size(fn, 4, 128256) % 8 == 0
        for args in ((-1, 10), (10, -1), (1, 1 << 40)):
            with pytest.raises(q.QuakeError):
                size(fn, *args)
        assert getattr(q.lib, fn)(1, 10, None) == q.EINVAL
    assert size("quake_distill_workspace_size", 4096, 128256) == 0
    assert size("quake_distill_workspace_size", 4, 128256) > 0


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(cols=-1), dict(cols=0), dict(cols=(1 << 22) + 1, ldx=1 << 23), dict(ldx=99),
    dict(x=None), dict(u=None), dict(token=None), dict(x=A + 2), dict(u=A + 2), dict(token=A + 1),
    dict(prob=A + 2), dict(temp=A + 3), dict(k=A + 2), dict(p=A + 2), dict(m=A + 1), dict(ws=A + 8),
    dict(nws=-1), dict(rows=1 << 31), dict(ldx=BIG)], ids=str)
def test_sample_refusals(q, bad):
    names = "x u token prob rows cols ldx temp k p m dt mode ws nws stream"
    call = caller(q.lib.quake_sample,
                  dict(x=A, u=A, token=A, prob=A, rows=4, cols=100, ldx=100, temp=None, k=None, p=None,
                       m=None, dt=0, mode=2, ws=None, nws=0, stream=None), names)
    assert call(**bad) == q.EINVAL
    assert call(dt=3) == q.EDTYPE and call(mode=-1) == q.EMODE
    assert call(rows=0, x=None, u=None, token=None) == q.OK
    need = q._size("quake_sample_workspace_size", 4, 128256)
    if need:
        assert call(cols=128256, ldx=128256, ws=A, nws=need - 1) == q.EINVAL


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(cols=-1), dict(cols=0), dict(cols=(1 << 30) + 1, ldx=1 << 31, ldg=1 << 31),
    dict(k=-1), dict(k=1025, ldi=2000, ldy=2000), dict(ldx=99), dict(ldi=9), dict(ldy=9), dict(ldg=99),
    dict(x=None), dict(idx=None), dict(y=None), dict(x=A + 1), dict(idx=A + 2), dict(y=A + 2),
    dict(w=A + 2), dict(stats=A + 1), dict(grad=A + 1), dict(t=0.0), dict(t=-2.0), dict(t=math.nan),
    dict(t=math.inf), dict(t=1e38), dict(rows=1 << 31), dict(ldx=BIG), dict(ldi=BIG)], ids=str)
def test_distill_refusals(q, bad):
    args = dict(x=A, idx=A, y=A, w=A, loss=A, stats=A, grad=A, rows=4, cols=100, k=10, ldx=100, ldi=10,
                ldy=10, ldg=100, dt=2, ydt=0, mode=2, t=1.0, ws=None, nws=0, stream=None)
    both = "rows cols k ldx ldi ldy ldg dt ydt mode t"
    loss = caller(q.lib.quake_distill, args, "x idx y w loss stats grad %s ws nws stream" % both)
    grad = caller(q.lib.quake_distill_grad, args, "x idx y stats w grad %s stream" % both)
    for call in (loss, grad):
        assert call(**bad) == q.EINVAL
        assert call(dt=5) == q.EDTYPE and call(ydt=-1) == q.EDTYPE and call(mode=9) == q.EMODE
        assert call(rows=0, x=None, idx=None, y=None) == q.OK
    assert loss(loss=None) == q.EINVAL and loss(loss=A + 2) == q.EINVAL and loss(ws=A + 8) == q.EINVAL
    assert loss(nws=-1) == q.EINVAL
    need = q._size("quake_distill_workspace_size", 4, 128256)
    assert loss(cols=128256, ldx=128256, ldg=128256, ws=A, nws=need - 1) == q.EINVAL
    assert grad(stats=None) == q.EINVAL and grad(grad=None) == q.EINVAL


def test_binding_refuses_host_tensors(q):
    x = torch.zeros(1, 2, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        q.quake_attention_window(x, x, x, window=4)
    l, i = torch.zeros(2, 8), torch.zeros(2, 3, dtype=torch.int32)
    with pytest.raises(ValueError):
        q.quake_sample(l, torch.zeros(2))
    with pytest.raises(ValueError):
        q.quake_distill(l, i, torch.zeros(2, 3))
    with pytest.raises(ValueError):
        q.quake_distill_grad(l, i, torch.zeros(2, 3), torch.zeros(2, 2))
